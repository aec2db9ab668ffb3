"""Binding of the serving operators (include/tsq_cache.h): a key/value cache held in 8 bits and what fills and
reads it.  Argument marshalling and checks only; every step runs in the HIP kernels of libtsq.so.

A step of one layer, for requests of any lengths, new or going on:

    c = Cache(blocks, 16, q_heads, kv_heads, head_dim, "bf16", max_blocks)
    memory, table = c.new_memory(), c.new_table(requests)
    ring, counters, lengths = c.new_ring(), c.new_counters(), c.new_lengths(requests)
    s = c.schedule(new, lengths, table, ring, counters, c.new_schedule(requests, tokens))
    q, k = c.norm_rotate(q, k, s.positions, angles, q_weight, k_weight)
    c.append(memory, k, v, s.slots)
    out = c.attend(memory, q, table, s.starts, s.lengths, max_new, max_length)
    lengths, counters = s.lengths, s.counters         # what the next step begins with

All calls run on torch's current stream, and their tensors are on its device.  A tensor that is left out is allocated on it.
"""
from __future__ import annotations

import ctypes as C

from . import tsq
from .tsq import TSQ_OK, TsqError

TSQ_PAIRS_HALVES, TSQ_PAIRS_NEIGHBOURS = 0, 1
_MOST = 2 ** 32 - 1                                       # (ctypes passes the lower 32 bits of what is larger)

EXPORTS = ("tsq_cache_create", "tsq_cache_destroy", "tsq_cache_memory_sizes", "tsq_cache_schedule", "tsq_cache_norm_rotate",
           "tsq_cache_append", "tsq_cache_gather", "tsq_cache_attend", "tsq_cache_attend_workspace_bytes")


class tsq_cache_config(C.Structure):
    _fields_ = [("blocks", C.c_uint32), ("block_tokens", C.c_uint32), ("q_heads", C.c_uint32), ("kv_heads", C.c_uint32),
                ("head_dim", C.c_uint32), ("dtype", C.c_int32), ("max_blocks", C.c_uint32), ("reserved", C.c_uint32)]


class tsq_cache_memory(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("d_k", "d_v", "d_k_scale", "d_v_scale")]


class tsq_cache_sizes(C.Structure):
    _fields_ = [("code_bytes", C.c_uint64), ("scale_bytes", C.c_uint64)]


_lib = None


def lib():
    """libtsq.so with the argument types of tsq_cache.h set.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        L = tsq.lib()
        vp, u32, i32, u64, f32, st = C.c_void_p, C.c_uint32, C.c_int32, C.c_uint64, C.c_float, C.c_int
        mem = C.POINTER(tsq_cache_memory)
        for name, res, args in (
                ("tsq_cache_create", st, [C.POINTER(tsq_cache_config), C.POINTER(vp)]),
                ("tsq_cache_destroy", None, [vp]),
                ("tsq_cache_memory_sizes", st, [vp, C.POINTER(tsq_cache_sizes)]),
                ("tsq_cache_schedule", st, [vp, u32, vp, vp, vp, vp, vp, u32, vp, vp, vp, vp, vp, vp, vp]),
                ("tsq_cache_norm_rotate", st, [vp, u32, vp, u64, vp, u64, vp, vp, u32, u32, i32, vp, vp, f32, vp, u64, vp, u64, vp]),
                ("tsq_cache_append", st, [vp, mem, u32, vp, u64, vp, u64, vp, vp]),
                ("tsq_cache_gather", st, [vp, mem, u32, vp, vp, vp, u32, vp, u64, vp, u64, vp]),
                ("tsq_cache_attend", st, [vp, mem, u32, vp, vp, vp, u32, u32, u32, vp, u64, f32, i32, u32, vp, u64, vp, vp, vp]),
                ("tsq_cache_attend_workspace_bytes", C.c_size_t, [vp, u32, u32, u32, u32, u32])):
            getattr(L, name).restype = res
            getattr(L, name).argtypes = args
        _lib = L
    return _lib


# ------------------------------------------------------------------ the C entry points that give back a value, same names

def _done(status: int, what: str) -> None:
    if status != TSQ_OK:
        raise TsqError(status, what)


def tsq_cache_create(cfg: tsq_cache_config) -> int:
    """-> opaque handle (int).  Raises TsqError on a rejected configuration."""
    h = C.c_void_p()
    _done(lib().tsq_cache_create(C.byref(cfg), C.byref(h)), "tsq_cache_create")
    return h.value


def tsq_cache_destroy(cache: int) -> None:
    lib().tsq_cache_destroy(cache)


def tsq_cache_memory_sizes(cache: int) -> tsq_cache_sizes:
    out = tsq_cache_sizes()
    _done(lib().tsq_cache_memory_sizes(cache, C.byref(out)), "tsq_cache_memory_sizes")
    return out


def tsq_cache_attend_workspace_bytes(cache: int, requests: int, tokens: int, max_new: int, max_length: int, window: int = 0) -> int:
    return int(lib().tsq_cache_attend_workspace_bytes(cache, requests, tokens, max_new, max_length, window))


# ------------------------------------------------------------------ convenience over torch tensors

class Memory:
    """The four tensors of one cache, and the C structure that holds their pointers: k int8 [blocks, kv_heads, block_tokens,
    head_dim], v int8 [blocks, kv_heads, head_dim, block_tokens], scales float32 [blocks, kv_heads].  They are looked at once,
    here, and stay what they are; a cache takes a memory of its own shape only."""

    def __init__(self, k, v, k_scale, v_scale):
        import torch
        shape = tuple(k.shape)
        n, h, b, d = shape if len(shape) == 4 else (0, 0, 0, 0)
        device = k.get_device()
        for x, size, kind in ((k, (n, h, b, d), torch.int8), (v, (n, h, d, b), torch.int8), (k_scale, (n, h), torch.float32), (v_scale, (n, h), torch.float32)):
            if not (x.is_cuda and x.get_device() == device and x.is_contiguous() and tuple(x.shape) == size and x.dtype == kind):
                _refuse("a cache's tensor is %s on one GPU, contiguous, %s" % (size, kind))
        c = tsq_cache_memory(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())
        self.__dict__.update(k=k, v=v, k_scale=k_scale, v_scale=v_scale, shape=shape, device=device, c=c, ref=C.byref(c))

    def __setattr__(self, name, value):
        raise AttributeError("a memory's tensors are not replaced")


class Schedule:
    """What one step's schedule is written to (see tsq_cache_schedule): made by Cache.new_schedule, and kept by a program as it
    keeps the cache's memory.  Its tensors are looked at once, here, and stay what they are."""

    def __init__(self, lengths, counters, starts, positions, slots, status):
        import torch
        n, capacity, device = lengths.numel(), slots.numel(), lengths.get_device()
        for x, kind, size in ((lengths, torch.int32, n), (counters, torch.int64, 2), (starts, torch.int32, n + 1), (positions, torch.int32, capacity),
                              (slots, torch.int32, capacity), (status, torch.int32, 1)):
            if not (x.is_cuda and x.get_device() == device and x.is_contiguous() and x.dtype is kind and x.numel() == size):
                _refuse("a schedule's tensors are those of Cache.new_schedule")
        self.__dict__.update(lengths=lengths, counters=counters, starts=starts, positions=positions, slots=slots, status=status, requests=n,
                             capacity=capacity, device=device, pointers=tuple(x.data_ptr() for x in (lengths, counters, starts, positions, slots, status)))

    def __setattr__(self, name, value):
        raise AttributeError("a schedule's tensors are not replaced")

    def check(self) -> None:
        """Raises TsqError if the step could not be taken.  Synchronizes."""
        _done(int(self.status.item()), "tsq_cache_schedule")


def _refuse(what: str):
    raise ValueError(what)


def _device() -> int:
    """Number of the current device, whose stream the calls use."""
    global _device
    import torch
    _device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return _device()


class Cache:
    """One tsq_cache plus helpers that allocate torch buffers, check them and pass their pointers."""

    def __init__(self, blocks: int, block_tokens: int, q_heads: int, kv_heads: int, head_dim: int, dtype: str, max_blocks: int):
        import torch
        if dtype not in tsq._DTYPES:
            _refuse("dtype is 'f16' or 'bf16'")
        numbers = (blocks, block_tokens, q_heads, kv_heads, head_dim, max_blocks)
        if min(numbers) < 0 or max(numbers) > _MOST:
            _refuse("a cache's numbers are not negative, and have 32 bits")
        self.kind = torch.float16 if dtype == "f16" else torch.bfloat16
        self.int32, self.int64, self.float32 = torch.int32, torch.int64, torch.float32
        self.blocks, self.block_tokens, self.q_heads, self.kv_heads = blocks, block_tokens, q_heads, kv_heads
        self.head_dim, self.dtype, self.max_blocks = head_dim, dtype, max_blocks
        self.shape = (blocks, kv_heads, block_tokens, head_dim)
        self.cfg = tsq_cache_config(blocks, block_tokens, q_heads, kv_heads, head_dim, tsq._DTYPES[dtype], max_blocks, 0)
        self.handle = tsq_cache_create(self.cfg)
        self._torch, self._lib = torch, lib()

    def __del__(self):
        h = getattr(self, "handle", None)
        if h and tsq_cache_destroy is not None:
            tsq_cache_destroy(h)
            self.handle = None

    @staticmethod
    def _stream() -> int:
        return (tsq._current_stream or tsq.Plan._stream)()

    # -------------------------------------------------------------- buffers

    def _empty(self, shape, kind):
        return self._torch.empty(shape, dtype=kind, device="cuda")

    def new_memory(self) -> Memory:
        t = self._torch
        n, h, b, d = self.blocks, self.kv_heads, self.block_tokens, self.head_dim
        return Memory(self._empty((n, h, b, d), t.int8), self._empty((n, h, d, b), t.int8),
                      self._empty((n, h), t.float32), self._empty((n, h), t.float32))

    def wrap(self, k, v, k_scale, v_scale) -> Memory:
        """A cache in tensors that are there: k [blocks, kv_heads, block_tokens, head_dim] int8,
        v [blocks, kv_heads, head_dim, block_tokens] int8, scales [blocks, kv_heads] float32."""
        memory = Memory(k, v, k_scale, v_scale)
        self._memory(memory, memory.device)
        return memory

    def new_table(self, requests: int):
        return self._torch.full((requests, self.max_blocks), -1, dtype=self.int32, device="cuda")

    def new_ring(self):
        return self._torch.arange(self.blocks, dtype=self.int32, device="cuda")

    def new_counters(self):
        return self._torch.tensor([0, self.blocks], dtype=self.int64, device="cuda")

    def new_lengths(self, requests: int):
        return self._torch.zeros(requests, dtype=self.int32, device="cuda")

    def new_schedule(self, requests: int, tokens: int) -> Schedule:
        e, i32 = self._empty, self.int32
        return Schedule(e(requests, i32), e(2, self.int64), e(requests + 1, i32), e(tokens, i32), e(tokens, i32), e(1, i32))

    # -------------------------------------------------------------- checks

    # (a step calls these for every tensor of every operator: what a tensor holds is told by its type, place and number
    # of elements, and its shape is looked at only where it is not contiguous; `device` is the current one)

    def _memory(self, memory, device):
        if memory.device == device and memory.shape == self.shape:
            return memory.ref
        _refuse("the memory is that of a cache of %s on device %d, this one is %s, the current device %d (blocks, kv_heads, block_tokens, head_dim)"
                % (memory.shape, memory.device, self.shape, device))

    def _ints(self, x, n, what, device):
        if not (x.dtype is self.int32 and x.get_device() == device and x.numel() == n and x.is_contiguous()):
            _refuse("%s is int32 on the current GPU, contiguous, %d elements" % (what, n))
        return x.data_ptr()

    def _requests(self, table, starts, lengths, n, device):
        i32 = self.int32
        if not (table.dtype is i32 and starts.dtype is i32 and lengths.dtype is i32 and
                table.get_device() == device and starts.get_device() == device and lengths.get_device() == device and
                table.is_contiguous() and starts.is_contiguous() and lengths.is_contiguous() and
                table.numel() == n * self.max_blocks and starts.numel() == n + 1):
            _refuse("table, starts and lengths are int32 on the current GPU, contiguous, [%d, %d], [%d] and [%d]" % (n, self.max_blocks, n + 1, n))
        return table.data_ptr(), starts.data_ptr(), lengths.data_ptr()

    def _rows(self, x, tokens, heads, what, device):
        """x: [tokens, heads, head_dim], or [tokens, heads * head_dim]; rows anywhere, the heads of a row together.
        -> pointer, elements from row to row."""
        width = heads * self.head_dim
        if x.dtype is self.kind and x.get_device() == device and x.numel() == tokens * width:
            if x.is_contiguous():
                return x.data_ptr(), width
            shape, stride = x.shape, x.stride()
            if shape[0] == tokens and ((len(shape) == 3 and shape[1] == heads and stride[2] == 1 and (heads == 1 or stride[1] == self.head_dim)) or
                                       (len(shape) == 2 and stride[1] == 1)):
                return x.data_ptr(), (stride[0] if tokens > 1 else width)
        _refuse("%s is [%d, %d, %d] of %s on the current GPU, the heads of a row together" % (what, tokens, heads, self.head_dim, self.kind))

    def _into(self, x, tokens, heads, what, device):
        x = self._empty((tokens, heads, self.head_dim), self.kind) if x is None else x
        return (x,) + self._rows(x, tokens, heads, what, device)

    def _weight(self, w, device):
        if w is None:
            return None
        if not (w.dtype is self.kind and w.get_device() == device and w.is_contiguous() and w.numel() == self.head_dim):
            _refuse("a norm's weight is [head_dim] of the cache's dtype on the current GPU, contiguous")
        return w.data_ptr()

    # -------------------------------------------------------------- the operators

    def schedule(self, new, lengths, table, ring, counters, out: Schedule) -> Schedule:
        """Block tables, slots and positions of a step: new [requests] int32 new tokens of each request (-1: done),
        lengths [requests] int32 what it has.  table and ring are updated; the rest is written to `out`
        (from new_schedule(requests, most new tokens of a step))."""
        n, i32, device = new.numel(), self.int32, _device()
        if not (new.dtype is i32 and lengths.dtype is i32 and table.dtype is i32 and ring.dtype is i32 and counters.dtype is self.int64 and
                new.get_device() == device and lengths.get_device() == device and table.get_device() == device and ring.get_device() == device and
                counters.get_device() == device and out.device == device and
                new.is_contiguous() and lengths.is_contiguous() and table.is_contiguous() and ring.is_contiguous() and counters.is_contiguous() and
                lengths.numel() == n and table.numel() == n * self.max_blocks and ring.numel() == self.blocks and counters.numel() == 2 and
                out.requests == n):
            _refuse("on the current GPU and contiguous: new, lengths int32 [%d], table int32 [%d, %d], ring int32 [%d], counters int64 [2], and a "
                    "schedule of as many requests" % (n, n, self.max_blocks, self.blocks))
        status = self._lib.tsq_cache_schedule(self.handle, n, new.data_ptr(), lengths.data_ptr(), table.data_ptr(), ring.data_ptr(),
                                              counters.data_ptr(), out.capacity, *out.pointers, self._stream())
        if status:
            raise TsqError(status, "tsq_cache_schedule")
        return out

    def norm_rotate(self, q, k, positions, angles, q_weight=None, k_weight=None, eps: float = 1e-6, pairs: str = "halves",
                    q_out=None, k_out=None):
        """RMS norm of each head of q [tokens, q_heads, head_dim] and k [tokens, kv_heads, head_dim] (weights [head_dim],
        or None: no norm), then the rotation by position: angles [rows, rotary] float32 holds the cosines of a
        position's rotary / 2 angles, then their sines.  q_out, k_out may be q, k themselves."""
        tokens, device = q.shape[0], _device()
        qp, qs = self._rows(q, tokens, self.q_heads, "q", device)
        kp, ks = self._rows(k, tokens, self.kv_heads, "k", device)
        q_out, qo, qos = self._into(q_out, tokens, self.q_heads, "q_out", device)
        k_out, ko, kos = self._into(k_out, tokens, self.kv_heads, "k_out", device)
        if not (angles.dtype is self.float32 and angles.get_device() == device and angles.is_contiguous() and angles.dim() == 2):
            _refuse("angles is float32 [rows, rotary] on the current GPU, contiguous")
        if pairs != "halves" and pairs != "neighbours":
            _refuse("pairs is 'halves' or 'neighbours'")
        known, rotary = angles.shape
        status = self._lib.tsq_cache_norm_rotate(
            self.handle, tokens, qp, qs, kp, ks, self._ints(positions, tokens, "positions", device), angles.data_ptr(), known, rotary,
            TSQ_PAIRS_HALVES if pairs == "halves" else TSQ_PAIRS_NEIGHBOURS, self._weight(q_weight, device), self._weight(k_weight, device),
            eps, qo, qos, ko, kos, self._stream())
        if status:
            raise TsqError(status, "tsq_cache_norm_rotate")
        return q_out, k_out

    def append(self, memory: Memory, k, v, slots) -> None:
        """Stores k and v [tokens, kv_heads, head_dim] at slots [tokens] int32 (from a schedule; -1: not stored)."""
        tokens, device = k.shape[0], _device()
        kp, ks = self._rows(k, tokens, self.kv_heads, "k", device)
        vp, vs = self._rows(v, tokens, self.kv_heads, "v", device)
        status = self._lib.tsq_cache_append(self.handle, self._memory(memory, device), tokens, kp, ks, vp, vs,
                                            self._ints(slots, tokens, "slots", device), self._stream())
        if status:
            raise TsqError(status, "tsq_cache_append")

    def gather(self, memory: Memory, table, starts, lengths, k_out, v_out):
        """The last starts[r + 1] - starts[r] tokens of each request r, up to lengths[r], into rows starts[r] ... of k_out
        and v_out [tokens, kv_heads, head_dim] (or [tokens, kv_heads * head_dim], as Plan.compress_batch takes them)."""
        tokens, n, device = k_out.shape[0], lengths.numel(), _device()
        kp, ks = self._rows(k_out, tokens, self.kv_heads, "k_out", device)
        vp, vs = self._rows(v_out, tokens, self.kv_heads, "v_out", device)
        status = self._lib.tsq_cache_gather(self.handle, self._memory(memory, device), n, *self._requests(table, starts, lengths, n, device), tokens,
                                            kp, ks, vp, vs, self._stream())
        if status:
            raise TsqError(status, "tsq_cache_gather")
        return k_out, v_out

    def new_workspace(self, requests: int, tokens: int, max_new: int, max_length: int, window: int = 0):
        """A workspace for attend calls of these numbers on one stream; None where they need none."""
        n = tsq_cache_attend_workspace_bytes(self.handle, requests, tokens, min(max_new, _MOST), min(max_length, _MOST), min(window, _MOST))
        return self._empty(n, self._torch.uint8) if n else None

    def attend(self, memory: Memory, q, table, starts, lengths, max_new: int, max_length: int, scale=None, causal: bool = True,
               window: int = 0, out=None, lse=None, ws=None):
        """Attention of q [tokens, q_heads, head_dim] over the cache: rows starts[r] .. starts[r + 1] - 1 are the last tokens of
        request r, which has lengths[r] in the cache.  max_new, max_length: the largest of both over the requests (how the
        work is split goes by them).  scale: 1 / sqrt(head_dim) if left out.  lse: float32 [tokens, q_heads] to be written."""
        tokens, n, device = q.shape[0], lengths.numel(), _device()
        qp, qs = self._rows(q, tokens, self.q_heads, "q", device)
        out, op, os_ = self._into(out, tokens, self.q_heads, "out", device)
        lp = None
        if lse is not None:
            if not (lse.dtype is self.float32 and lse.get_device() == device and lse.is_contiguous() and lse.numel() == tokens * self.q_heads):
                _refuse("lse is float32 [tokens, q_heads] on the current GPU, contiguous")
            lp = lse.data_ptr()
        if not (0 <= max_new <= 0xFFFFFFFF and 0 <= max_length <= 0xFFFFFFFF and 0 <= window <= 0xFFFFFFFF):
            if max_new < 0 or max_length < 0 or window < 0:
                _refuse("max_new, max_length and window are not negative")
            # (no request is as long: what is larger says the same)
            max_new, max_length, window = min(max_new, _MOST), min(max_length, _MOST), min(window, _MOST)
        L, wp = self._lib, None
        # (256 tokens are never cut, and then there is no workspace)
        need = 0 if max_length <= 256 else L.tsq_cache_attend_workspace_bytes(self.handle, n, tokens, max_new, max_length, window)
        if need:
            if ws is None:
                ws = self._empty(need, self._torch.uint8)
            if not (ws.get_device() == device and ws.is_contiguous() and ws.numel() * ws.element_size() >= need):
                _refuse("ws has %d bytes on the current GPU, contiguous" % need)
            wp = ws.data_ptr()
        status = L.tsq_cache_attend(
            self.handle, self._memory(memory, device), n, *self._requests(table, starts, lengths, n, device), tokens, max_new, max_length, qp, qs,
            self.head_dim ** -0.5 if scale is None else scale, causal, window, op, os_, lp, wp, self._stream())
        if status:
            raise TsqError(status, "tsq_cache_attend")
        return out
