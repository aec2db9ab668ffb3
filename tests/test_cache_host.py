"""Host-only checks of the serving operators' C ABI (include/tsq_cache.h): every function is exported, configurations and
arguments are refused as the header says, workspace sizes follow the call's numbers.  No kernel is launched here."""
import ctypes as C
import os
import re

import pytest

from paper_2511_04002_amd import build as tsq_build
from paper_2511_04002_amd import cache, tsq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    tsq_build.build()
    return cache.lib()


def test_every_declared_symbol_is_exported(L):
    text = open(os.path.join(ROOT, "include", "tsq_cache.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(tsq_cache_[a-z_]+)\s*\(", text))
    assert names == set(cache.EXPORTS)
    for n in names:
        assert hasattr(L, n), n


def cfg(**kw):
    base = dict(blocks=10, block_tokens=16, q_heads=8, kv_heads=2, head_dim=128, dtype=tsq.TSQ_F16, max_blocks=4, reserved=0)
    base.update(kw)
    return cache.tsq_cache_config(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(blocks=0), tsq.TSQ_ERR_INVALID_ARG),
    (dict(block_tokens=0), tsq.TSQ_ERR_INVALID_ARG),
    (dict(q_heads=0), tsq.TSQ_ERR_INVALID_ARG),
    (dict(kv_heads=0), tsq.TSQ_ERR_INVALID_ARG),
    (dict(head_dim=0), tsq.TSQ_ERR_INVALID_ARG),
    (dict(max_blocks=0), tsq.TSQ_ERR_INVALID_ARG),
    (dict(reserved=1), tsq.TSQ_ERR_INVALID_ARG),
    (dict(dtype=2), tsq.TSQ_ERR_INVALID_ARG),
    (dict(q_heads=9), tsq.TSQ_ERR_INVALID_ARG),
    (dict(block_tokens=8), tsq.TSQ_ERR_UNSUPPORTED),
    (dict(block_tokens=48), tsq.TSQ_ERR_UNSUPPORTED),
    (dict(block_tokens=256), tsq.TSQ_ERR_UNSUPPORTED),
    (dict(head_dim=96), tsq.TSQ_ERR_UNSUPPORTED),
    (dict(q_heads=2048), tsq.TSQ_ERR_UNSUPPORTED),
    (dict(blocks=1 << 27), tsq.TSQ_ERR_UNSUPPORTED),
    (dict(max_blocks=1 << 27), tsq.TSQ_ERR_UNSUPPORTED),
])
def test_create_refuses(L, kw, status):
    with pytest.raises(tsq.TsqError) as e:
        cache.tsq_cache_create(cfg(**kw))
    assert e.value.status == status


def test_null_create(L):
    h, c = C.c_void_p(), cfg()
    assert L.tsq_cache_create(None, C.byref(h)) == tsq.TSQ_ERR_INVALID_ARG
    assert L.tsq_cache_create(C.byref(c), None) == tsq.TSQ_ERR_INVALID_ARG


@pytest.fixture()
def handle(L):
    h = cache.tsq_cache_create(cfg())
    yield h
    cache.tsq_cache_destroy(h)


def test_memory_sizes(L, handle):
    s = cache.tsq_cache_memory_sizes(handle)
    assert s.code_bytes == 10 * 2 * 16 * 128 and s.scale_bytes == 10 * 2 * 4
    assert L.tsq_cache_memory_sizes(handle, None) == tsq.TSQ_ERR_INVALID_ARG


MEM = dict(d_k=0x10000, d_v=0x20000, d_k_scale=0x30000, d_v_scale=0x40000)


def memory(**kw):
    return C.byref(cache.tsq_cache_memory(**{**MEM, **kw}))


def refused(f, good, changes):
    """Each change of one argument of a call that would be good is refused (the good call itself is not made)."""
    names = list(good)
    for name, value, status in changes:
        args = dict(good)
        assert name in args
        args[name] = value
        assert f(*[args[n] for n in names]) == status, (name, value)


BAD, UNS = tsq.TSQ_ERR_INVALID_ARG, tsq.TSQ_ERR_UNSUPPORTED


def test_schedule_refuses(L, handle):
    good = dict(cache=handle, requests=3, new=0x1000, lengths=0x2000, table=0x3000, ring=0x4000, counters=0x5000, capacity=7,
                lengths_out=0x6000, counters_out=0x7000, starts=0x8000, positions=0x9000, slots=0xA000, status=0xB000, stream=None)
    refused(L.tsq_cache_schedule, good,
            [(n, None, BAD) for n in good if n not in ("requests", "capacity", "stream")] +
            [("requests", 0, BAD), ("requests", 4097, UNS), ("counters", 0x5004, BAD), ("counters_out", 0x7004, BAD), ("new", 0x1002, BAD),
             ("lengths_out", 0x2000, BAD), ("counters_out", 0x5000, BAD), ("capacity", 1 << 31, BAD)])


def test_norm_rotate_refuses(L, handle):
    good = dict(cache=handle, tokens=5, q=0x1000, q_stride=1024, k=0x2000, k_stride=256, positions=0x3000, angles=0x4000, angle_rows=9,
                rotary=128, pairs=0, qw=0x5000, kw=0x6000, eps=1e-6, q_out=0x7000, q_out_stride=1024, k_out=0x8000, k_out_stride=256,
                stream=None)
    f = L.tsq_cache_norm_rotate
    refused(f, good, [(n, None, BAD) for n in ("cache", "q", "k", "positions", "angles", "q_out", "k_out")] +
            [("q", 0x1008, BAD), ("k", 0x2002, BAD), ("qw", 0x5004, BAD), ("angles", 0x4008, BAD), ("q_stride", 1016, BAD), ("q_stride", 1028, BAD),
             ("k_stride", 248, BAD), ("q_out_stride", 1000, BAD), ("k_out_stride", 255, BAD), ("rotary", 0, BAD), ("rotary", 8, BAD),
             ("rotary", 24, BAD), ("rotary", 144, BAD), ("pairs", 2, BAD), ("pairs", -1, BAD), ("eps", -1.0, BAD), ("eps", float("nan"), BAD),
             ("eps", float("inf"), BAD)])
    assert f(*{**good, "tokens": 0, "q": None, "k": None}.values()) == tsq.TSQ_OK


def test_append_refuses(L, handle):
    good = dict(cache=handle, memory=memory(), tokens=5, k=0x1000, k_stride=256, v=0x2000, v_stride=256, slots=0x3000, stream=None)
    refused(L.tsq_cache_append, good, [(n, None, BAD) for n in ("cache", "memory", "k", "v", "slots")] +
            [("memory", memory(**{n: None}), BAD) for n in MEM] + [("memory", memory(**{n: MEM[n] + 8}), BAD) for n in MEM] +
            [("k", 0x1004, BAD), ("v_stride", 128, BAD), ("k_stride", 260, BAD), ("slots", 0x3001, BAD)])
    assert L.tsq_cache_append(handle, memory(), 0, None, 0, None, 0, None, None) == tsq.TSQ_OK


def test_gather_refuses(L, handle):
    good = dict(cache=handle, memory=memory(), requests=2, table=0x1000, starts=0x2000, lengths=0x3000, tokens=5, k=0x4000, k_stride=256,
                v=0x5000, v_stride=256, stream=None)
    refused(L.tsq_cache_gather, good, [(n, None, BAD) for n in ("cache", "memory", "table", "starts", "lengths", "k", "v")] +
            [("requests", 0, BAD), ("requests", 65536, UNS), ("k", 0x4004, BAD), ("v_stride", 8, BAD)])


def test_attend_refuses(L, handle):
    good = dict(cache=handle, memory=memory(), requests=2, table=0x1000, starts=0x2000, lengths=0x3000, tokens=5, max_new=4, max_length=4096,
                q=0x4000, q_stride=1024, scale=0.1, causal=1, window=0, out=0x5000, out_stride=1024, lse=0x6000, ws=0x7000, stream=None)
    refused(L.tsq_cache_attend, good, [(n, None, BAD) for n in ("cache", "memory", "table", "starts", "lengths", "q", "out", "ws")] +
            [("requests", 0, BAD), ("requests", 65536, UNS), ("tokens", 1 << 28, UNS), ("q", 0x4008, BAD), ("out_stride", 1000, BAD),
             ("scale", 0.0, BAD), ("scale", -1.0, BAD), ("scale", float("nan"), BAD), ("scale", float("inf"), BAD), ("causal", 2, BAD),
             ("lse", 0x6002, BAD), ("ws", 0x7010, BAD)])


def test_attend_workspace(L, handle):
    f = cache.tsq_cache_attend_workspace_bytes
    assert f(handle, 1, 1, 1, 64) == 0                       # a short cache is not split
    assert f(handle, 0, 1, 1, 64) == 0 and f(handle, 1, 0, 0, 64) == 0
    one = f(handle, 1, 1, 1, 1 << 20)
    assert one > 0 and one % (8 * 130 * 4) == 0              # pieces of [q_heads] rows: sums and two statistics each
    assert f(handle, 1, 1, 1, 1 << 20, 100) == 0             # a window leaves little to split


def test_attend_of_256_tokens_needs_no_workspace(L):
    for heads, dim in ((1, 64), (8, 128), (1, 256)):
        h = cache.tsq_cache_create(cfg(q_heads=heads, kv_heads=1, head_dim=dim))
        for tokens, new in ((1, 1), (7, 7), (256, 256), (5000, 1)):
            assert cache.tsq_cache_attend_workspace_bytes(h, 1, tokens, new, 256) == 0
        cache.tsq_cache_destroy(h)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_workspace_of_single_tokens_beside_a_prompt(L, dim):
    """The rows of the single tokens have pieces along a long cache, the prompt's have none where it would have none alone."""
    h = cache.tsq_cache_create(cfg(q_heads=64, kv_heads=8, head_dim=dim))
    f = cache.tsq_cache_attend_workspace_bytes
    rows = 64 * 8 * (32 if dim == 256 else 64)               # of 64 requests of as few rows of a kv head as go by themselves
    for prompt in (512, 4096, 8192, 65536):
        alone = f(h, 1, prompt, prompt, 131072)
        assert alone == 0 or prompt < 4096
        assert 0 < f(h, 64, 63 + prompt, prompt, 131072) <= rows * 16 * (dim + 2) * 4 + alone * (63 + prompt) // prompt + 256
    assert f(h, 64, 63 + 8192, 8192, 8192) == 0              # nothing is long: no pieces
    cache.tsq_cache_destroy(h)


def test_calls_of_too_many_threads_are_refused_before_anything_is_enqueued(L):
    """2^32 threads, in each of the kernels that a call may need, the last one of an attend call among them."""
    def made(**kw):
        return cache.tsq_cache_create(cfg(**{**dict(q_heads=1, kv_heads=1, head_dim=64), **kw}))

    h = made()
    n = 1 << 26
    assert L.tsq_cache_norm_rotate(h, n, 0x1000, 64, 0x2000, 64, 0x3000, 0x4000, 9, 64, 0, None, None, 1e-6, 0x5000, 64, 0x6000, 64, None) == UNS
    n = 1 << 30
    assert L.tsq_cache_append(h, memory(), n, 0x1000, 64, 0x2000, 64, 0x3000, None) == UNS
    assert L.tsq_cache_gather(h, memory(), 2, 0x1000, 0x2000, 0x3000, n, 0x4000, 64, 0x5000, 64, None) == UNS
    cache.tsq_cache_destroy(h)

    def attend(h, requests, tokens, max_new, max_length, width):
        return L.tsq_cache_attend(h, memory(), requests, 0x1000, 0x2000, 0x3000, tokens, max_new, max_length, 0x4000, width, 0.1, 1, 0, 0x5000, width,
                                  None, 0x10000, None)

    for heads, requests, tokens, new, length in ((1024, 16384, 16384, 1, 64), (1024, 65535, 1 << 17, 1 << 17, 64)):
        h = made(q_heads=heads, kv_heads=heads)
        assert attend(h, requests, tokens, new, length, heads * 64) == UNS
        cache.tsq_cache_destroy(h)
    h = made(q_heads=64, head_dim=128)                       # the join: 2^23 rows of 512 threads
    assert attend(h, 65535, 1 << 17, 1, 140000, 64 * 128) == UNS
    cache.tsq_cache_destroy(h)


def test_attend_workspace_of_a_length_that_no_request_can_have(L):
    f = cache.tsq_cache_attend_workspace_bytes
    h = cache.tsq_cache_create(cfg(q_heads=64, kv_heads=8))
    for requests, tokens, new in ((1, 8192, 8192), (1, 1, 1), (64, 64, 1), (64, 1000, 900)):
        for length in (2 ** 31, 2 ** 32 - 128, 2 ** 32 - 1):
            assert f(h, requests, tokens, new, length) == f(h, requests, tokens, new, 2 ** 31 - 1)
    assert f(h, 1, 8192, 8192, 2 ** 32 - 1) == 0
    cache.tsq_cache_destroy(h)


@pytest.mark.parametrize("at", range(6))
def test_cache_numbers_past_32_bits_are_refused(L, at):
    numbers = [4, 16, 4, 2, 64, 2]
    cache.Cache(*numbers[:5], "f16", numbers[5])
    numbers[at] += 2 ** 32
    with pytest.raises(ValueError):
        cache.Cache(*numbers[:5], "f16", numbers[5])
