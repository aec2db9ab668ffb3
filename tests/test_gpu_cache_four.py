"""The operators of a cache in 4 bits, and the rotation by positions of several axes, on the GPU through the C ABI, against
the plain oracle (oracle/cache_oracle.py)."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as O
from paper_2511_04002_amd import cache as cachelib
from paper_2511_04002_amd import tsq

pytestmark = pytest.mark.gpu

KIND = {"f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}       # relative, of one rounding
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134}         # absolute, below the normal range


def dev(x, kind=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if kind is None else t.to(kind)


def host(t):
    return (t.float() if t.dtype in (torch.float16, torch.bfloat16) else t).cpu().numpy()


def rows(g, tokens, heads, dim, dtype, size=1.0):
    return dev(g.standard_normal((tokens, heads, dim)) * size, KIND[dtype])


class Both:
    """A cache on the GPU and the same one in the oracle."""

    def __init__(self, blocks, block, heads, dim, dtype, max_blocks, seed, q_heads=None):
        self.c = cachelib.Cache(blocks, block, q_heads or heads, heads, dim, dtype, max_blocks, bits=4)
        g = self.g = np.random.default_rng(seed)
        self.block, self.heads, self.dim, self.dtype, self.max_blocks = block, heads, dim, dtype, max_blocks
        self.k, self.v = (g.integers(0, 256, (blocks, heads, block, dim // 2)).astype(np.uint8) for _ in range(2))
        self.ks, self.vs = (g.integers(123, 128, (blocks, heads, dim // 32, block)).astype(np.uint8) for _ in range(2))
        self.wrap()

    def wrap(self):
        self.m = self.c.wrap(dev(self.k), dev(self.v), dev(self.ks), dev(self.vs))

    def append(self, k, v, slots):
        """k, v: CUDA tensors [tokens, heads, dim]."""
        slots = np.asarray(slots, np.int32)
        self.c.append(self.m, k, v, dev(slots))
        O.four_append(self.k, self.v, self.ks, self.vs, host(k), host(v), slots, self.block, self.dtype)

    def same(self):
        """All scales, and all codes but those of tokens that are marked, are the oracle's."""
        for codes, scale, k, s in ((self.m.k, self.m.k_scale, self.k, self.ks), (self.m.v, self.m.v_scale, self.v, self.vs)):
            assert np.array_equal(host(scale), s)
            fine = (s != 255).all(2)                         # [blocks, heads, block tokens]
            assert np.array_equal(host(codes)[fine], k[fine])


# ------------------------------------------------------------------ append

@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads,dim", [(1, 64), (3, 64), (8, 128), (5, 128), (1, 256), (3, 256)])
@pytest.mark.parametrize("block", [16, 128])
def test_append_of_tokens_anywhere(dtype, heads, dim, block):
    b = Both(20, block, heads, dim, dtype, 1, heads + dim + block)
    for tokens in (1, 2, 67):
        slots = b.g.permutation(20 * block)[:tokens].astype(np.int64)
        slots[b.g.random(tokens) < 0.1] = -1
        size = np.exp2(b.g.integers(-9, 9, (tokens, heads, 1))) * b.g.choice([1, 1, 1, 8], (1, 1, dim))
        k = dev(b.g.standard_normal((tokens, heads, dim)) * size, KIND[dtype])
        b.append(k, rows(b.g, tokens, heads, dim, dtype, 2.0 ** -5), slots)
        b.same()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_append_of_every_number(dtype):
    """Every finite pattern of the type, as the largest of its 32 and beside larger ones: scales, ties, the ends of the range."""
    bits = np.arange(0x8000, dtype=np.uint16)
    bits = bits[bits < (0x7C00 if dtype == "f16" else 0x7F80)]
    b = Both(len(bits) // 128 + 1, 128, 1, 64, dtype, 1, 1)
    x = np.zeros((len(bits), 64), np.uint16)
    x[:, 0] = bits
    x[1:, 1:32] = (b.g.integers(0, 1 << 16, (len(bits) - 1, 31)) % bits[1:, None]) | (b.g.integers(0, 2, (len(bits) - 1, 31)) << 15)
    x[:, 32:] = bits[b.g.integers(0, len(bits), (len(bits), 32))] | (b.g.integers(0, 2, (len(bits), 32)) << 15)
    x = dev(x.astype(np.uint16).view(np.int16)).view(KIND[dtype])[:, None]
    # (the oracle's own slots by whole arrays: a token each)
    b.c.append(b.m, x, x, torch.arange(len(bits), dtype=torch.int32, device="cuda"))
    want = host(x)[:, 0].astype(np.float64).reshape(-1, 2, 32)
    byte = O.four_scale(want, dtype)
    assert np.array_equal(host(b.m.k_scale).swapaxes(2, 3).reshape(-1, 2)[:len(bits)], byte)
    c = O.four_code(want, byte.astype(np.float64)).reshape(-1, 64)
    for codes in (b.m.k, b.m.v):
        assert np.array_equal(host(codes).reshape(-1, 32)[:len(bits)], c[:, 0::2] + 16 * c[:, 1::2])


def test_append_of_strided_rows_and_slots_outside_the_cache():
    b = Both(6, 16, 2, 128, "bf16", 2, 3)
    qkv = rows(b.g, 9, 8, 128, "bf16")
    before = [x.clone() for x in (b.m.k, b.m.v, b.m.k_scale, b.m.v_scale)]
    outside = torch.tensor([-1, -2 ** 31, 96, 97, 2 ** 31 - 1, -16, 111, 1 << 20, 96 + 1], dtype=torch.int32, device="cuda")
    b.c.append(b.m, qkv[:, 4:6], qkv[:, 6:], outside)
    for x, y in zip(before, (b.m.k, b.m.v, b.m.k_scale, b.m.v_scale)):
        assert torch.equal(x, y)
    b.append(qkv[:, 4:6], qkv[:, 6:], [95, -1, 0, 17, 96, 16, 15, 94, 80])
    b.same()
    wide = qkv.flatten(1)
    b.append(wide[:, 512:768].unflatten(1, (2, 128)), wide[:, 768:].unflatten(1, (2, 128)), np.arange(30, 39))
    b.same()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_append_of_what_is_not_finite_marks_the_token_and_a_new_use_clears_it(bad, dim):
    b = Both(4, 16, 3, dim, "bf16", 2, 4)
    k, v = rows(b.g, 5, 3, dim, "bf16"), rows(b.g, 5, 3, dim, "bf16")
    k[1, 0, dim - 1], v[3, 2, 0] = bad, bad
    b.append(k, v, [3, 4, 20, 21, 50])
    b.same()
    assert (b.ks[0, 0, :, 4] == 255).all() and (b.vs[0, 0, :, 4] == 255).all() and (b.ks[1, 2, :, 5] == 255).all()
    assert (b.ks != 255).sum() == b.ks.size - 2 * (dim // 32)
    table, starts, lengths = dev(np.array([[0, 1]], np.int32)), dev(np.array([0, 32], np.int32)), dev(np.array([32], np.int32))
    out = [torch.empty((32, 3, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    b.c.gather(b.m, table, starts, lengths, *out)
    for x in out:
        assert x[4, 0].isnan().all() and x[21, 2].isnan().all() and int(x.isnan().sum()) == 2 * dim
    b.append(rows(b.g, 2, 3, dim, "bf16"), rows(b.g, 2, 3, dim, "bf16"), [4, 21])
    b.same()
    assert (b.ks != 255).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_what_is_stored_is_near(dtype):
    """Off by half a step at most: a quarter of the scale below 2, half below 4, and the scale itself above."""
    b = Both(8, 64, 4, 128, dtype, 8, 5)
    k = rows(b.g, 500, 4, 128, dtype)
    b.c.append(b.m, k, k, torch.arange(500, dtype=torch.int32, device="cuda"))
    out = [torch.empty_like(k) for _ in range(2)]
    table = torch.arange(8, dtype=torch.int32, device="cuda")[None]
    b.c.gather(b.m, table, dev(np.array([0, 500], np.int32)), dev(np.array([500], np.int32)), *out)
    x = host(k).astype(np.float64).reshape(500, 4, 4, 32)
    scale = 2.0 ** (O.four_scale(x, dtype).astype(np.float64) - 127)[..., None]
    assert (np.abs(x).max(-1, keepdims=True) > 3.5 * scale).all() and (np.abs(x).max(-1, keepdims=True) <= 7 * scale).all()
    off, a = np.abs(host(out[0]).reshape(x.shape) - x) / scale, np.abs(x) / scale
    assert (off <= np.where(a <= 2, 0.25, np.where(a <= 4, 0.5, 1.0))).all() and torch.equal(out[0], out[1])


# ------------------------------------------------------------------ gather

@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("block", [16, 32, 128])
def test_gather(dtype, dim, block):
    b = Both(60, block, 3, dim, dtype, 8, dim + block)
    g = b.g
    lengths = np.array([1, 0, block, 5 * block + 3, block - 1, 2, 8 * block], np.int32)
    # all of a request, a part of it, more than it has, and none
    counts = [1, 2, block, 2 * block + 5, 0, 2, 8 * block - 3]
    table = g.permutation(60)[:56].reshape(7, 8).astype(np.int32)
    table[3, 4] = 60
    starts = np.concatenate(([0], np.cumsum(counts))).astype(np.int32)
    total = int(starts[-1])
    out = [torch.full((total + 3, 3, dim), 7.0, dtype=KIND[dtype], device="cuda") for _ in range(2)]
    b.c.gather(b.m, dev(table), dev(starts), dev(lengths), *out)
    for got, codes, scale in ((out[0], b.k, b.ks), (out[1], b.v, b.vs)):
        got = host(got)
        assert (got[total:] == 7).all()
        for r, n in enumerate(counts):
            want = O.four_tokens_of(codes, scale, table[r], int(lengths[r]), block, 8)
            want = np.concatenate((np.full((max(0, n - len(want)), 3, dim), np.nan), want))[len(want) - n if n < len(want) else 0:]
            assert np.array_equal(got[starts[r]:starts[r + 1]], want, equal_nan=True), r           # (exact in either type)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_gather_of_every_scale_is_exact(dtype):
    low, high = (104, 140) if dtype == "f16" else (7, 252)
    b = Both(2, 128, 1, 64, dtype, 2, 6)
    b.k[:] = np.arange(256, dtype=np.uint8).reshape(2, 1, 128, 1)
    b.ks[:] = np.resize(np.arange(low, high + 1), (2, 1, 1, 128)).astype(np.uint8)
    b.wrap()
    out = [torch.empty((256, 1, 64), dtype=KIND[dtype], device="cuda") for _ in range(2)]
    b.c.gather(b.m, dev(np.array([[0, 1]], np.int32)), dev(np.array([0, 256], np.int32)), dev(np.array([256], np.int32)), *out)
    assert np.array_equal(host(out[0]), O.four_tokens_of(b.k, b.ks, [0, 1], 256, 128, 2))


def test_gather_of_a_strided_part_and_rows_that_the_compressor_takes():
    b = Both(40, 16, 4, 128, "f16", 20, 9)
    table = dev(b.g.permutation(40).reshape(2, 20).astype(np.int32))
    starts, lengths = dev(np.array([0, 100, 320], np.int32)), dev(np.array([100, 220], np.int32))
    k, v = (torch.empty((320, 512), dtype=torch.float16, device="cuda") for _ in range(2))
    b.c.gather(b.m, table, starts, lengths, k, v)
    wide = torch.zeros((320, 1536), dtype=torch.float16, device="cuda")
    b.c.gather(b.m, table, starts, lengths, wide[:, 512:1024], wide[:, 1024:])
    assert torch.equal(wide[:, 512:1024], k) and torch.equal(wide[:, 1024:], v) and (wide[:, :512] == 0).all()
    plan = tsq.Plan(640, 512, "f16", 1e4, (8,), 0.05)
    blob, _ = plan.compress_batch([k, v])
    back = [torch.empty_like(k), torch.empty_like(v)]
    plan.decompress_batch(blob, back)
    for x, y in ((k, back[0]), (v, back[1])):
        assert (x - y).abs().max() <= x.abs().max() / 127


# ------------------------------------------------------------------ attention

def attend_both(b, q_heads, counts, lengths, causal=True, window=0, table=None, q=None, max_new=None, max_length=None, scale=None,
                extra=0, exact_scores=False):
    g, dim, dtype = b.g, b.dim, b.dtype
    counts, lengths = np.asarray(counts), np.asarray(lengths, np.int32)
    starts = np.concatenate(([0], np.cumsum(counts))).astype(np.int32)
    total = int(starts[-1])
    if table is None:
        ids = g.permutation(b.k.shape[0])
        table, at = np.full((len(counts), b.max_blocks), -1, np.int32), 0
        for r, n in enumerate(lengths):
            held = -(-int(n) // b.block)
            table[r, :held] = ids[at:at + held]
            at += held
    if q is None:
        q = rows(g, total + extra, q_heads, dim, dtype, 1.5)
    scale = dim ** -0.5 if scale is None else scale
    out = torch.full((total + extra, q_heads, dim), 7.0, dtype=KIND[dtype], device="cuda")
    lse = torch.full((total + extra, q_heads), 7.0, device="cuda")
    b.c.attend(b.m, q, dev(table), dev(starts), dev(lengths), max(counts) if max_new is None else max_new,
               max(lengths) if max_length is None else max_length, scale, causal, window, out, lse)
    got, got_lse = host(out), host(lse)
    assert (got[total:] == 7).all() and (got_lse[total:] == 7).all()
    with np.errstate(all="ignore"):
        want, want_lse, spread = O.four_attend(b.k, b.v, b.ks, b.vs, b.block, b.max_blocks, table, starts, lengths, host(q)[:total], scale, causal, window)
    got, got_lse = got[:total], got_lse[:total]
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isnan(got_lse), np.isnan(want_lse))
    # What a weight may be off, relative: half a unit of 11 bits; and its exponent, of which the products of a query and a
    # key are exact, their sum in binary32 is off by 2^-24 of the sum of magnitudes for each of the dim terms, and the scale, the
    # factor of the logarithm and the difference round to 2^-24 of the score each.  Both act on numerator and denominator.
    blocks = np.unique(table[(table >= 0) & (table < len(b.k))])
    size = np.nan_to_num(np.abs(O.four_values(b.k[blocks], b.ks[blocks]))).max(initial=0.0, axis=(0, 1, 2))
    most = float((np.nan_to_num(np.abs(host(q)[:total]).astype(np.float64), posinf=0.0) @ size).max(initial=0.0)) * scale
    off = 2.0 ** -11 + 2 * most * 2.0 ** -24 * (6 if exact_scores else dim + 6)
    # (weights that are halves, of values that halves hold, are rounded to 2^-25 below 2^-14 where the largest is at least 2^7;
    # those of other values, whose largest is at least 2^-16 - 8 below the reference, and 8 more until that moves - are lost below
    # 2^-126, binary32's and bfloat16's least normal number: 2^-110 of the largest)
    held = b.vs[b.vs != 255]
    largest = 6 * 2.0 ** (float(held.max(initial=0)) - 127)
    least = (2.0 ** -32 if dtype == "f16" or (held.min(initial=255) >= 104 and held.max(initial=0) <= 140) else 2.0 ** -110) * lengths.max() * largest
    # (sums of binary32: their order, and the parts that are joined)
    fine = ~np.isnan(want)
    bound = HALF_ULP[dtype] * np.abs(want) + (off + 2.0 ** -24 * (lengths.max() + 64)) * spread + TINY[dtype] + least
    assert (np.abs(got - want)[fine] <= bound[fine]).all(), float((np.abs(got - want) / bound)[fine].max())
    empty = np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(got_lse), empty)
    fine = np.isfinite(want_lse)
    assert (np.abs(got_lse[fine] - want_lse[fine]) <= off + 2.0 ** -21 * np.maximum(1, np.abs(want_lse[fine]))).all()
    assert (got[empty] == 0).all()
    return out, lse, want


SHAPES = [(1, 1, 64), (12, 12, 64), (5, 1, 128), (8, 1, 128), (16, 2, 128), (28, 4, 128), (40, 2, 128), (4, 2, 256), (16, 1, 256)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", SHAPES)
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_attend_single_tokens(dtype, heads, block):
    hq, hk, dim = heads
    b = Both(90, block, hk, dim, dtype, 40, hq + block, q_heads=hq)
    lengths = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 300]
    attend_both(b, hq, [1] * len(lengths), lengths)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [(2, 2, 64), (8, 1, 128), (6, 2, 128), (4, 1, 256)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 40), (False, 17), (True, 100000)])
def test_attend_several_tokens_and_chunks(dtype, heads, causal, window):
    hq, hk, dim = heads
    b = Both(90, 16, hk, dim, dtype, 40, hq + window, q_heads=hq)
    attend_both(b, hq, [1, 2, 0, 8, 33, 70, 150, 3], [1, 90, 5, 8, 100, 70, 171, 300], causal, window)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("block", [16, 64, 128])
def test_attend_prompt(dtype, block):
    b = Both(3000 // block + 2, block, 2, 128, dtype, 3000 // block + 1, block, q_heads=8)
    attend_both(b, 8, [517, 131], [517, 131])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [(1, 1, 64), (8, 1, 128), (4, 2, 256)])
def test_attend_of_states_of_another_length(dtype, heads):
    """Nothing hidden, and more queries than tokens as well as fewer."""
    hq, hk, dim = heads
    b = Both(90, 32, hk, dim, dtype, 40, hq, q_heads=hq)
    attend_both(b, hq, [70, 1, 33, 300, 5], [200, 90, 33, 17, 0], causal=False)
    attend_both(b, hq, [70, 1, 33, 300, 5], [200, 90, 33, 17, 0], causal=False, window=30)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [(1, 1, 64), (8, 1, 128), (4, 2, 256)])
@pytest.mark.parametrize("counts,lengths", [([1], [7001]), ([3], [5000]), ([1, 1], [4097, 31]), ([40], [6000])])
def test_attend_along_a_long_cache(dtype, heads, counts, lengths):
    hq, hk, dim = heads
    b = Both(620, 16, hk, dim, dtype, 500, 11, q_heads=hq)
    need = cachelib.tsq_cache_attend_workspace_bytes(b.c.handle, len(counts), sum(counts), max(counts), max(lengths))
    assert need > 0                                          # the cache's length is split and joined
    attend_both(b, hq, counts, lengths)


def test_attend_of_requests_larger_than_they_were_announced():
    b = Both(300, 16, 2, 128, "f16", 120, 12, q_heads=8)
    for max_new, max_length in ((1, 1), (1, 600), (0, 0)):
        attend_both(b, 8, [9, 1, 40], [1800, 700, 40], max_new=max_new, max_length=max_length)


def test_attend_rows_that_see_nothing_and_rows_that_no_request_has():
    b = Both(20, 16, 1, 64, "f16", 8, 13, q_heads=3)
    # more queries than tokens, and a request without any
    attend_both(b, 3, [5, 1, 40], [3, 0, 20])
    attend_both(b, 3, [5, 1, 40], [3, 0, 20], causal=False)
    attend_both(b, 3, [5, 1, 40], [3, 0, 20], window=2)
    attend_both(b, 3, [1, 2], [0, 0], extra=3)
    b = Both(20, 16, 2, 128, "bf16", 8, 14, q_heads=2)
    attend_both(b, 2, [30, 2], [30, 40], extra=50)
    attend_both(b, 2, [300, 2], [30, 40], extra=5)


def test_attend_many_requests():
    b = Both(1400, 16, 1, 64, "f16", 12, 15, q_heads=2)
    g = b.g
    lengths = g.integers(0, 60, 300)
    attend_both(b, 2, [1] * 300, lengths)
    counts = np.minimum(g.integers(0, 9, 300), lengths)
    counts[7] = lengths[7] = 150
    attend_both(b, 2, counts, lengths)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attend_table_entries_outside_the_cache_and_lengths_past_the_table(dtype):
    b = Both(20, 16, 1, 128, dtype, 6, 16, q_heads=4)
    table = b.g.permutation(20)[:18].reshape(3, 6).astype(np.int32)
    table[1, 2] = 20
    table[2, 0] = -3
    attend_both(b, 4, [50, 45, 2], [90, 48, 30], table=table)
    attend_both(b, 4, [1, 1, 1], [97, 96, 10], table=table)
    attend_both(b, 4, [80, 90, 7], [97, 96, 10], table=table, window=20)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_marked_tokens_reach_only_the_rows_that_see_them(dtype, dim):
    b = Both(20, 16, 2, dim, dtype, 10, 17, q_heads=4)
    table = np.arange(20, dtype=np.int32).reshape(2, 10)
    for block, head, place in ((3, 0, 5), (5, 1, 0), (7, 0, 15), (14, 1, 7)):
        b.ks[block, head, :, place] = b.vs[block, head, :, place] = 255
    b.wrap()
    for counts in ([130, 1], [3, 2], [1, 1]):
        for window in (0, 20):
            attend_both(b, 4, counts, [150, 100], table=table, window=window)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_ignores_what_lies_behind_a_request_and_in_blocks_of_nobody(dtype, dim):
    b = Both(6, 16, 1, dim, dtype, 4, 18, q_heads=2)
    table = np.array([[1, 2, 5, 5], [3, 5, 5, 0]], np.int32)
    b.ks[[0, 4, 5]], b.vs[[0, 4, 5]] = 255, 254
    b.ks[2, :, :, 4:], b.vs[2, :, :, 4:] = 254, 255                            # places behind the requests' ends
    b.ks[3, :, :, 9:], b.vs[3, :, :, 9:] = 255, 254
    b.wrap()
    b.ks[b.ks >= 254] = b.vs[b.vs >= 254] = 0                                  # (the bounds go by what is seen)
    for counts in ([1, 3], [20, 9], [40, 40]):
        attend_both(b, 2, counts, [20, 9], table=table)
        attend_both(b, 2, counts, [20, 9], table=table, causal=False)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("counts,dim", [([1, 1, 1], 64), ([3, 1, 2], 128), ([150, 90, 1], 64), ([150, 90, 1], 128), ([60, 70, 1], 256)])
def test_attend_gives_the_same_bits_whatever_lies_behind_a_request(dtype, counts, dim):
    """Scales that have never been written do not decide how a request's own values are treated."""
    outs = []
    for behind in (127, 0, 255, 104):
        b = Both(60, 16, 2, dim, dtype, 20, 77, q_heads=8)
        table = b.g.permutation(60).reshape(3, 20).astype(np.int32)
        lengths = [301, 90, 5]
        for r, n in enumerate(lengths):
            for x in (b.ks, b.vs):
                x[table[r, n // 16], ..., n % 16:] = behind
                x[table[r, n // 16 + 1:]] = behind
        b.wrap()
        outs.append(attend_both(b, 8, counts, lengths, table=table, max_length=301)[:2])
    for out, lse in outs[1:]:
        assert torch.equal(out, outs[0][0]) and torch.equal(lse, outs[0][1])


ANY_SCALE = (127, 0, 255, 104, 112, 140)                 # what a byte of scales may be that nobody has written


def bits_of(b, q, table, starts, lengths, *more):
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    return b.c.attend(b.m, q, dev(table), dev(np.asarray(starts, np.int32)), dev(np.asarray(lengths, np.int32)), *more, lse=lse), lse


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("counts", [[1, 1, 1], [6, 1, 2], [1, 90, 1], [40, 90, 2]])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("window,block,causal", [(40, 16, True), (100, 128, True), (70, 32, False)])
def test_attend_gives_the_same_bits_whatever_lies_before_a_window(dtype, counts, dim, window, block, causal):
    """Blocks that every row's window has left behind may have been given back, and hold what others write to them."""
    lengths, starts, outs = [301, 290, 5], np.concatenate(([0], np.cumsum(counts))), []
    for before in ANY_SCALE + ((37, 250) if dtype == "bf16" else ()):
        for released in (False, True):
            b = Both(3 * 20 + 1, block, 2, dim, dtype, 20, 78, q_heads=8)
            table = 1 + b.g.permutation(60).reshape(3, 20).astype(np.int32)
            q = rows(b.g, sum(counts), 8, dim, dtype)
            for x in (b.ks, b.vs):
                x[0] = before
                for r, n in enumerate(lengths):
                    first = max(0, n - counts[r] - window + 1)
                    x[table[r, :first // block]] = before
                    x[table[r, first // block], ..., :first % block] = before
            for r, n in enumerate(lengths) if released else ():
                table[r, :max(0, n - counts[r] - window + 1) // block] = -1 if r else len(b.ks)
            b.wrap()
            outs.append(bits_of(b, q, table, starts, lengths, max(counts), 301, None, causal, window))
    assert outs[0][0].isfinite().all()
    for out, lse in outs[1:]:
        assert torch.equal(out, outs[0][0]) and torch.equal(lse, outs[0][1])
    b = Both(3 * 20 + 1, block, 2, dim, dtype, 20, 78, q_heads=8)
    table = 1 + b.g.permutation(60).reshape(3, 20).astype(np.int32)
    q = rows(b.g, sum(counts), 8, dim, dtype)
    got = attend_both(b, 8, counts, lengths, causal, window, table=table, q=q, max_length=301)
    assert torch.equal(got[0], outs[0][0]) and torch.equal(got[1], outs[0][1])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("counts", [[1, 1], [5, 2], [70, 60], [1, 1, 1, 1, 1, 90]])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_gives_the_same_bits_whatever_lies_before_a_window_in_pieces(dtype, counts, dim):
    window, lengths, outs = 2500, ([4000, 3333] if len(counts) == 2 else [3000, 9, 0, 2700, 40, 4000]), []
    starts = np.concatenate(([0], np.cumsum(counts)))
    for before in (127, 255) + ((37,) if dtype == "bf16" else ()):
        b = Both(1501, 16, 1, dim, dtype, 250, 81, q_heads=4)
        table = 1 + b.g.permutation(1500).reshape(6, 250)[:len(counts)].astype(np.int32)
        q = rows(b.g, sum(counts), 4, dim, dtype)
        for x in (b.ks, b.vs):
            x[0] = before
            for r, n in enumerate(lengths):
                first = max(0, n - counts[r] - window + 1)
                x[table[r, :first // 16]] = before
                x[table[r, first // 16], ..., :first % 16] = before
        for r, n in enumerate(lengths):
            table[r, :max(0, n - counts[r] - window + 1) // 16] = -1
        b.wrap()
        assert cachelib.tsq_cache_attend_workspace_bytes(b.c.handle, len(counts), sum(counts), max(counts), max(lengths), window) > 0
        outs.append(bits_of(b, q, table, starts, lengths, max(counts), max(lengths), None, True, window))
    assert outs[0][0].isfinite().all()
    for out, lse in outs[1:]:
        assert torch.equal(out, outs[0][0]) and torch.equal(lse, outs[0][1])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim,heads,queries,tile", [(64, 8, 8, 4), (128, 8, 8, 4), (256, 4, 8, 4), (64, 1, 600, 256), (128, 8, 200, 32), (256, 4, 90, 32)])
def test_attend_gives_the_same_bits_whatever_only_later_tiles_see(dtype, dim, heads, queries, tile):
    """`tile`: queries that one workgroup has; the token behind those of the first ones decides nothing for them."""
    outs = []
    for later in ANY_SCALE + ((37, 250) if dtype == "bf16" else ()):
        b = Both(60, 16, 1, dim, dtype, 60, 79, q_heads=heads)
        table = b.g.permutation(60)[None].astype(np.int32)
        q = rows(b.g, queries, heads, dim, dtype)
        past = 21
        at = past + tile
        b.ks[table[0, at // 16], ..., at % 16] = b.vs[table[0, at // 16], ..., at % 16] = later
        b.wrap()
        outs.append([x[:tile] for x in bits_of(b, q, table, [0, queries], [past + queries], queries, past + queries)])
    assert outs[0][0].isfinite().all()
    for out, lse in outs[1:]:
        assert torch.equal(out, outs[0][0]) and torch.equal(lse, outs[0][1])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("queries", [12, 24, 60, 130])
def test_attend_gives_the_same_bits_whatever_is_read_for_a_block_that_the_table_does_not_hold(dtype, dim, queries):
    outs = []
    for other in ANY_SCALE + ((37, 250) if dtype == "bf16" else ()):
        b = Both(20, 16, 1, dim, dtype, 19, 80, q_heads=2)
        table = 1 + b.g.permutation(19)[None].astype(np.int32)
        q = rows(b.g, queries, 2, dim, dtype)
        b.ks[0] = b.vs[0] = other
        b.wrap()
        length = max(queries, 24)
        hole = (length - queries) // 16 + 1
        table[0, hole] = -1
        outs.append(bits_of(b, q, table, [0, queries], [length], queries, length))
    before = 16 * hole - (length - queries)                  # rows that see nothing of it
    assert 0 < before < queries and outs[0][0][:before].isfinite().all() and outs[0][0][before:].isnan().all()
    for out, lse in outs[1:]:
        assert torch.equal(out[:before], outs[0][0][:before]) and torch.equal(lse[:before], outs[0][1][:before]) and out[before:].isnan().all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attend_one_token_that_takes_all_the_weight_and_queries_far_from_one(dtype):
    b = Both(40, 16, 1, 128, dtype, 20, 20, q_heads=3)
    for n in (3, 40):
        q = rows(b.g, n, 3, 128, dtype, 30.0)
        attend_both(b, 3, [n], [300], q=q)
        q = rows(b.g, n, 3, 128, dtype, 2.0 ** -10)
        attend_both(b, 3, [n], [300], q=q)
        q[:] = 0
        attend_both(b, 3, [n], [300], q=q)
        if dtype == "bf16":
            attend_both(b, 3, [n], [300], q=rows(b.g, n, 3, 128, dtype, 2.0 ** 60), scale=2.0 ** -64)


def test_attend_queries_that_are_not_finite_spoil_their_own_rows_only():
    b = Both(40, 16, 1, 128, "bf16", 20, 21, q_heads=4)
    q = rows(b.g, 41, 4, 128, "bf16")
    table = b.g.permutation(40).reshape(2, 20).astype(np.int32)
    args = dev(table), dev(np.array([0, 1, 41], np.int32)), dev(np.array([200, 90], np.int32)), 40, 200
    good = b.c.attend(b.m, q, *args)
    q2 = q.clone()
    q2[0, 1, 5], q2[20, 2, 100], q2[33, 0, 64] = float("nan"), float("inf"), -float("inf")
    got = b.c.attend(b.m, q2, *args)
    bad = torch.zeros((41, 4), dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[20, 2] = bad[33, 0] = True
    assert got[bad].isnan().all() and torch.equal(got[~bad], good[~bad])


@pytest.mark.parametrize("counts", [[1, 1], [5, 2], [80, 95]])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_attend_of_scores_past_the_exponents_resolution(dtype, counts, dim):
    """Scores of 2^23 and more, of whole numbers that binary32 adds exactly; a token's is far from the next one's."""
    b = Both(12, 16, 1, dim, dtype, 6, dim, q_heads=2)
    b.ks[:] = 127 + 8
    b.k[:] = np.where(b.g.random(b.k.shape) < 0.5, 0x22, 0xAA)                 # 1 and -1
    b.wrap()
    q = dev(np.where(b.g.random((sum(counts), 2, dim)) < 0.5, 2.0 ** 13, -2.0 ** 13), KIND[dtype])
    attend_both(b, 2, counts, [80, 95], q=q, exact_scores=True)


@pytest.mark.parametrize("counts", [[1, 1], [3, 2], [40, 90]])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_of_very_low_scores(counts, dim):
    b = Both(12, 16, 1, dim, "bf16", 6, dim, q_heads=2)
    b.k[:], b.ks[:], b.vs[:] = 0xFF, 127 + 45, 126                             # -6 each
    b.wrap()
    q = torch.full((sum(counts), 2, dim), 2.0 ** 60, dtype=torch.bfloat16, device="cuda")
    out, lse, _ = attend_both(b, 2, counts, [80, 95], q=q, exact_scores=True, causal=False)
    # equal scores: the mean of the values
    starts = np.concatenate(([0], np.cumsum(counts)))
    assert (host(lse) < -1e30).all() and len(starts) == 3


@pytest.mark.parametrize("counts", [[1, 1], [3, 2], [40, 90]])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype,low,high,size", [
    ("f16", 104, 107, 2.0 ** 8), ("f16", 138, 141, 2.0 ** -6), ("f16", 104, 141, 1.0), ("f16", 138, 141, 2.0 ** -17),
    ("bf16", 7, 13, 2.0 ** 100), ("bf16", 240, 253, 2.0 ** -100), ("bf16", 7, 253, 2.0 ** -20), ("bf16", 247, 253, 2.0 ** -128)])
def test_attend_of_keys_at_the_ends_of_their_range(dtype, low, high, size, dim, counts):
    """Keys that are below the type's normal range (binary16) or close to its ends, and queries below their type's normal range."""
    b = Both(40, 16, 1, dim, dtype, 20, 90 + dim, q_heads=3)
    b.ks[:] = b.g.integers(low, high, b.ks.shape)
    b.wrap()
    q = rows(b.g, sum(counts), 3, dim, dtype, size)
    assert bool((q != 0).any(-1).all())
    # scores of about 1 where the scales are the largest (the root mean square of the codes is 2.95)
    attend_both(b, 3, counts, [301, 317], q=q, scale=1.0 / (2.95 * dim ** 0.5 * size * 2.0 ** (high - 128)))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("counts", [[1, 1], [3, 2], [40, 90]])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_of_equal_scores_is_the_mean_of_the_values(dtype, counts, dim):
    """Of very low scores (where the type has them), of 0 and of high ones."""
    for key, q in ((0xFF, 2.0 ** (60 if dtype == "bf16" else 10)), (0x00, 1.0), (0x77, 2.0 ** (60 if dtype == "bf16" else 10))):
        b = Both(12, 16, 1, dim, dtype, 6, dim + 1, q_heads=2)
        b.k[:], b.ks[:], b.vs[:] = key, 127 + (45 if dtype == "bf16" else 10), 126
        b.wrap()
        lengths, n = [80, 95], sum(counts)
        table = b.g.permutation(12).reshape(2, 6).astype(np.int32)
        out, _ = bits_of(b, torch.full((n, 2, dim), q, dtype=KIND[dtype], device="cuda"), table, [0, counts[0], n], lengths, max(counts), 95, None, False)
        for r, rows_of in enumerate((slice(0, counts[0]), slice(counts[0], n))):
            v = O.four_tokens_of(b.v, b.vs, table[r], lengths[r], 16, 6)[:, 0]
            want = v.mean(0)
            # equal weights are all rounded alike, by half a unit of 11 bits; a sum of 95 in binary32 and its quotient
            bound = HALF_ULP[dtype] * np.abs(want) + (2.0 ** -11 + 2.0 ** -24 * 110) * np.abs(v).mean(0) + TINY[dtype]
            assert (np.abs(host(out)[rows_of] - want) <= bound).all()


@pytest.mark.parametrize("kind", ["small", "large", "far apart", "zeros beside large"])
@pytest.mark.parametrize("heads", [(2, 2, 64), (8, 1, 128), (4, 2, 256)])
def test_attend_of_values_at_the_ends_of_their_range(kind, heads):
    """bfloat16 values of 2^-90 to 2^100, side by side in one element's sum, too."""
    hq, hk, dim = heads
    b = Both(40, 16, hk, dim, "bf16", 20, 60 + dim, q_heads=hq)
    low, high = {"small": (37, 40), "large": (220, 227), "far apart": (37, 227), "zeros beside large": (227, 228)}[kind]
    b.vs[:] = b.g.integers(low, high, b.vs.shape)
    if kind == "zeros beside large":
        b.v[::2], b.vs[::2] = 0, 127
    b.wrap()
    for counts in ([1, 1], [9, 3], [33, 300]):
        attend_both(b, hq, counts, [301, 317])
        attend_both(b, hq, counts, [301, 317], window=50)


def test_attend_of_a_sink_whose_values_are_tiny():
    """A token that takes nearly all the weight and whose values are 2^40 times smaller than the others'."""
    b = Both(40, 16, 1, 128, "bf16", 20, 61, q_heads=4)
    table = b.g.permutation(40).reshape(2, 20).astype(np.int32)
    b.k[table[:, 0], :, 0], b.ks[table[:, 0], :, :, 0] = 0x77, 127             # 6 each, along the queries
    b.vs[table[:, 0], :, :, 0] = 80
    b.wrap()
    q = rows(b.g, 90, 4, 128, "bf16") * 0.1 + 0.9
    for counts in ([1, 1], [2, 88]):
        attend_both(b, 4, counts, [301, 317], table=table, q=q[:sum(counts)].contiguous())


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_of_binary16_values_at_the_ends_of_their_range(dim):
    b = Both(40, 16, 1, dim, "f16", 20, 80 + dim, q_heads=3)
    for low, high in ((104, 106), (138, 141), (104, 141)):
        b.vs[:] = b.g.integers(low, high, b.vs.shape)
        if high == 141:
            b.v[:] = (b.v & 0x88) | np.minimum(b.v & 0x77, 0x44)               # (the mean of several 6 * 2^13 may pass binary16's range)
        b.wrap()
        for counts in ([1, 1], [50, 3]):
            attend_both(b, 3, counts, [301, 317])


def test_attend_gives_the_same_bits_again_on_another_stream_with_a_workspace_of_its_own():
    b = Both(620, 16, 2, 128, "f16", 300, 22, q_heads=16)
    table = dev(b.g.permutation(620)[:600].reshape(2, 300).astype(np.int32))
    starts, lengths = dev(np.array([0, 1, 2], np.int32)), dev(np.array([4800, 3333], np.int32))
    q = rows(b.g, 2, 16, 128, "f16")
    first = b.c.attend(b.m, q, table, starts, lengths, 1, 4800)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        ws = b.c.new_workspace(2, 2, 1, 4800)
        assert ws is not None
        outs = [b.c.attend(b.m, q, table, starts, lengths, 1, 4800, ws=ws) for _ in range(20)]
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, first)


def test_attend_reads_strided_queries_and_writes_strided_outputs():
    b = Both(30, 16, 2, 64, "f16", 10, 23, q_heads=4)
    for counts, lengths in (([1, 2, 2], [100, 150, 7]), ([90, 2, 2], [100, 150, 7])):
        n = sum(counts)
        qkv = rows(b.g, n, 8, 64, "f16")
        wide = torch.zeros((n, 11 * 64), dtype=torch.float16, device="cuda")
        table = dev(b.g.permutation(30).reshape(3, 10).astype(np.int32))
        starts, lengths = dev(np.concatenate(([0], np.cumsum(counts))).astype(np.int32)), dev(np.array(lengths, np.int32))
        want = b.c.attend(b.m, qkv[:, :4].contiguous(), table, starts, lengths, max(counts), 150)
        b.c.attend(b.m, qkv[:, :4], table, starts, lengths, max(counts), 150, out=wide[:, 128:384])
        assert torch.equal(wide[:, 128:384], want.flatten(1)) and (wide[:, :128] == 0).all() and (wide[:, 384:] == 0).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [(1, 1, 64), (2, 1, 128), (1, 1, 256)])
@pytest.mark.parametrize("rows_of", [15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 257])
def test_attend_around_the_lines_between_the_kernels(dtype, heads, rows_of):
    """The most rows of a kv head that a request has decide which kernel runs and with how many rows a workgroup."""
    hq, hk, dim = heads
    new = -(-rows_of // hq)
    for block, past in ((16, 0), (128, 300)):
        b = Both(2 * (new + past) // block + 6, block, hk, dim, dtype, (new + past) // block + 2, rows_of, q_heads=hq)
        attend_both(b, hq, [new, max(1, new // 2)], [new + past, new + past - 7 if past else new])


def test_attend_requests_of_one_call_in_two():
    """A call may cover a part of the requests: rows and requests are those of the whole step."""
    b = Both(60, 16, 2, 128, "f16", 20, 31, q_heads=8)
    table = dev(b.g.permutation(60).reshape(3, 20).astype(np.int32))
    starts, lengths = dev(np.array([0, 1, 2, 102], np.int32)), dev(np.array([200, 310, 100], np.int32))
    q = rows(b.g, 102, 8, 128, "f16")
    want = b.c.attend(b.m, q, table, starts, lengths, 100, 310)
    out = torch.zeros_like(want)
    b.c.attend(b.m, q, table[:2], starts[:3], lengths[:2], 1, 310, out=out)
    assert (out[2:] == 0).all()
    b.c.attend(b.m, q, table[2:], starts[2:], lengths[2:], 100, 100, out=out)
    # (other kernels sum in another order: a few units of an 11-bit significand)
    assert ((out - want).abs() <= 2.0 ** -9 * want.abs().amax(-1, keepdim=True)).all()


@pytest.mark.parametrize("requests", [2, 33, 64, 65])
def test_attend_of_many_heads_and_lengths_in_more_workgroups_than_run_at_once(requests):
    """Enough workgroups that they go by the requests' lengths (up to 64 requests), equal and zero lengths among them."""
    heads = min(1024, 4000 // requests)
    b = Both(3 * requests, 16, heads, 64, "f16", 4, requests, q_heads=heads)
    lengths = b.g.integers(0, 45, requests)
    lengths[0] = lengths[-1] = 44
    table = b.g.integers(0, 3 * requests, (requests, 4)).astype(np.int32)
    starts = dev(np.arange(requests + 1, dtype=np.int32))
    q = rows(b.g, requests, heads, 64, "f16")
    got = host(b.c.attend(b.m, q, dev(table), starts, dev(lengths.astype(np.int32)), 1, 4000))
    for h in (0, heads // 2, heads - 1):
        want, _, spread = O.four_attend(b.k[:, h:h + 1], b.v[:, h:h + 1], b.ks[:, h:h + 1], b.vs[:, h:h + 1], 16, 4, table, np.arange(requests + 1),
                                        lengths.astype(np.int32), host(q)[:, h:h + 1], 0.125, True, 0)
        bound = HALF_ULP["f16"] * np.abs(want) + (2.0 ** -11 + 2.0 ** -14) * spread + TINY["f16"] + 2.0 ** -32 * 45 * 6
        assert (np.abs(got[:, h:h + 1] - want) <= bound).all(), h


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("requests,heads,longest", [(40, (8, 8, 128), 90), (64, (8, 8, 64), 70), (5, (128, 64, 64), 70), (20, (16, 8, 128), 1500),
                                                    (32, (64, 8, 128), 700), (3, (24, 24, 64), 1300), (40, (16, 16, 64), 80), (33, (8, 8, 256), 60)])
def test_attend_where_long_and_short_requests_share_a_compute_unit(dtype, requests, heads, longest):
    """More than 256 workgroups, and no more than run at once: they go by the requests' lengths, those after 256 from the shortest on."""
    hq, hk, dim = heads
    b = Both(requests * -(-longest // 16) + 1, 16, hk, dim, dtype, -(-longest // 16), requests, q_heads=hq)
    lengths = b.g.integers(0, longest + 1, requests)
    lengths[0] = lengths[requests // 2] = longest
    counts = np.minimum(b.g.integers(0, 3, requests), lengths)
    attend_both(b, hq, counts, lengths, max_length=3000)         # (requests that may be short go in the order given)
    attend_both(b, hq, counts, lengths)
    attend_both(b, hq, np.ones(requests, int), np.full(requests, longest), max_length=1500)
    lengths[-1] = longest + 40                               # past the table
    table = b.g.integers(0, len(b.k), (requests, b.max_blocks)).astype(np.int32)
    attend_both(b, hq, counts, lengths, table=table, max_length=2000)
    attend_both(b, hq, counts, lengths, window=50, table=table)


@pytest.mark.parametrize("heads", [(2, 2, 64), (8, 1, 128), (4, 1, 256)])
def test_attend_one_request_far_longer_than_the_others(heads):
    hq, hk, dim = heads
    b = Both(700, 16, hk, dim, "f16", 600, 50, q_heads=hq)
    attend_both(b, hq, [1, 1, 0, 1], [30, 9001, 7, 0])
    attend_both(b, hq, [3, 9, 2], [30, 8500, 700], window=300)
    attend_both(b, hq, [40, 41], [40, 8400])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [(1, 1, 64), (8, 1, 128), (4, 2, 128), (2, 1, 256)])
def test_attend_single_tokens_beside_a_prompt(dtype, heads):
    hq, hk, dim = heads
    group, few = hq // hk, 32 if dim == 256 else 64
    line, long = few // group, 5 * few // group + 3
    b = Both(1200, 16, hk, dim, dtype, 600, 91, q_heads=hq)
    counts = [1, long, 1, line, 0, 1, line + 1, 2, 1, 1, 1, 1]
    attend_both(b, hq, counts, [300, long + 17, 1, line + 5, 9, 40, line + 1, 700, 16, 0, 129, 33])
    attend_both(b, hq, counts, [300, long, 1, line, 0, 40, line + 90, 2, 16, 17, 128, 33], window=21)
    attend_both(b, hq, counts, [300, long, 1, line, 0, 40, line + 90, 2, 16, 17, 128, 33], causal=False)
    attend_both(b, hq, [1] * 7 + [long], [5, 8300, 2, 1, 64, 0, 31, long + 1])
    attend_both(b, hq, [1] * 70 + [long], [1 + 7 * (r % 30) for r in range(70)] + [long], max_new=long + 40)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads,counts,lengths", [
    ((1, 1, 64), [1] * 7 + [600], [5000, 3, 4097, 700, 1, 0, 300, 650]),
    ((4, 2, 256), [1, 17, 2, 16, 0, 1, 300], [4500, 17, 2, 1000, 9, 0, 310]),
    ((8, 1, 128), [1] * 5 + [8, 9, 2] + [1] * 7 + [40], [3000, 1, 2, 63, 64, 1500, 700, 3, 0, 5, 6, 7, 8, 2500, 10, 60]),
    ((8, 8, 64), [1] * 19 + [300], [40 * r for r in range(19)] + [1000]),
])
def test_attend_single_tokens_beside_a_prompt_in_pieces(dtype, heads, counts, lengths):
    hq, hk, dim = heads
    b = Both(sum(-(-n // 16) for n in lengths) + 1, 16, hk, dim, dtype, 320, 92, q_heads=hq)
    attend_both(b, hq, counts, lengths, extra=2)
    attend_both(b, hq, counts, lengths, window=600)
    # announced shorter and longer than they are
    attend_both(b, hq, counts, lengths, max_length=1100)
    attend_both(b, hq, counts, lengths, max_length=140000)


@pytest.mark.parametrize("heads", [(1, 1, 64), (8, 1, 128), (4, 2, 256)])
@pytest.mark.parametrize("causal", [True, False])
def test_attend_windows_past_the_table(heads, causal):
    hq, hk, dim = heads
    b = Both(180, 16, hk, dim, "bf16", 30, 3, q_heads=hq)
    table = b.g.permutation(180).reshape(6, 30).astype(np.int32)
    for counts in ([1] * 6, [2, 150, 90, 1, 0, 3], [1, 150, 1, 1, 1, 2]):
        attend_both(b, hq, counts, [2000, 9000, 470, 481, 5, 700], window=700, table=table, causal=causal)
        attend_both(b, hq, counts, [2000, 2900, 470, 481, 480, 700], window=20, table=table, causal=causal)


def test_attend_of_a_window_past_32_bits_sees_everything():
    b = Both(20, 16, 1, 64, "f16", 20, 93, q_heads=2)
    for counts, lengths in (([1, 2], [100, 200]), ([90, 1], [120, 60])):
        attend_both(b, 2, counts, lengths, window=2 ** 32 + 5, max_new=2 ** 32 + max(counts), max_length=2 ** 32)


def test_a_long_cache_whose_bytes_pass_32_bits():
    """5 GB of keys: blocks past the first 4 GB are read, written and gathered where they are."""
    c = cachelib.Cache(5 * 2 ** 30 // (128 * 128 * 8), 128, 8, 8, 256, "bf16", 8, bits=4)
    m = c.new_memory()
    last = c.blocks - 1
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    k, v, q = (torch.randn((300, 8, 256), device="cuda", generator=g).bfloat16() for _ in range(3))
    ids = [last, last - 5, 3]
    table = torch.tensor([ids + [0] * 5], dtype=torch.int32, device="cuda")
    slots = torch.tensor([ids[t // 128] * 128 + t % 128 for t in range(300)], dtype=torch.int32, device="cuda")
    c.append(m, k, v, slots)
    starts, lengths = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 300], [300]))
    out = c.attend(m, q, table, starts, lengths, 300, 300)
    one = c.attend(m, q[-1:].contiguous(), table, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), lengths, 1, 300)
    kk, vv = torch.empty_like(k), torch.empty_like(v)
    c.gather(m, table, starts, lengths, kk, vv)
    few = cachelib.Cache(4, 128, 8, 8, 256, "bf16", 8, bits=4)
    small = few.new_memory()
    few.append(small, k, v, torch.arange(300, dtype=torch.int32, device="cuda"))
    there = torch.arange(8, dtype=torch.int32, device="cuda")[None]
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    few.gather(small, there, starts, lengths, k2, v2)
    assert torch.equal(kk, k2) and torch.equal(vv, v2) and (k.float() - kk.float()).abs().max() <= 1.0
    assert torch.equal(out, few.attend(small, q, there, starts, lengths, 300, 300))
    assert (one - out[-1:]).abs().max() <= 2.0 ** -6 * out[-1:].abs().max()


# ------------------------------------------------------------------ rotation by positions of several axes

def many_axes(g, axes, half, order):
    cuts = np.sort(g.integers(0, half + 1, axes - 1))
    return np.diff(np.concatenate(([0], cuts, [half]))).tolist(), order


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [(1, 1), (12, 12), (40, 8), (7, 1)])
@pytest.mark.parametrize("dim,rotary", [(64, 64), (64, 16), (128, 128), (128, 48), (256, 256), (256, 64)])
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
def test_norm_rotate_by_several_axes(dtype, heads, dim, rotary, pairs):
    g = np.random.default_rng(dim + rotary)
    hq, hk = heads
    for tokens, normed, packed, axes, order in ((1, True, False, 3, "runs"), (5, False, True, 2, "turns"), (67, True, True, 3, "turns"), (3, True, True, 4, "runs"),
                                                (2, False, True, 1, "runs")):
        c = cachelib.Cache(1, 16, hq, hk, dim, dtype, 1, bits=4)
        width = (hq + 2 * hk) * dim
        x = dev(g.standard_normal((tokens, width)) * g.choice([0.01, 1.0, 30.0], (1, width)), KIND[dtype])
        q, k = x[:, :hq * dim], x[:, hq * dim:(hq + hk) * dim]
        if not packed:
            q, k = q.contiguous().view(tokens, hq, dim), k.contiguous().view(tokens, hk, dim)
        angles = g.uniform(-1, 1, (300, rotary)).astype(np.float32)
        positions = g.integers(0, 300, (axes, tokens)).astype(np.int32)
        axis = c.new_axes(many_axes(g, axes, rotary // 2, order)[0], order)
        weights = [dev(g.standard_normal(dim), KIND[dtype]) if normed else None for _ in range(2)]
        got = c.norm_rotate(q, k, dev(positions), dev(angles), weights[0], weights[1], 1e-5, pairs, axes=axis)
        for y, z, h, w in ((q, got[0], hq, weights[0]), (k, got[1], hk, weights[1])):
            src, more = host(y).reshape(tokens, h, dim), (positions, host(axis), rotary, pairs == "neighbours")
            want = O.norm_rotate_axes(src, None if w is None else host(w), 1e-5, angles, *more)
            # one rounding to 16 bits, and a few in binary32 of the two products
            size = np.abs(O.norm_rotate_axes(np.abs(src), None if w is None else np.abs(host(w)), 1e-5, np.abs(angles), *more))
            size = np.maximum(size, np.abs(want)).max(-1, keepdims=True)
            assert (np.abs(host(z) - want) <= HALF_ULP[dtype] * np.abs(want) + 2.0 ** -18 * size + TINY[dtype]).all()


@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
def test_norm_rotate_by_axes_that_stand_at_one_place_is_that_by_one(pairs):
    g = np.random.default_rng(7)
    c = cachelib.Cache(1, 16, 8, 2, 128, "bf16", 1)
    x = rows(g, 33, 10, 128, "bf16")
    angles, w = dev(g.uniform(-1, 1, (50, 128)).astype(np.float32)), dev(g.standard_normal(128), torch.bfloat16)
    positions = dev(g.integers(0, 50, 33).astype(np.int32))
    want = c.norm_rotate(x[:, :8], x[:, 8:], positions, angles, w, w, pairs=pairs)
    for order in ("runs", "turns"):
        got = c.norm_rotate(x[:, :8], x[:, 8:], positions.expand(3, 33).contiguous(), angles, w, w, pairs=pairs, axes=c.new_axes((24, 20, 20), order))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_norm_rotate_by_axes_in_place_without_a_position_and_past_the_angles():
    g = np.random.default_rng(5)
    c = cachelib.Cache(1, 16, 4, 2, 128, "bf16", 1)
    x = dev(g.standard_normal((8, 8 * 128)), torch.bfloat16)
    before = x.clone()
    q, k = x[:, :512], x[:, 512:768]
    angles = dev(g.uniform(-1, 1, (50, 128)).astype(np.float32))
    positions = dev(np.array([[0, -1, 49, 3, 3, 3, 7, 8], [0, 1, 49, -5, 50, 3, 7, 9], [0, 2, 49, 3, 3, 2 ** 31 - 1, -1, 10]], np.int32))
    axis = c.new_axes((16, 24, 24))
    w = dev(g.standard_normal(128), torch.bfloat16)
    want = c.norm_rotate(q, k, positions, angles, w, w, axes=axis)
    c.norm_rotate(q, k, positions, angles, w, w, q_out=q, k_out=k, axes=axis)
    for a, b in ((q, want[0]), (k, want[1])):
        assert torch.equal(a[[0, 2, 7]], b.flatten(1)[[0, 2, 7]])
        assert a[[4, 5]].isnan().all()                       # past the angles
    assert torch.equal(x[[1, 3, 6]], before[[1, 3, 6]]) and torch.equal(x[:, 768:], before[:, 768:])
    # a pair whose axis there is not
    axis[9] = 3
    got = c.norm_rotate(x[7:, :512], x[7:, 512:768], positions[:, 7:].contiguous(), angles, w, w, axes=axis)[0]
    assert got[0, :, [9, 73]].isnan().all() and int(got.isnan().sum()) == 2 * 4


def test_norm_rotate_by_axes_of_no_tokens():
    c = cachelib.Cache(1, 16, 1, 1, 64, "f16", 1)
    x = torch.empty((0, 64), dtype=torch.float16, device="cuda")
    q, k = c.norm_rotate(x, x, torch.empty((3, 0), dtype=torch.int32, device="cuda"), torch.zeros((1, 64), device="cuda"), axes=c.new_axes((12, 10, 10)))
    assert q.shape == (0, 1, 64) and k.shape == (0, 1, 64)


# ------------------------------------------------------------------ the step as a whole, and refusals

def test_a_step_in_a_graph_replayed_with_other_data_between():
    """All operators of a step, captured once and replayed among eager steps of a cache of its own; both split the cache's length."""
    requests, start = 3, 700
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    angles = torch.rand((800, 128), device="cuda", generator=g)
    new = torch.ones(requests, dtype=torch.int32, device="cuda")
    x = torch.zeros((requests, 12 * 128), dtype=torch.bfloat16, device="cuda")

    class Side:
        def __init__(self):
            c = self.c = cachelib.Cache(160, 16, 8, 2, 128, "bf16", 50, bits=4)
            self.memory, self.table, self.ring = c.new_memory(), c.new_table(requests), c.new_ring()
            self.lengths, self.counters = c.new_lengths(requests), c.new_counters()
            self.out, self.y = c.new_schedule(requests, requests), torch.zeros((requests, 8, 128), dtype=torch.bfloat16, device="cuda")
            self.axis, self.ws = c.new_axes((16, 24, 24)), c.new_workspace(requests, requests, 1, 800)
            first = c.new_schedule(requests, requests * start)
            c.schedule(new * start, self.lengths, self.table, self.ring, self.counters, first)
            torch.manual_seed(2)
            k = torch.randn((requests * start, 2, 128), device="cuda").bfloat16()
            c.append(self.memory, k, k.flip(0), first.slots)
            self.lengths.copy_(first.lengths)
            self.counters.copy_(first.counters)

        def step(self):
            c, o = self.c, self.out
            c.schedule(new, self.lengths, self.table, self.ring, self.counters, o)
            places = torch.stack((o.positions, o.positions % 48, o.positions // 48))
            q, k = c.norm_rotate(x[:, :1024], x[:, 1024:1280], places, angles, axes=self.axis)
            c.append(self.memory, k, x[:, 1280:].unflatten(1, (2, 128)), o.slots)
            c.attend(self.memory, q, self.table, o.starts, o.lengths, 1, 800, out=self.y, ws=self.ws)
            self.lengths.copy_(o.lengths)
            self.counters.copy_(o.counters)

    warm, captured, eager = Side(), Side(), Side()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm.step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.step()
    for i in range(40):
        x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        assert torch.equal(captured.y, eager.y) and torch.equal(captured.lengths, eager.lengths) and torch.equal(captured.table, eager.table), i
        assert captured.y.isfinite().all()
    assert int(captured.lengths[0]) == start + 40


@pytest.mark.parametrize("dtype,heads", [("f16", (8, 1, 128)), ("bf16", (8, 1, 128)), ("bf16", (4, 2, 64)), ("bf16", (2, 1, 256))])
def test_calls_at_once_on_two_streams_and_graphs_that_share_a_workspace(dtype, heads):
    """Each of two memories needs the second pass somewhere, and each call is in pieces; the graphs' calls follow one another."""
    hq, hk, dim = heads
    sides = []
    for seed in (1, 2):
        b = Both(200, 16, hk, dim, dtype, 190, seed, q_heads=hq)
        b.vs[seed::7, 0, 0, 3] = 127 - 22
        b.wrap()
        table = dev(np.stack([b.g.permutation(200)[:190], b.g.permutation(200)[:190]]).astype(np.int32))
        for counts, lengths in (((1, 1), (3000, 2900)), ((40, 30), (3000, 1700))):
            starts = dev(np.array([0, counts[0], sum(counts)], np.int32))
            q, ws = rows(b.g, sum(counts), hq, dim, dtype), b.c.new_workspace(2, sum(counts), max(counts), 3000)
            assert ws is not None
            call = (b.m, q, table, starts, dev(np.array(lengths, np.int32)), max(counts), 3000)
            sides.append((b, call, ws, b.c.attend(*call, out=torch.empty_like(q), ws=ws)))
    for one, two in ((sides[0], sides[2]), (sides[1], sides[3]), (sides[0], sides[3])):
        torch.cuda.synchronize()
        streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.full_like(x[3], 7.0) for x in (one, two)]
        torch.cuda.synchronize()
        for _ in range(20):
            for (b, call, ws, _), stream, out in zip((one, two), streams, outs):
                with torch.cuda.stream(stream):
                    b.c.attend(*call, out=out, ws=ws)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], one[3]) and torch.equal(outs[1], two[3])
    shared = max((x[2] for x in sides), key=lambda ws: ws.numel())
    graphs, outs = [], [torch.full_like(x[3], 7.0) for x in sides]
    for (b, call, _, _), out in zip(sides, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.c.attend(*call, out=out, ws=shared)
        graphs.append(graph)
    for _ in range(3):
        for out in outs:
            out.fill_(7.0)
        for graph in graphs + graphs[::-1]:
            graph.replay()
        torch.cuda.synchronize()
        for (_, _, _, want), out in zip(sides, outs):
            assert torch.equal(out, want)


def test_calls_of_no_tokens_do_nothing():
    b = Both(4, 16, 2, 128, "f16", 2, 40, q_heads=4)
    none, starts, lengths, table = dev(np.zeros(0, np.int32)), dev(np.zeros(3, np.int32)), dev(np.array([5, 0], np.int32)), dev(np.zeros((2, 2), np.int32))
    k, v = (torch.empty((0, 2, 128), dtype=torch.float16, device="cuda") for _ in range(2))
    b.c.append(b.m, k, v, none)
    b.c.gather(b.m, table, starts, lengths, k, v)
    q = torch.empty((0, 4, 128), dtype=torch.float16, device="cuda")
    assert b.c.attend(b.m, q, table, starts, lengths, 0, 5).shape == (0, 4, 128)
    b.same()


@pytest.mark.parametrize("call", ["norm_rotate", "append", "gather", "attend", "wrap", "new_axes"])
def test_what_does_not_fit_is_refused(call):
    c = cachelib.Cache(4, 16, 4, 2, 128, "f16", 2, bits=4)
    m, eight = c.new_memory(), cachelib.Cache(4, 16, 4, 2, 128, "f16", 2).new_memory()
    h = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda")        # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")          # noqa: E731
    if call == "norm_rotate":
        axes = c.new_axes((16, 24, 24))
        good = [h(3, 4, 128), h(3, 2, 128), i(3, 3), torch.zeros((9, 128), device="cuda"), None, None, 1e-6, "halves", None, None, axes]
        wrong = [(2, i(3)), (2, i(5, 3)), (2, i(3, 2)), (2, i(0, 3)), (2, i(3, 3).long()), (2, i(3, 6)[:, ::2]), (10, axes[:32]), (10, axes.int()), (10, axes.cpu()),
                 (10, axes.repeat(2)[::2])]
        f = c.norm_rotate
    elif call == "append":
        good = [m, h(3, 2, 128), h(3, 2, 128), i(3)]
        wrong = [(0, eight), (1, h(3, 4, 128)), (2, h(4, 2, 128)), (3, i(4)), (3, i(6)[::2])]
        f = c.append
    elif call == "gather":
        good = [m, i(2, 2), i(3), i(2), h(3, 2, 128), h(3, 2, 128)]
        wrong = [(0, eight), (1, i(2, 3)), (2, i(2)), (4, h(3, 2, 64)), (5, h(2, 2, 128))]
        f = c.gather
    elif call == "attend":
        good = [m, h(3, 4, 128), i(2, 2), i(3), i(2), 2, 9]
        wrong = [(0, eight), (1, h(3, 2, 128)), (2, i(3, 2)), (3, i(4)), (4, i(2).long()), (5, -1), (6, -1)]
        f = c.attend
    elif call == "new_axes":
        good = [(16, 24, 24), "runs"]
        wrong = [(0, ()), (0, (1, 2)), (0, (16, 24, 32)), (0, (8, 8, 8, 8, 8)), (0, (-8, 16)), (0, (0, 0)), (1, "blocks")]
        f = c.new_axes
    else:
        good = [m.k, m.v, m.k_scale, m.v_scale]
        wrong = [(0, m.k.char()), (0, m.k[..., :32]), (1, m.v.char()), (1, m.v.transpose(2, 3)), (2, m.k_scale.cpu()), (2, m.k_scale.float()), (3, m.v_scale[:3]),
                 (3, m.v_scale.transpose(2, 3))]
        f = c.wrap
    f(*good)
    for at, x in wrong:
        args = list(good)
        args[at] = x
        with pytest.raises(ValueError):
            f(*args)


def test_a_memory_in_other_bits_is_refused_by_a_cache_in_8():
    c = cachelib.Cache(4, 16, 4, 2, 128, "f16", 2)
    four = cachelib.Cache(4, 16, 4, 2, 128, "f16", 2, bits=4).new_memory()
    k, slots = torch.zeros((1, 2, 128), dtype=torch.float16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="the memory is that of"):
        c.append(four, k, k, slots)
    with pytest.raises(ValueError):
        cachelib.Cache(4, 16, 4, 2, 128, "f16", 2, bits=6)


@pytest.mark.parametrize("call", ["norm_rotate", "append", "gather", "attend"])
def test_tensors_on_another_device_than_the_current_one_are_refused(call, monkeypatch):
    c = cachelib.Cache(4, 16, 4, 2, 128, "f16", 2, bits=4)
    m = c.new_memory()
    h = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda")        # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")          # noqa: E731
    args = dict(norm_rotate=[h(3, 4, 128), h(3, 2, 128), i(3, 3), torch.zeros((9, 128), device="cuda"), None, None, 1e-6, "halves", None, None, c.new_axes((16, 24, 24))],
                append=[m, h(3, 2, 128), h(3, 2, 128), i(3) - 1],
                gather=[m, i(2, 2), i(3), i(2), h(3, 2, 128), h(3, 2, 128)],
                attend=[m, h(3, 4, 128), i(2, 2), i(3), i(2), 2, 9])[call]
    getattr(c, call)(*args)
    # as if another device had been made the current one
    monkeypatch.setattr(cachelib, "_device", lambda: torch.cuda.current_device() + 1)
    with pytest.raises(ValueError, match="current"):
        getattr(c, call)(*args)
