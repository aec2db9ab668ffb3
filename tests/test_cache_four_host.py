"""Host-only checks of what a cache in 4 bits and the rotation by several axes add to the C ABI, and of their oracle against what
is known without it.  No kernel is launched here."""
import ctypes as C

import numpy as np
import pytest

from oracle import cache_oracle as O
from paper_2511_04002_amd import build as tsq_build
from paper_2511_04002_amd import cache, tsq

BAD, UNS = tsq.TSQ_ERR_INVALID_ARG, tsq.TSQ_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def L():
    tsq_build.build()
    return cache.lib()


def cfg(**kw):
    base = dict(blocks=10, block_tokens=16, q_heads=8, kv_heads=2, head_dim=128, dtype=tsq.TSQ_F16, max_blocks=4, reserved=0)
    base.update(kw)
    return cache.tsq_cache_config(**base)


@pytest.fixture()
def handle(L):
    h = cache.tsq_cache_create_bits(cfg(), 4)
    yield h
    cache.tsq_cache_destroy(h)


def test_create(L):
    h, c = C.c_void_p(), cfg()
    assert L.tsq_cache_create_bits(None, 4, C.byref(h)) == BAD and L.tsq_cache_create_bits(C.byref(c), 4, None) == BAD
    for bits in (0, 1, 2, 3, 5, 7, 16, 2 ** 32 - 1):
        assert L.tsq_cache_create_bits(C.byref(c), bits, C.byref(h)) == BAD and not h.value
    for kw in (dict(blocks=0), dict(reserved=4), dict(q_heads=9), dict(dtype=2)):
        with pytest.raises(tsq.TsqError):
            cache.tsq_cache_create_bits(cfg(**kw), 4)


def test_memory_sizes(L, handle):
    s = cache.tsq_cache_memory_sizes(handle)
    assert s.code_bytes == 10 * 2 * 16 * 64 and s.scale_bytes == 10 * 2 * 16 * 4
    h = cache.tsq_cache_create_bits(cfg(), 8)
    t = cache.tsq_cache_memory_sizes(h)
    assert t.code_bytes == 2 * s.code_bytes and t.scale_bytes == 10 * 2 * 4
    cache.tsq_cache_destroy(h)


MEM = dict(d_k=0x10000, d_v=0x20000, d_k_scale=0x30000, d_v_scale=0x40000)


def memory(**kw):
    return C.byref(cache.tsq_cache_memory(**{**MEM, **kw}))


def refused(f, good, changes):
    """Each change of one argument of a call that would be good is refused (the good call itself is not made)."""
    for name, value, status in changes:
        assert name in good
        assert f(*{**good, name: value}.values()) == status, (name, value)


def test_norm_rotate_axes_refuses(L, handle):
    good = dict(cache=handle, tokens=5, q=0x1000, q_stride=1024, k=0x2000, k_stride=256, axes=3, positions=0x3000, axis=0x3800, angles=0x4000,
                angle_rows=9, rotary=128, pairs=0, qw=0x5000, kw=0x6000, eps=1e-6, q_out=0x7000, q_out_stride=1024, k_out=0x8000, k_out_stride=256,
                stream=None)
    f = L.tsq_cache_norm_rotate_axes
    refused(f, good, [(n, None, BAD) for n in ("cache", "q", "k", "positions", "axis", "angles", "q_out", "k_out")] +
            [("axes", 0, BAD), ("axes", 5, BAD), ("axis", 0x3804, BAD), ("positions", 0x3002, BAD), ("q", 0x1008, BAD), ("rotary", 24, BAD), ("rotary", 144, BAD),
             ("pairs", 2, BAD), ("eps", -1.0, BAD), ("q_stride", 1016, BAD), ("tokens", 1 << 31, BAD)])
    assert f(*{**good, "tokens": 0, "q": None, "axis": None}.values()) == tsq.TSQ_OK


def test_calls_refuse(L, handle):
    good = dict(cache=handle, memory=memory(), tokens=5, k=0x1000, k_stride=256, v=0x2000, v_stride=256, slots=0x3000, stream=None)
    refused(L.tsq_cache_append, good, [(n, None, BAD) for n in ("cache", "memory", "k", "v", "slots")] +
            [("memory", memory(**{n: MEM[n] + 8}), BAD) for n in MEM] + [("k", 0x1004, BAD), ("v_stride", 128, BAD), ("slots", 0x3001, BAD)])
    assert L.tsq_cache_append(handle, memory(), 0, None, 0, None, 0, None, None) == tsq.TSQ_OK
    good = dict(cache=handle, memory=memory(), requests=2, table=0x1000, starts=0x2000, lengths=0x3000, tokens=5, k=0x4000, k_stride=256,
                v=0x5000, v_stride=256, stream=None)
    refused(L.tsq_cache_gather, good, [(n, None, BAD) for n in ("cache", "memory", "table", "starts", "lengths", "k", "v")] +
            [("requests", 0, BAD), ("requests", 65536, UNS), ("k", 0x4004, BAD)])
    good = dict(cache=handle, memory=memory(), requests=2, table=0x1000, starts=0x2000, lengths=0x3000, tokens=5, max_new=4, max_length=4096,
                q=0x4000, q_stride=1024, scale=0.1, causal=1, window=0, out=0x5000, out_stride=1024, lse=0x6000, ws=0x7000, stream=None)
    refused(L.tsq_cache_attend, good, [(n, None, BAD) for n in ("cache", "memory", "table", "starts", "lengths", "q", "out", "ws")] +
            [("requests", 65536, UNS), ("tokens", 1 << 28, UNS), ("q", 0x4008, BAD), ("scale", 0.0, BAD), ("causal", 2, BAD), ("ws", 0x7010, BAD)])


def test_calls_of_too_many_threads_are_refused_before_anything_is_enqueued(L):
    h = cache.tsq_cache_create_bits(cfg(q_heads=1, kv_heads=1, head_dim=64), 4)
    assert L.tsq_cache_norm_rotate_axes(h, 1 << 26, 0x1000, 64, 0x2000, 64, 3, 0x3000, 0x3800, 0x4000, 9, 64, 0, None, None, 1e-6, 0x5000, 64, 0x6000, 64, None) == UNS
    assert L.tsq_cache_append(h, memory(), 1 << 30, 0x1000, 64, 0x2000, 64, 0x3000, None) == UNS
    assert L.tsq_cache_gather(h, memory(), 2, 0x1000, 0x2000, 0x3000, 1 << 30, 0x4000, 64, 0x5000, 64, None) == UNS
    cache.tsq_cache_destroy(h)
    h = cache.tsq_cache_create_bits(cfg(q_heads=1024, kv_heads=1024, head_dim=64), 4)
    assert L.tsq_cache_attend(h, memory(), 65535, 0x1000, 0x2000, 0x3000, 1 << 17, 1 << 17, 64, 0x4000, 65536, 0.1, 1, 0, 0x5000, 65536, None, 0x10000, None) == UNS
    cache.tsq_cache_destroy(h)


def test_attend_of_256_tokens_needs_no_workspace(L):
    for heads, dim in ((1, 64), (8, 128), (1, 256)):
        h = cache.tsq_cache_create_bits(cfg(q_heads=heads, kv_heads=1, head_dim=dim), 4)
        for tokens, new in ((1, 1), (7, 7), (256, 256), (5000, 1)):
            assert cache.tsq_cache_attend_workspace_bytes(h, 1, tokens, new, 256) == 0
        cache.tsq_cache_destroy(h)


# ------------------------------------------------------------------ the oracle

def test_the_oracles_numbers_by_hand():
    x = np.zeros((4, 32))
    x[0, :5] = 7, 0.25, 0.75, -5, 3.5                        # a scale of 1: 7 is 6, ties go to 0, 1, -4 and 4
    x[1, :2] = 7.0001, -3                                    # a scale of 2
    x[2, 0] = 2.0 ** -30
    byte = O.four_scale(x, "f16")
    assert byte.tolist() == [127, 128, 104, 127]
    code = O.four_code(x, byte.astype(float))
    assert O.FOUR[code][0, :5].tolist() == [6, 0, 1, -4, 4] and O.FOUR[code][1, :2].tolist() == [4, -1.5] and code[2:].sum() == 0
    assert O.four_scale(np.full((1, 32), 65504.0), "f16")[0] == 140 and O.four_scale(np.full((1, 32), 3e38), "bf16")[0] == 252
    assert O.four_scale(np.full((1, 32), 2.0 ** -30), "bf16")[0] == 127 - 32


def test_the_oracles_numbers_are_the_nearest_and_come_back():
    g = np.random.default_rng(0)
    x = g.standard_normal((300, 32)) * np.exp2(g.integers(-6, 6, (300, 1)))
    byte = O.four_scale(x, "bf16").astype(float)
    y = O.FOUR[O.four_code(x, byte)] * 2.0 ** (byte - 127)[:, None]
    a = np.abs(x) / 2.0 ** (byte - 127)[:, None]
    assert (a.max(-1) <= 7).all() and (a.max(-1) > 3.5).all()
    assert (np.abs(x - y) / 2.0 ** (byte - 127)[:, None] <= np.where(a <= 2, 0.25, np.where(a <= 4, 0.5, 1))).all()
    # what is there already is stored as it is, at the scale that it had or at half of it
    again = O.four_scale(y, "bf16").astype(float)
    assert np.array_equal(O.FOUR[O.four_code(y, again)] * 2.0 ** (again - 127)[:, None], y)


def test_the_oracles_cache_and_attention():
    g = np.random.default_rng(1)
    k, v = (np.full((3, 2, 16, 32), 0x77, np.uint8) for _ in range(2))
    ks, vs = (np.full((3, 2, 2, 16), 130, np.uint8) for _ in range(2))
    x, y = (O.FOUR[g.integers(0, 16, (20, 2, 64))] for _ in range(2))
    x[..., ::32], y[..., ::32] = 6, -6                       # (so that every scale is 1)
    O.four_append(k, v, ks, vs, x, y, np.array([32 + i if i < 16 else i - 16 for i in range(20)]), 16, "f16")
    assert np.array_equal(O.four_tokens_of(k, ks, [2, 0], 20, 16, 2), x) and np.array_equal(O.four_tokens_of(v, vs, [2, 0], 20, 16, 2), y)
    assert np.isnan(O.four_tokens_of(k, ks, [2, 3], 20, 16, 2)[16:]).all()
    assert (k[1] == 0x77).all() and (ks[0, :, :, 4:] == 130).all()
    q = g.standard_normal((3, 4, 64))
    out, lse, spread = O.four_attend(k, v, ks, vs, 16, 2, np.array([[2, 0]]), np.array([0, 3]), np.array([20]), q, 0.3, True, 0)
    for i in range(3):
        for h in range(4):
            s = x[:18 + i, h // 2] @ q[i, h] * 0.3
            w = np.exp(s - s.max())
            assert np.allclose(out[i, h], w @ y[:18 + i, h // 2] / w.sum()) and np.isclose(lse[i, h], s.max() + np.log(w.sum()))
    x[3, 1, 40] = np.inf
    O.four_append(k, v, ks, vs, x[3:4], y[3:4], np.array([5]), 16, "f16")
    assert (ks[0, 1, :, 5] == 255).all() and (vs[0, 1, :, 5] == 255).all() and (ks[0, 0, :, 5] == 127).all()


def test_the_oracles_rotation_by_axes():
    g = np.random.default_rng(2)
    x, angles = g.standard_normal((5, 3, 64)), g.uniform(-1, 1, (40, 32))
    at = g.integers(0, 40, 5)
    for neighbours in (False, True):
        one = O.norm_rotate(x, None, 0.0, angles, at, 32, neighbours)
        assert np.array_equal(O.norm_rotate_axes(x, None, 0.0, angles, np.stack((at, at, at)), g.integers(0, 3, 16), 32, neighbours), one)
        other = O.norm_rotate_axes(x, None, 0.0, angles, np.stack((at, (at + 1) % 40)), np.arange(16) // 15, 32, neighbours)
        last = (30, 31) if neighbours else (15, 31)
        assert np.array_equal(np.delete(other, last, -1), np.delete(one, last, -1)) and not np.allclose(other[..., last], one[..., last])
        lost = O.norm_rotate_axes(x, None, 0.0, angles, np.stack((at, at + 40)), np.zeros(16, int), 32, neighbours)
        assert np.isnan(lost).all()
