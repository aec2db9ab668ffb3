"""The serving operators' oracle against what is known without it: examples worked by hand, closed forms, and the same
formulas in another form."""
import numpy as np
import torch

from oracle import cache_oracle as O


def test_schedule_by_hand():
    # blocks of 16; request 0 grows from 15 to 17 tokens (one new block), 1 is done (two blocks back), 2 begins with 20 (two blocks)
    table = np.array([[4, -1, -1], [7, 2, -1], [-1, -1, -1]], np.int32)
    ring = np.array([6, 9, 9, 0, 1, 3, 5, 9], np.int32)                    # free: places 3, 4, 5, 6, then 0 of the next round
    got = O.schedule(np.array([2, -1, 20]), np.array([15, 30, 0]), table, ring, np.array([3, 10]), 16, 3, 24)
    assert got["status"] == O.INVALID                                      # seven free and two that come back: the ring has eight
    ring = np.array([6, 9, 9, 0, 1, 3, 5, 9], np.int32)
    got = O.schedule(np.array([2, -1, 20]), np.array([15, 30, 0]), table, ring, np.array([3, 7]), 16, 3, 24)
    assert got["status"] == O.OK and got["counters"].tolist() == [6, 9] and got["lengths"].tolist() == [17, 0, 20]
    assert got["starts"].tolist() == [0, 2, 2, 22]
    assert got["table"].tolist() == [[4, 0, -1], [7, 2, -1], [1, 3, -1]]
    assert got["ring"].tolist() == [2, 9, 9, 0, 1, 3, 5, 7]                # 7 at place 7, 2 at place 8 mod 8
    assert got["positions"].tolist() == [15, 16] + list(range(20)) + [-1, -1]
    assert got["slots"].tolist() == [4 * 16 + 15, 0] + [16 + i for i in range(16)] + [3 * 16 + i for i in range(4)] + [-1, -1]


def test_norm_leaves_unit_rms_and_rotation_keeps_lengths():
    g = np.random.default_rng(0)
    x = g.standard_normal((5, 3, 64)) * 7
    angle = g.uniform(0, 6, (9, 16))
    angles = np.concatenate((np.cos(angle), np.sin(angle)), 1)
    for neighbours in (False, True):
        y = O.norm_rotate(x, np.ones(64), 0.0, angles, np.array([0, 3, 8, 8, 1]), 32, neighbours)
        assert np.allclose((y * y).mean(-1), 1, atol=1e-12)
        z = O.norm_rotate(x, None, 0.0, angles, np.array([0, 3, 8, 8, 1]), 32, neighbours)
        assert np.allclose((z * z).sum(-1), (x * x).sum(-1)) and np.array_equal(z[..., 32:], x[..., 32:])
    # a pair turned by a known angle: (1, 0) by 90 degrees is (0, 1)
    one = np.zeros((1, 1, 64))
    one[..., 2] = 1
    turn = np.concatenate((np.zeros((1, 16)), np.ones((1, 16))), 1)
    assert O.norm_rotate(one, None, 0.0, turn, np.array([0]), 32, False)[0, 0].nonzero()[0].tolist() == [18]
    assert O.norm_rotate(one, None, 0.0, turn, np.array([0]), 32, True)[0, 0].nonzero()[0].tolist() == [3]
    assert np.isnan(O.norm_rotate(one, None, 0.0, turn, np.array([1]), 32, True)).all()


def cache(blocks, heads, block, dim):
    return (np.zeros((blocks, heads, block, dim), np.int8), np.zeros((blocks, heads, dim, block), np.int8),
            np.full((blocks, heads), 5, np.float32), np.full((blocks, heads), 5, np.float32))


def test_append_by_hand():
    k, v, ks, vs = cache(2, 1, 16, 64)
    x = np.zeros((3, 1, 64), np.float32)
    x[0, 0, 0], x[1, 0, 1], x[2, 0, 2] = 127, 63.5, -254
    O.append(k, v, ks, vs, x[:1], x[:1], [16], 16)
    assert ks[1, 0] == 1 and k[1, 0, 0, 0] == 127 and v[1, 0, 0, 0] == 127 and ks[0, 0] == 5
    O.append(k, v, ks, vs, x[1:2], x[1:2], [17], 16)                       # smaller: the scale stays; 63.5 is a tie, to even
    assert ks[1, 0] == 1 and k[1, 0, 1, 1] == 64
    O.append(k, v, ks, vs, x[2:], x[2:], [18], 16)                         # larger: what is there is halved, 127 to 64 (63.5 to even)
    assert ks[1, 0] == 2 and k[1, 0, 0, 0] == 64 and k[1, 0, 1, 1] == 32 and k[1, 0, 2, 2] == -127 and v[1, 0, 2, 2] == -127


def test_append_is_within_half_a_step_and_a_run_is_as_good_as_its_largest():
    g = np.random.default_rng(1)
    k, v, ks, vs = cache(3, 2, 32, 64)
    x = g.standard_normal((90, 2, 64)).astype(np.float32)
    O.append(k, v, ks, vs, x, 3 * x, range(90), 32)
    got = O.tokens_of(k, ks, np.arange(3), 90, 32, 3)
    for b in range(3):
        part = slice(32 * b, min(90, 32 * b + 32))
        assert np.array_equal(ks[b], np.abs(x[part]).max((0, 2)) / np.float32(127))
        assert (np.abs(got[part] - x[part]) <= 0.5 * ks[b][:, None] * (1 + 1e-5)).all()
    assert np.allclose(vs, 3 * ks)


def test_attend_against_torch_in_64_bits():
    g = np.random.default_rng(2)
    block, heads, group, dim, lengths, counts = 16, 2, 3, 64, [37, 5, 20], [4, 5, 1]
    k = g.integers(-127, 128, (9, heads, block, dim)).astype(np.int8)
    v = g.integers(-127, 128, (9, heads, dim, block)).astype(np.int8)
    ks, vs = (g.uniform(0.01, 0.02, (9, heads)).astype(np.float32) for _ in range(2))
    table = np.array([[8, 0, 3], [1, -1, -1], [2, 7, -1]], np.int32)
    starts = np.concatenate(([0], np.cumsum(counts)))
    q = g.standard_normal((10, heads * group, dim))
    for causal, window in ((True, 0), (False, 0), (True, 3), (False, 7)):
        out, lse, spread = O.attend(k, v, ks, vs, block, 3, table, starts, np.array(lengths), q, 0.1, causal, window)
        for r, (n, length) in enumerate(zip(counts, lengths)):
            ids = table[r, :-(-length // block)]
            keys = torch.from_numpy(np.concatenate([k[i].astype(float) * ks[i][:, None, None] for i in ids], 1)[:, :length])
            values = torch.from_numpy(np.concatenate([(v[i].astype(float) * vs[i][:, None, None]).swapaxes(1, 2) for i in ids], 1)[:, :length])
            rows = torch.from_numpy(q[starts[r]:starts[r + 1]]).view(n, heads, group, dim)
            s = torch.einsum("nhgd,htd->nhgt", rows, keys) * 0.1
            at, t = torch.arange(length - n, length)[:, None], torch.arange(length)[None]
            hidden = torch.zeros(n, length, dtype=torch.bool)
            if causal:
                hidden |= t > at
            if window:
                hidden |= t <= at - window
            s = s.masked_fill(hidden[:, None, None], -torch.inf)
            want = torch.einsum("nhgt,htd->nhgd", s.softmax(-1), values).reshape(n, heads * group, dim)
            part = slice(starts[r], starts[r + 1])
            assert np.allclose(out[part], want.numpy(), atol=1e-12)
            assert np.allclose(lse[part], s.logsumexp(-1).reshape(n, heads * group).numpy(), atol=1e-12)
            assert (spread[part] >= np.abs(out[part]) - 1e-12).all()


def test_attend_rows_that_see_nothing_are_zero():
    k, v, ks, vs = cache(1, 1, 16, 64)
    out, lse, _ = O.attend(k, v, ks, vs, 16, 1, np.zeros((1, 1), np.int32), np.array([0, 3]), np.array([1]), np.ones((3, 1, 64)), 1.0, True, 0)
    assert (out == 0).all() and lse[:2].tolist() == [[-np.inf], [-np.inf]] and lse[2, 0] == 0
