"""Pins of the oracle of attention over keys of their own: torch's attention in 64 bits, the append's bounds, the pool's invariants."""
import numpy as np
import torch

from oracle import keys as K
from oracle.layer import e4m3_values


def test_attention_is_torchs():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((5, 16)), rng.standard_normal((9, 16)), rng.standard_normal((9, 16))
    there = rng.random((5, 9)) < 0.6
    there[2], there[3, 1] = False, True
    o, lse, size, _ = K.attention(q, k, v, there, 0.3)
    x = torch.from_numpy(q) @ torch.from_numpy(k).T * 0.3
    x[~torch.from_numpy(there)] = -torch.inf
    want = torch.softmax(x, -1) @ torch.from_numpy(v)
    want[2] = 0
    np.testing.assert_allclose(o, want, rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(lse, torch.logsumexp(x, -1), rtol=1e-12)
    assert (size >= np.abs(o) - 1e-12).all() and lse[2] == -np.inf


def test_append_in_pieces_stays_within_its_steps():
    """Values survive with the error of one rounding under the page's final scale, and one more for each time that their page got a larger one."""
    rng = np.random.default_rng(1)
    page, T = 16, 61
    x = rng.standard_normal((1, 2, T, 8)) * np.exp(rng.standard_normal((1, 1, T, 1)))
    codes, scale = np.zeros((5, 2, page, 8), np.uint8), np.full((5, 2), 7.0)
    table, at, grown = [[3, 0, 4, 1]], 0, np.zeros((4, 2))
    while at < T:
        n = min(int(rng.integers(1, 9)), T - at)
        before = scale.copy()
        K.append(codes, scale, x[:, :, at:at + n], table, [at], [n], page)
        for place in range(at // page, (at + n - 1) // page + 1):
            grown[place] += (scale[table[0][place]] > before[table[0][place]]) & (place * page < at)
        at += n
    got = K.gathered(codes, scale, table[0], T, page)
    s = np.repeat(scale[table[0]].T, page, 1)[:, :T, None]
    steps = 1 + np.repeat(grown.T, page, 1)[:, :T, None]
    assert (np.abs(got - x[0]) <= steps * np.maximum(np.abs(x[0]) * 2.0 ** -4 * 1.07, s * 2.0 ** -10)).all()
    assert np.array_equal(scale[2], [7.0, 7.0]) and (np.abs(e4m3_values(codes)) <= 448).all()


def test_the_pool_keeps_its_books():
    rng = np.random.default_rng(2)
    pool = K.Pool([0] * 40, [[-1] * 6 for _ in range(5)], [0] * 5, 4)
    for _ in range(60):
        what, r = rng.integers(4), [int(i) for i in rng.permutation(5)[:2]]
        if what == 0:
            counts = [int(rng.integers(0, 24 - n + 1)) for n in pool.lengths]
            pool.take(counts)
            pool.lengths = [a + b for a, b in zip(pool.lengths, counts)]
        elif what == 1:
            pool.free([r[1]], [0])
            pool.fork([r[0]], [r[1]])
        elif what == 2:
            pool.free([r[0]], [int(rng.integers(0, 24))])
        else:
            assert pool.compact() == sum(n > 0 for n in pool.refs) and all(n > 0 for n in pool.refs[:pool.compact()])
        named = np.bincount([i for row in pool.table for i in row if i >= 0], minlength=40)
        assert np.array_equal(named, pool.refs) and not pool.short
        assert [sum(i >= 0 for i in row) for row in pool.table] == [-(-n // 4) for n in pool.lengths]
