"""Attention over the paged cache where scores and queries are far beyond the usual: finite inputs give finite results, and those are what the formula gives
as far as float32 scores can tell.

A score passes about 16 roundings of 2^-24 of S = sum |q| (15 scale + |minimum|) / sqrt(d) (as in the oracle), so two scores further apart than 32 2^-24 S + 20 leave the
smaller one a weight below e^-20 = 2^-28: with all others that far below, the result is the value of the largest score, rounded once."""
import numpy as np
import pytest

from oracle import kvpr_paged_oracle as po
from paged_testlib import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def k():
    import paper_2411_17089_amd as k
    return k


def _rows(b, q):
    """(row, head, scores, values, S) of every row that sees something"""
    group = b.heads // b.kv_heads
    for r, (L, m) in enumerate(zip(b.lens, b.new)):
        cache = [po.load(b.pages, b.table[r, t // b.page] * b.page + t % b.page, b.kv_heads, b.d, b.page) for t in range(L)]
        for g in range(b.kv_heads):
            keys = np.stack([po.values(*(a[g] for a in c[0])) for c in cache])
            v = np.stack([po.values(*(a[g] for a in c[1])) for c in cache]).astype(np.float16).astype(np.float64)
            size = np.stack([np.repeat(15 * c[0][1][g].astype(np.float64) + np.abs(c[0][2][g].astype(np.float64)), 64) for c in cache])
            for i in range(m):
                row, n = int(b.row_start[r]) + i, L - m + i + 1
                for h in range(g * group, (g + 1) * group):
                    x = q[row, h * b.d:(h + 1) * b.d].astype(np.float64) / np.sqrt(b.d)
                    yield row, h, keys[:n] @ x, v[:n], (size[:n] @ np.abs(x)).max()


def _check(b, q, z):
    assert np.isfinite(z).all()
    decided = 0
    for row, h, s, v, big in _rows(b, q):
        got = z[row, h * b.d:(h + 1) * b.d]
        at = int(np.argmax(s))
        assert (got >= v.min(0) - 2.0 ** -10 * np.abs(v).max(0)).all() and (got <= v.max(0) + 2.0 ** -10 * np.abs(v).max(0)).all()
        others = np.delete(s, at)
        if others.size == 0 or s[at] - others.max() > 32 * 2.0 ** -24 * big + 20:
            decided += 1
            # the rest's weights are below len 2^-28 together
            assert (np.abs(got - v[at]) <= 2.0 ** -11 * np.abs(v[at]) + (2.0 ** -22 + len(s) * 2.0 ** -28) * np.abs(v).max() + 2.0 ** -25).all(), (row, h)
    return decided


@pytest.mark.parametrize("power", [10, 16, 20, 22, 24, 26, 28, 30, 40, 60, 84, 86, 100, 106, 112, 118, 124])
@pytest.mark.parametrize("heads,kv_heads,d,lens,new", [(4, 2, 128, [200, 33], [2, 1]), (24, 1, 64, [90, 40], [2, 1]), (16, 1, 64, [150], [9])])
def test_large_queries(k, power, heads, kv_heads, d, lens, new):
    b = Batch(lens, new, heads, kv_heads, d, 16, seed=power)
    q = (b.q("f32", scale=1.0) * 2.0 ** power).astype(np.float32)
    assert np.isfinite(q).all()
    for max_len in (None, 100000):                                      # a workgroup for each unit, and runs
        decided = _check(b, q, b.attention(k, q, max_len=max_len))
        assert power < 16 or decided > 0.9 * b.rows * heads


@pytest.mark.parametrize("q_type", ["f16", "f32"])
def test_large_float16_queries_and_keys(k, q_type):
    b = Batch([180, 21], [3, 1], 4, 2, 128, 16, seed=5, spread=1.0)
    block = b.pages.reshape(b.n_pages, b.kv_heads, -1)
    at = slice(b.page * b.d, b.page * b.d + b.page * 8)
    pairs = block[..., at].copy().view(np.float16)
    block[..., at] = (pairs.astype(np.float32) * 8000).astype(np.float16).view(np.uint8)
    q = (b.q("f16", scale=1.0).astype(np.float32) * 14000).clip(-65504, 65504).astype(np.float16)
    q = q.astype(np.float32) if q_type == "f32" else q
    for max_len in (None, 100000):
        assert _check(b, q, b.attention(k, q, max_len=max_len)) > 0.9 * b.rows * b.heads


@pytest.mark.parametrize("power", [0, 12, 20, 24, 25, 26, 27, 28, 29, 30, 33, 50, 110, 126])
@pytest.mark.parametrize("sign", [1, -1])
def test_equal_keys_give_the_mean(k, power, sign):
    """Equal scores, however large, have equal weights: the result is the mean of the values, each weight rounded as usual."""
    b = Batch([700, 130, 64], [3, 2, 20], 4, 2, 128, 32, seed=6)
    block = b.pages.reshape(b.n_pages, b.kv_heads, -1)
    codes, pairs = slice(0, b.page * b.d // 2), slice(b.page * b.d, b.page * b.d + b.page * 8)
    block[..., codes] = np.tile(block[:1, :1, :b.d // 2], (b.n_pages, b.kv_heads, b.page))
    block[..., pairs] = np.tile(block[:1, :1, pairs][..., :8], (b.n_pages, b.kv_heads, b.page))
    q = np.full((b.rows, b.heads * b.d), sign * 2.0 ** power, np.float32)
    q[:, ::3] *= 0.7
    want = {(row, h): (v.mean(0), np.abs(v).mean(0)) for row, h, _, v, _ in _rows(b, q)}
    for max_len in (None, 100000):
        z = b.attention(k, q, max_len=max_len)
        for (row, h), (mean, size) in want.items():
            # the weights' second float16 number leaves 2^-22 of each, sums in float32 16 roundings, the result half a step of float16
            assert (np.abs(z[row, h * b.d:(h + 1) * b.d] - mean) <= 2.0 ** -11 * np.abs(mean) + 2.0 ** -19 * size + 2.0 ** -25).all(), (row, h)
