"""Every attention kernel at least once - head width, type of q, tiles of rows, rows of a wave's own, units or runs - and batches of prompt chunks beside single
rows, against float64; and a bound that one float16 number a weight does not keep."""
import numpy as np
import pytest

from oracle import kvpr_paged_oracle as po
from paged_testlib import Batch

gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def k():
    import paper_2411_17089_amd as k
    return k


def _cache(b, r):
    """k, v [kv_heads, len, d] and 15 scale + |minimum| of k, float64, v rounded to float16, of request r; all of its pages there."""
    n, d, page, length = b.kv_heads, b.d, b.page, b.lens[r]
    block = b.pages[b.table[r, :-(-length // page)]].reshape(-1, n, page * 9 * d // 8)
    out = []
    for is_key in (True, False):
        at = np.array([po._addresses(0, t, d, page, is_key)[0] for t in range(page)])
        pair = np.array([po._addresses(0, t, d, page, is_key)[1] for t in range(page)])[:, None] + np.arange(d // 64 * 4)
        b8 = block[:, :, at]
        codes = np.stack([b8 & 15, b8 >> 4], -1).reshape(*b8.shape[:3], d)
        pairs = np.ascontiguousarray(block[:, :, pair]).view(np.float16).reshape(*b8.shape[:3], d // 64, 2)
        by_head = lambda a: a.transpose(1, 0, 2, 3).reshape(n, -1, a.shape[-1])[:, :length]           # noqa: E731
        out.append((by_head(codes), by_head(pairs[..., 0]), by_head(pairs[..., 1])))
    size = np.repeat(15 * out[0][1].astype(np.float64) + np.abs(out[0][2].astype(np.float64)), 64, -1)
    return po.values(*out[0]), po.values(*out[1]).astype(np.float16).astype(np.float64), size


def _exact(b, q, weight_bits=None):
    """(z, bound): float64, and what the kernel's own roundings leave: half a step of float16 of the result (2^-11), weights as two float16 numbers (2^-22 of each) in
    sums of float32 (16 roundings of 2^-24), scores of 16 roundings of 2^-24 of sum |q| (15 scale + |minimum|).  weight_bits: weights rounded to so many bits."""
    q = q.astype(np.float64)
    z, tol = np.zeros(q.shape), np.zeros(q.shape)
    group, d = b.heads // b.kv_heads, b.d
    for r, (length, m) in enumerate(zip(b.lens, b.new)):
        if m == 0:
            continue
        keys, v, size = _cache(b, r)
        rows = slice(int(b.row_start[r]), int(b.row_start[r]) + m)
        hidden = np.arange(length)[None] > np.arange(length - m, length)[:, None]
        for h in range(b.heads):
            x = q[rows, h * d:(h + 1) * d] / np.sqrt(d)
            s = np.where(hidden, -np.inf, x @ keys[h // group].T)
            e = np.exp(s - s.max(1, keepdims=True))
            total = e.sum(1, keepdims=True)
            if weight_bits:
                f, ex = np.frexp(e)
                e = np.ldexp(np.round(f * 2.0 ** weight_bits), ex - weight_bits)
            p = e / total
            noise = 16 * 2.0 ** -24 * ((np.abs(x) @ size[h // group].T).max(1, keepdims=True) + 1)
            z[rows, h * d:(h + 1) * d] = p @ v[h // group]
            spread = p @ np.abs(v[h // group])
            tol[rows, h * d:(h + 1) * d] = 2.0 ** -11 * np.abs(p @ v[h // group]) + (2 * noise + 2.0 ** -20) * spread + 2.0 ** -25
    return z, tol


def _check(b, q, got):
    want, tol = _exact(b, q)
    off = np.abs(got - want) / tol
    assert (off <= 1).all(), (np.argwhere(~(off <= 1))[:3], np.nanmax(off))


def test_the_same_as_the_oracle():
    b = Batch([70, 3, 33], [4, 3, 1], 6, 2, 64, 32, seed=1)
    q = b.q("f32")
    want, tol, done = po.attention(q, b.pages, b.table, b.row_start, b.lens, 6, 2, 64, 32, q.shape[0])
    got, bound = _exact(b, q)
    assert done.all() and np.allclose(got, want, rtol=0, atol=1e-12) and (bound <= tol).all()


def test_the_bound_tells_one_float16_number_a_weight_from_two():
    """On the CPU: weights of 11 bits pass it, those of 22 do not."""
    b = Batch([9, 12, 40, 300], [1, 2, 3, 1], 4, 2, 128, 16, seed=2)
    q = b.q("f16", scale=0.3)
    want, tol = _exact(b, q)
    one, two = (np.abs(_exact(b, q, bits)[0] - want) > tol - 2.0 ** -11 * np.abs(want) for bits in (11, 22))
    assert one.mean() > 0.2 and not two.any()
    assert (np.abs(_exact(b, q, 11)[0].astype(np.float16).astype(np.float64) - want) > tol).any()


# heads, kv_heads, new tokens, requests, what the launch is then: tiles of 16 rows a wave, rows of its own
SHAPES = [(32, 32, 1, 12, "one tile"), (32, 8, 4, 48, "one tile"), (32, 8, 5, 40, "two tiles"), (16, 8, 31, 34, "two tiles"), (24, 24, 70, 12, "many rows"), (64, 8, 40, 14, "many rows")]


@gpu
@pytest.mark.parametrize("heads,kv_heads,m,n,kind", SHAPES, ids=[f"{s[0]}x{s[1]}x{s[2]}-{s[4].replace(' ', '_')}" for s in SHAPES])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q_type", ["f16", "f32"])
def test_kernels_by_units(k, heads, kv_heads, m, n, kind, d, q_type):
    rows = m * heads // kv_heads
    assert (rows <= 16) == (kind == "one tile") and (rows > 64) == (kind == "many rows")
    units = kv_heads * -(-rows // (16 if rows <= 16 else 32 if rows <= 64 else 128)) * n
    assert units >= 256 * (3 if rows <= 16 else 2) // 2
    rng = np.random.default_rng(heads + m)
    lens = rng.integers(m, 420, n)
    b = Batch(lens, [m] * n, heads, kv_heads, d, 32, seed=m)
    q = b.q(q_type)
    _check(b, q, b.attention(k, q, max_len=2000))


@gpu
@pytest.mark.parametrize("heads,kv_heads,m,n", [(8, 8, 1, 3), (8, 2, 4, 3), (8, 2, 5, 2), (8, 8, 40, 2), (4, 2, 70, 3), (16, 1, 9, 2)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q_type", ["f16", "f32"])
def test_kernels_by_runs(k, heads, kv_heads, m, n, d, q_type):
    rng = np.random.default_rng(heads + m)
    lens = rng.integers(m, 1500, n)
    lens[0] = 1700
    b = Batch(lens, [m] * n, heads, kv_heads, d, 16, seed=m)
    q = b.q(q_type)
    _check(b, q, b.attention(k, q))


@gpu
@pytest.mark.parametrize("chunk,others", [(200, 9), (700, 30), (65, 3)])
@pytest.mark.parametrize("q_type", ["f16", "f32"])
def test_prompt_chunk_beside_single_rows(k, chunk, others, q_type):
    """One request with a chunk, the others with a row or a few over long caches, the chunk's own rows from its first position on."""
    rng = np.random.default_rng(chunk)
    new = [chunk] + [int(m) for m in rng.integers(1, 5, others)]
    lens = [chunk + 100] + [int(x) for x in rng.integers(200, 2500, others)]
    lens[-1] = new[-1]                                                  # and one that has only its new rows
    order = rng.permutation(others + 1)
    b = Batch([lens[i] for i in order], [new[i] for i in order], 32, 8, 128, 64, seed=chunk)
    q = b.q(q_type)
    for max_new, max_len in ((chunk, max(lens)), (chunk, 1 << 20), (1, 1 << 20)):
        _check(b, q, b.attention(k, q, max_new=max_new, max_len=max_len))


@gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q_type", ["f16", "f32"])
def test_weights_are_two_float16_numbers(k, d, q_type):
    """Few positions of nearly equal weights and values that cancel: an error of 2^-12 of each weight would pass the bound in many columns."""
    b = Batch([2, 3, 5, 9, 12, 40, 300], [1, 1, 2, 3, 2, 3, 1], 8, 2, d, 16, seed=2)
    q = b.q(q_type, scale=0.3)
    for max_len in (None, 100000):
        _check(b, q, b.attention(k, q, max_len=max_len))
