"""Attention of ragged batches over a paged 4-bit cache against the oracle.  Tolerances come with the oracle's values:
half a step of float16 of the weights and of the result, and float32 sums."""
import numpy as np
import pytest
import torch

from oracle import kvpr_paged_oracle as po
from paged_testlib import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def k():
    import paper_2411_17089_amd as k
    return k


def _check(got, want, tol, done, fill=7.0):
    bad = ~(np.abs(got - want) <= tol)                                  # NaN is bad
    bad[~done] = False
    assert not bad.any(), (np.argwhere(bad)[:3], np.max((np.abs(got - want) / tol)[done]))
    assert (got[~done] == fill).all()


HEADS = [(1, 1, 64), (2, 2, 128), (8, 2, 128), (5, 1, 64), (16, 1, 128), (40, 8, 128), (24, 1, 64), (33, 1, 128)]


@pytest.mark.parametrize("heads,kv_heads,d", HEADS)
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("q_type", ["f16", "f32"])
def test_ragged(k, heads, kv_heads, d, page, q_type):
    lens, new = [1, 17, 40, 130, 64, 333, 2, 8], [1, 1, 3, 2, 5, 1, 2, 8]
    b = Batch(lens, new, heads, kv_heads, d, page, seed=heads * 100 + page)
    q = b.q(q_type)
    print("ragged", heads, kv_heads, d, page, q_type, flush=True)
    _check(b.attention(k, q), *b.oracle(q))


@pytest.mark.parametrize("L", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1023, 1025])
def test_lengths(k, L):
    b = Batch([L], [1], 4, 2, 128, 16, seed=L)
    q = b.q("f16")
    _check(b.attention(k, q), *b.oracle(q))


@pytest.mark.parametrize("m", [1, 2, 3, 7, 8, 9, 16, 17, 31, 33, 64, 65, 100, 150])
@pytest.mark.parametrize("heads,kv_heads,d,page", [(2, 1, 64, 32), (3, 3, 128, 128)])
def test_new_tokens(k, m, heads, kv_heads, d, page):
    b = Batch([m, m + 37], [m, m], heads, kv_heads, d, page, seed=m)
    q = b.q("f32")
    _check(b.attention(k, q), *b.oracle(q))


def test_long_one_request(k):
    b = Batch([9000], [2], 4, 1, 128, 32, seed=3)
    q = b.q("f16")
    _check(b.attention(k, q), *b.oracle(q))


def test_rows_that_see_nothing_idle_and_refused_requests(k):
    # refused: length 0 with rows; idle: no rows; fewer positions than rows: the first rows see nothing
    b = Batch([0, 20, 3, 50], [2, 0, 5, 1], 6, 3, 128, 16, seed=1)
    q = b.q("f16")
    z = b.attention(k, q)
    _check(z, *b.oracle(q))
    assert (z[:4] == 0).all() and (z[4] != 0).any()


def test_entries_outside_the_pool_take_no_part(k):
    for bad in (-1, -2 ** 31, 10 ** 6, 2 ** 31 - 1):
        b = Batch([100, 40, 16], [2, 1, 1], 4, 2, 128, 16, seed=2)
        b.table[0, 1] = bad
        b.table[0, 6] = bad                                             # the page of the new tokens
        b.table[2, 0] = b.n_pages                                       # the only page: nothing is left
        q = b.q("f32")
        z = b.attention(k, q)
        _check(z, *b.oracle(q))
        assert (z[3] == 0).all()


def test_lengths_beyond_the_table(k):
    b = Batch([64, 30], [2, 1], 2, 1, 64, 16, seed=4, extra_width=0)
    b.lens[0] = 90                                                      # 26 positions have no table entry
    q = b.q("f16")
    _check(b.attention(k, q), *b.oracle(q))


def test_rows_behind_the_last_and_fewer_rows_than_tokens(k):
    b = Batch([40, 70, 33], [3, 4, 2], 4, 2, 64, 16, seed=5)
    q = b.q("f16", rows=12)
    _check(b.attention(k, q), *b.oracle(q))                             # rows 9 .. 11 belong to nobody
    z, want, tol, done = b.attention(k, q, rows=5), *b.oracle(q, rows=5)
    full = np.zeros(12, bool)
    full[:5] = done
    _check(z[:5], want, tol, full[:5])
    assert (z[5:] == 7.0).all()


@pytest.mark.parametrize("max_new,max_len", [(1, 1), (2, 100), (64, 100000), (1000, 16)])
def test_host_bounds_only_size_the_launch(k, max_new, max_len):
    b = Batch([700, 5, 333, 90], [40, 1, 3, 90], 4, 2, 128, 32, seed=6)
    q = b.q("f16")
    _check(b.attention(k, q, max_new=max_new, max_len=max_len), *b.oracle(q))


def test_strides(k):
    b = Batch([100, 37], [2, 3], 4, 4, 64, 16, seed=7)
    for q_type in ("f16", "f32"):
        q = b.q(q_type)
        _check(b.attention(k, q, ldq=3 * 256 + 8, ldz=256 + 40), *b.oracle(q))


@pytest.mark.parametrize("garbage", ["nan", "inf", "huge"])
def test_positions_that_no_row_sees_hold_anything(k, garbage):
    """What lies behind the last position of a page, and later tokens' rows, may hold NaN or infinite pairs."""
    b = Batch([21, 70], [1, 3], 4, 2, 128, 32, seed=8)
    q = b.q("f16")
    want = b.oracle(q)
    value = {"nan": np.nan, "inf": np.inf, "huge": 60000.0}[garbage]
    for r, L in enumerate(b.lens):
        for t in range(L, -(-L // b.page) * b.page):
            for h in range(b.kv_heads):
                for is_key in (True, False):
                    _, pair = po._addresses(h, t % b.page, b.d, b.page, is_key)
                    b.pages[b.table[r, t // b.page]][pair:pair + 8] = np.full(4, value, np.float16).view(np.uint8)
    _check(b.attention(k, q), *want)
    # the last new token of request 1: rows 1 and 2 do not see it, row 3 does
    for h in range(b.kv_heads):
        _, pair = po._addresses(h, 69 % b.page, b.d, b.page, False)
        b.pages[b.table[1, 69 // b.page]][pair:pair + 8] = np.full(4, value, np.float16).view(np.uint8)
    z = b.attention(k, q)
    done = want[2].copy()
    done[3] = False
    bad = ~(np.abs(z - want[0])[done] <= want[1][done])
    assert not bad.any()
    if garbage != "huge":
        assert not np.isfinite(z[3]).all()


@pytest.mark.parametrize("spread", [1e-3, 30.0, 3000.0])
def test_ranges_of_values(k, spread):
    """Values from 10^-3 to 10^4: weights times scales must neither run out of float16 nor below it."""
    b = Batch([300, 33], [1, 2], 4, 2, 128, 16, seed=9, spread=1.0)
    block = b.pages.reshape(b.n_pages, b.kv_heads, -1)
    pairs = block[..., b.page * b.d + b.page * 8:].copy().view(np.float16)
    block[..., b.page * b.d + b.page * 8:] = (pairs.astype(np.float32) * spread).astype(np.float16).view(np.uint8)
    q = b.q("f16")
    _check(b.attention(k, q), *b.oracle(q))


def test_scales_that_differ_from_position_to_position(k):
    """Each position's values a power of two of its own, 2^-12 to 2^12, constant groups among them, and large scores."""
    b = Batch([200], [2], 2, 1, 128, 16, seed=10)
    block = b.pages.reshape(b.n_pages, 1, b.page * 144)
    pairs = block[..., b.page * b.d + b.page * 8:].copy().view(np.float16).reshape(b.n_pages, b.page, 2, 2)
    pairs *= (2.0 ** b.rng.integers(-12, 13, pairs.shape[:-1]))[..., None].astype(np.float16)
    pairs[b.rng.random(pairs.shape[:-1]) < 0.1, 0] = 0
    block[..., b.page * b.d + b.page * 8:] = pairs.reshape(b.n_pages, 1, -1).view(np.uint8)
    for scale in (0.1, 8.0):
        q = b.q("f32", scale=scale)
        _check(b.attention(k, q), *b.oracle(q))


@pytest.mark.parametrize("scale", [1e-6, 1e-3, 200.0])
def test_ranges_of_queries(k, scale):
    b = Batch([90, 40], [2, 1], 4, 2, 64, 16, seed=11)
    q = b.q("f32", scale=scale)
    _check(b.attention(k, q), *b.oracle(q))
    q[0] = 0
    _check(b.attention(k, q), *b.oracle(q))


def test_nan_of_one_row_stays_there(k):
    b = Batch([90, 40], [3, 1], 4, 2, 64, 16, seed=12)
    q = b.q("f16")
    q[1, 70] = np.nan                                                   # head 1 of row 1
    clean = q.copy()
    clean[1] = 0
    z, (want, tol, done) = b.attention(k, q), b.oracle(clean)
    done[1] = False
    assert (np.abs(z - want)[done] <= tol[done]).all()
    assert np.isnan(z[1, 64:128]).all() and np.isfinite(z[1, :64]).all() and np.isfinite(z[1, 128:]).all()


def test_another_stream_and_twice_the_same(k):
    b = Batch([1500, 700, 33], [2, 1, 5], 8, 2, 128, 16, seed=13)
    q = b.q("f16")
    want = b.attention(k, q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        assert np.array_equal(b.attention(k, q, stream=side), want)
    assert np.array_equal(b.attention(k, q), want)


def test_pool_beyond_4_gib(k):
    heads, kv_heads, d, page = 64, 64, 128, 256
    desc_bytes = po.page_bytes(kv_heads, d, page)
    n_pages = (1 << 32) // desc_bytes + 2
    small = Batch([300], [1], heads, kv_heads, d, page, seed=14, spare=0)
    pages = torch.zeros((n_pages, desc_bytes), dtype=torch.uint8, device="cuda")
    at = [n_pages - 1, n_pages - 2]
    pages[at] = torch.from_numpy(small.pages[small.table[0, :2]]).cuda()
    q = small.q("f16")
    table = torch.tensor([at], dtype=torch.int32, device="cuda")
    z = torch.zeros((1, heads * d), dtype=torch.float16, device="cuda")
    desc = k.make_paged_desc(heads, kv_heads, d, page, n_pages, 2)
    ws = torch.zeros(k.kvpr_paged_attention_workspace_bytes(desc, 1, 1, 1, 300), dtype=torch.uint8, device="cuda")
    one = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")                  # noqa: E731
    k.kvpr_paged_attention(desc, torch.from_numpy(q).cuda(), k.KVPR_F16, heads * d, pages, table, one(0, 1), one(300), 1, 1, 1, 300, z, heads * d, ws, ws.numel())
    torch.cuda.synchronize()
    assert np.array_equal(z.double().cpu().numpy(), small.attention(k, q))


def test_many_requests(k):
    """More requests than a workgroup has threads, most of them short: equal runs of the work, with many units each."""
    rng = np.random.default_rng(15)
    lens = rng.integers(1, 40, 700)
    lens[[5, 300, 699]] = 900, 450, 130
    new = np.minimum(rng.integers(0, 3, 700), lens)
    b = Batch(lens, new, 2, 1, 64, 16, seed=15)
    q = b.q("f16")
    want = b.oracle(q)
    for max_len in (900, 100000):
        _check(b.attention(k, q, max_len=max_len), *want)


@pytest.mark.parametrize("heads,kv_heads,d,m", [(8, 8, 128, 1), (32, 8, 64, 7), (8, 8, 64, 3)])
@pytest.mark.parametrize("q_type", ["f16", "f32"])
def test_a_unit_for_each_workgroup(k, heads, kv_heads, d, m, q_type):
    """Batches that fill the GPU with whole units (of several turns), and the same by runs, as a looser bound of the lengths gives."""
    rng = np.random.default_rng(16)
    lens = rng.integers(m, 300, 50)
    b = Batch(lens, [m] * 50, heads, kv_heads, d, 16, seed=16)
    q = b.q(q_type)
    want = b.oracle(q)
    _check(b.attention(k, q, max_len=300), *want)
    _check(b.attention(k, q, max_len=100000), *want)


@pytest.mark.parametrize("q_type", ["f16", "f32"])
def test_many_rows_and_units(k, q_type):
    """Rows of their own for each wave, a unit for each workgroup, against the launch that is made for few rows."""
    b = Batch([500, 150, 333], [150, 150, 90], 64, 64, 64, 32, seed=17)
    q = b.q(q_type)
    z = b.attention(k, q)
    few = b.attention(k, q, max_new=1, max_len=100000)
    tol = 2.0 ** -10 * (np.abs(few) + 4.2)                              # twice the bound of either; no value is larger than 15 0.4 - 1.8
    assert (np.abs(z - few) <= tol).all()
    rows, heads = [0, 149, 150, 299, 300, 389], [0, 63]
    sub = Batch([500, 150, 333], [150, 150, 90], 64, 64, 64, 32, seed=17)
    for h in heads:
        block = sub.page * 9 * sub.d // 8
        one = sub.pages.reshape(sub.n_pages, 64, block)[:, h]
        want, t, _ = po.attention(q[:, h * 64:(h + 1) * 64], one, sub.table, sub.row_start, sub.lens, 1, 1, 64, 32, q.shape[0])
        got = z[:, h * 64:(h + 1) * 64]
        assert (np.abs(got - want)[rows] <= t[rows]).all()
