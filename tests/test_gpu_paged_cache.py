"""Append and read-back of paged rows against the oracle, byte for byte."""
import numpy as np
import pytest
import torch

from oracle import kvpr_int4_oracle as io
from oracle import kvpr_paged_oracle as po
from paged_testlib import i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def k():
    import paper_2411_17089_amd as k
    return k


def _append(k, x, slots, positions, heads, kv_heads, d, page, n_pages, rope=None, q_out=True, ld=None, in_place=False):
    """-> (pages, q_out or None) after one append into pages of 0xA5"""
    rows, cols = x.shape
    ld = ld or cols
    buf = torch.full((rows + 1, ld), 3.0, dtype=torch.float16, device="cuda")
    buf[:rows, :cols] = torch.from_numpy(x).cuda()
    pages = torch.full((n_pages, po.page_bytes(kv_heads, d, page)), 0xA5, dtype=torch.uint8, device="cuda")
    desc = k.make_paged_desc(heads, kv_heads, d, page, n_pages, 1)
    assert k.kvpr_page_bytes(desc) == pages.shape[1]
    q = None
    if rope is not None and q_out:
        q = buf if in_place else torch.full((rows + 1, heads * d + 8), 3.0, dtype=torch.float16, device="cuda")
    k.kvpr_paged_append(desc, buf, ld, i32(slots), i32(positions) if positions is not None else None, rows,
                        None if rope is None else torch.from_numpy(rope).cuda(), 0 if rope is None else rope.shape[0], q, 0 if q is None else q.shape[1], pages)
    torch.cuda.synchronize()
    if q is not None and not in_place:
        assert (q[rows:] == 3.0).all() and (q[:, heads * d:] == 3.0).all()
    if not in_place:
        assert torch.equal(buf[:rows, :cols].cpu().view(torch.int16), torch.from_numpy(x).view(torch.int16))
    return pages.cpu().numpy(), None if q is None else q[:rows, :heads * d].cpu().numpy()


def _want(x, slots, positions, heads, kv_heads, d, page, n_pages, rope):
    rows = x.shape[0]
    h = x.reshape(rows, -1, d)
    q, kk, v = h[:, :heads], h[:, heads:heads + kv_heads], h[:, heads + kv_heads:]
    ok = np.ones(rows, bool)
    if rope is not None:
        ok = (np.asarray(positions) >= 0) & (np.asarray(positions) < len(rope))
        at = np.where(ok, positions, 0)
        q, kk = (po.rotate(a, rope, at).astype(np.float16) for a in (q, kk))
    pages = np.full((n_pages, po.page_bytes(kv_heads, d, page)), 0xA5, np.uint8)
    for i, slot in enumerate(slots):
        if ok[i] and 0 <= slot < n_pages * page:
            po.store(pages, slot, kk[i], v[i], page)
    return pages, q.reshape(rows, -1), ok


CASES = [(12, 12, 64, 16, 1), (4, 4, 128, 32, 33), (8, 2, 128, 16, 50), (5, 1, 64, 256, 7), (6, 3, 128, 64, 129), (14, 2, 64, 128, 90), (3, 3, 128, 16, 16)]


@pytest.mark.parametrize("heads,kv_heads,d,page,rows", CASES)
@pytest.mark.parametrize("rope", [False, True])
def test_append(k, heads, kv_heads, d, page, rows, rope):
    rng = np.random.default_rng(rows)
    n_pages = rows // page + 3
    x = rng.standard_normal((rows, (heads + 2 * kv_heads) * d)).astype(np.float16)
    slots = rng.permutation(n_pages * page)[:rows]
    if rows > 20:                                                       # runs of consecutive positions, as a prompt has them, among single ones
        slots = np.concatenate([np.arange(page + 3, page + 3 + 13), np.setdiff1d(slots, np.arange(page + 3, page + 16))])[:rows]
        rows = len(slots)
        x = x[:rows]
    table = k.kvpr_rope_table(700, d) if rope else None
    positions = rng.integers(0, 700, rows) if rope else None
    for ld, in_place in ((None, False), (x.shape[1] + 24, False), (None, True)):
        got, q = _append(k, x, slots, positions, heads, kv_heads, d, page, n_pages, table, ld=ld, in_place=in_place)
        want, wq, _ = _want(x, slots, positions, heads, kv_heads, d, page, n_pages, table)
        assert np.array_equal(got, want)
        if rope:
            assert np.array_equal(q.view(np.uint16), wq.view(np.uint16))


def test_slots_and_positions_outside(k):
    rng = np.random.default_rng(5)
    heads, kv_heads, d, page, n_pages = 4, 2, 128, 16, 2
    slots = [-1, 3, 32, 31, 0, 2 ** 31 - 1, -2 ** 31, 17]
    positions = [0, 9, 1, 10, -1, 0, 2, 5]                              # 10 and -1 lie outside the table
    x = rng.standard_normal((8, 8 * d)).astype(np.float16)
    table = k.kvpr_rope_table(10, d)
    got, q = _append(k, x, slots, positions, heads, kv_heads, d, page, n_pages, table)
    want, wq, ok = _want(x, slots, positions, heads, kv_heads, d, page, n_pages, table)
    assert np.array_equal(got, want)
    assert np.array_equal(q[ok].view(np.uint16), wq[ok].view(np.uint16)) and (q[~ok] == 3.0).all()
    got, q = _append(k, x, slots, positions, heads, kv_heads, d, page, n_pages, table, q_out=False)
    assert q is None and np.array_equal(got, want)
    got, _ = _append(k, x, slots, None, heads, kv_heads, d, page, n_pages, None)
    assert np.array_equal(got, _want(x, slots, None, heads, kv_heads, d, page, n_pages, None)[0])


@pytest.mark.parametrize("d", [64, 128])
def test_special_values(k, d):
    """Constant groups, zeros, the largest and the smallest numbers, infinities and NaN: the codec's own bytes; no other row is touched."""
    page, n_pages = 16, 1
    x = np.random.default_rng(1).standard_normal((12, 3 * d)).astype(np.float16)
    x[0], x[1], x[2] = 0, 1.5, -0.0
    x[3, :] = 65504
    x[3, ::2] = -65504
    x[4] = np.float16(6e-8) * np.arange(3 * d) % 5
    x[5, 7], x[6, d + 3], x[7, 2 * d + 5], x[8, 2 * d + 1] = np.inf, np.inf, -np.inf, np.inf
    x[9, d + 1], x[10, 2 * d:] = np.nan, np.nan
    got, _ = _append(k, x, np.arange(12), None, 1, 1, d, page, n_pages)
    with np.errstate(all="ignore"):
        want, _, _ = _want(x, np.arange(12), None, 1, 1, d, page, n_pages, None)
    finite = [0, 1, 2, 3, 4, 5, 11]
    for t in finite:
        for a, b in zip(po.load(got, t, 1, d, page), po.load(want, t, 1, d, page)):
            assert all(np.array_equal(u, w) for u, w in zip(a, b)), t
    # a group with an infinity or a NaN: no finite value comes back from it, and the groups beside it are untouched
    back = lambda pages, t: [po.values(*a)[0].reshape(-1, 64) for a in po.load(pages, t, 1, d, page)]   # noqa: E731
    with np.errstate(all="ignore"):
        for t, side, group in ((6, 0, 0), (7, 1, 0), (8, 1, 0)):
            assert not np.isfinite(back(got, t)[side][group]).any()
    assert np.array_equal(got[:, 0] * 0, got[:, 0] * 0)
    for t in (6, 7, 8, 9, 10):
        for side in (0, 1):
            g, w = po.load(got, t, 1, d, page)[side], po.load(want, t, 1, d, page)[side]
            for group in range(d // 64):
                if np.isfinite(x[t, (side + 1) * d + 64 * group:(side + 1) * d + 64 * group + 64]).all():
                    assert np.array_equal(g[0][0, 64 * group:64 * group + 64], w[0][0, 64 * group:64 * group + 64]) and g[1][0, group] == w[1][0, group]
    for t in range(12, 16):
        codes, pair = po._addresses(0, t, d, page, True)
        assert (got[0][codes] == 0xA5).all() and (got[0][pair:pair + 4] == 0xA5).all()


@pytest.mark.parametrize("heads,kv_heads,d,page,rows", CASES)
def test_read(k, heads, kv_heads, d, page, rows):
    rng = np.random.default_rng(rows + 1)
    n_pages, cols = rows // page + 3, 2 * kv_heads * d
    kv = rng.standard_normal((n_pages * page, 2, kv_heads, d)).astype(np.float16)
    pages = np.zeros((n_pages, po.page_bytes(kv_heads, d, page)), np.uint8)
    for slot in range(n_pages * page):
        po.store(pages, slot, kv[slot, 0], kv[slot, 1], page)
    slots = rng.integers(0, n_pages * page, rows)                       # the same slot twice is fine
    if rows > 3:
        slots[1], slots[2] = -1, n_pages * page
    out = torch.full((rows + 1, cols + 16), 3.0, dtype=torch.float16, device="cuda")
    k.kvpr_paged_read(k.make_paged_desc(heads, kv_heads, d, page, n_pages, 1), torch.from_numpy(pages).cuda(), i32(slots), rows, out, cols + 16)
    torch.cuda.synchronize()
    out = out.cpu().numpy()
    assert (out[rows:] == 3.0).all() and (out[:, cols:] == 3.0).all()
    for i, slot in enumerate(slots):
        if 0 <= slot < n_pages * page:
            want = np.concatenate([io.roundtrip(kv[slot, s].reshape(1, -1))[0] for s in (0, 1)])
            assert np.array_equal(out[i, :cols].view(np.uint16), want.view(np.uint16))
        else:
            assert (out[i] == 3.0).all()


def test_pool_beyond_4_gib(k):
    """Slots whose bytes lie behind the first 2^32."""
    heads, kv_heads, d, page = 64, 64, 128, 256
    n_pages = (1 << 32) // po.page_bytes(kv_heads, d, page) + 3
    pages = torch.zeros((n_pages, po.page_bytes(kv_heads, d, page)), dtype=torch.uint8, device="cuda")
    x = torch.randn((3, 192 * d), device="cuda", dtype=torch.float16)
    slots = i32([n_pages * page - 1, (n_pages - 1) * page, 5])
    desc = k.make_paged_desc(heads, kv_heads, d, page, n_pages, 1)
    out = torch.zeros((3, 128 * d), dtype=torch.float16, device="cuda")
    k.kvpr_paged_append(desc, x, 192 * d, slots, None, 3, None, 0, None, 0, pages)
    k.kvpr_paged_read(desc, pages, slots, 3, out, 128 * d)
    torch.cuda.synchronize()
    want = io.roundtrip(x[:, 64 * d:].cpu().numpy())
    assert np.array_equal(out.cpu().numpy().view(np.uint16), want.view(np.uint16))
    assert int((pages[1:n_pages - 1] != 0).sum()) == 0


@pytest.mark.parametrize("d", [64, 128])
def test_rotation_of_infinities_and_to_nothing(k, d):
    """q with infinities keeps their signs; angles whose products are below the smallest float32 give zeros of the right sign."""
    page, rows = 16, 8
    x = np.random.default_rng(2).standard_normal((rows, 3 * d)).astype(np.float16)
    x[0, 3], x[1, 3], x[2, d // 2 + 5], x[3, d - 1] = np.inf, -np.inf, np.inf, -np.inf
    x[4, 0], x[4, d // 2], x[5, 1] = np.inf, -np.inf, np.nan
    x[6:] = np.float16(2.0 ** -24) * np.where(np.arange(3 * d) % 3 == 0, -1, 1).astype(np.float16)
    table = np.concatenate([k.kvpr_rope_table(6, d), np.full((2, d // 2, 2), 1e-45, np.float32)])
    positions = np.array([1, 2, 3, 4, 5, 0, 6, 7])
    _, q = _append(k, x, np.arange(rows), positions, 1, 1, d, page, 1, table)
    with np.errstate(all="ignore"):
        want = po.rotate(x.reshape(rows, 3, d)[:, :1], table, positions).astype(np.float16).reshape(rows, d)
    assert (np.isinf(want) & (want < 0)).any() and (np.isinf(want) & (want > 0)).any() and (want[6:] == 0).all()
    assert np.array_equal(np.isnan(q), np.isnan(want))
    assert np.array_equal(q.view(np.uint16)[~np.isnan(want)], want.view(np.uint16)[~np.isnan(want)])
