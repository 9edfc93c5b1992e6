"""Append and read-back of thousands of rows, whose kernels take several heads a wave, and what a NaN becomes, against the oracle."""
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


def _store_all(pages, slots, kk, v, page):
    """po.store for many rows: the codec over all of them at once."""
    d, heads = kk.shape[-1], kk.shape[1]
    for x, is_key in ((kk, True), (v, False)):
        codes, scale, mn = io.quantize_rows(x)
        nib = codes[..., 0::2] | codes[..., 1::2] << 4
        pairs = np.stack([scale, mn], -1).astype(np.float16).reshape(*x.shape[:2], -1).view(np.uint8)
        for h in range(heads):
            for t in range(page):
                rows = np.nonzero(slots % page == t)[0]
                at, pair = po._addresses(h, t, d, page, is_key)
                pages[(slots[rows] // page)[:, None], at[None]] = nib[rows, h]
                pages[(slots[rows] // page)[:, None], np.arange(pair, pair + d // 64 * 4)[None]] = pairs[rows, h]


def _slots(rng, rows, page, n_pages):
    """Runs of positions as prompts and drafts have them, from any position of a page, with rows of no slot between; no slot twice."""
    free, slots = list(rng.permutation(n_pages)), []
    while len(slots) < rows:
        m, t = int(rng.choice([1, 2, 3, 5, 37, 300])), int(rng.integers(0, page))
        at = None
        for i in range(m):
            if at is None or t == page:
                if not free:
                    break
                at, t = free.pop(), t % page
            slots.append(at * page + t)
            t += 1
        if not free:
            slots += [-1] * (rows - len(slots))
        if rng.random() < 0.2:
            slots += [-1] * int(rng.integers(1, 4))
    return np.array(slots[:rows])


# heads, kv_heads, d, page, rows: at least 16384 quads of rows times pairs of 64 columns
APPENDS = [(12, 4, 128, 16, 3301), (4, 2, 128, 64, 8200), (9, 3, 64, 32, 8201), (12, 2, 64, 16, 8199), (4, 4, 128, 256, 8202)]


@pytest.mark.parametrize("heads,kv_heads,d,page,rows", APPENDS)
@pytest.mark.parametrize("rope", [False, True])
def test_append_many_rows(k, heads, kv_heads, d, page, rows, rope):
    if not rope:                                                        # without q there are fewer heads
        rows = max(rows, -(-16384 // (2 * kv_heads * d // 128)) * 4 + 1)
    rng = np.random.default_rng(rows)
    n_pages = rows // page + rows // 60 + 8
    x = rng.standard_normal((rows, heads + 2 * kv_heads, d)).astype(np.float16)
    slots = _slots(rng, rows, page, n_pages)
    assert (slots >= 0).sum() > rows // 2 and len(set(slots[slots >= 0])) == (slots >= 0).sum()
    quads = (rows + 3) // 4 * ((((heads if rope else 0) + 2 * kv_heads) * d + 127) // 128)
    assert quads >= 16384
    table = k.kvpr_rope_table(500, d) if rope else None
    positions = rng.integers(-3, 503, rows) if rope else np.zeros(rows, int)
    pages = torch.full((n_pages, po.page_bytes(kv_heads, d, page)), 0xA5, dtype=torch.uint8, device="cuda")
    qkv = torch.from_numpy(x.reshape(rows, -1)).cuda()
    q = torch.full((rows + 1, heads * d + 8), 3.0, dtype=torch.float16, device="cuda") if rope else None
    desc = k.make_paged_desc(heads, kv_heads, d, page, n_pages, 1)
    k.kvpr_paged_append(desc, qkv, x[0].size, i32(slots), i32(positions) if rope else None, rows, torch.from_numpy(table).cuda() if rope else None, 500 if rope else 0, q,
                        heads * d + 8 if rope else 0, pages)
    torch.cuda.synchronize()
    there = (positions >= 0) & (positions < 500) if rope else np.ones(rows, bool)
    kk = x[:, heads:heads + kv_heads]
    if rope:
        turned = po.rotate(x[:, :heads + kv_heads], table, np.where(there, positions, 0)).astype(np.float16)
        kk, got = turned[:, heads:], q.cpu().numpy()
        assert np.array_equal(got[:rows][there][:, :heads * d].view(np.uint16), turned[there][:, :heads].reshape(-1, heads * d).view(np.uint16))
        assert (got[:rows][~there] == 3.0).all() and (got[rows] == 3.0).all() and (got[:, heads * d:] == 3.0).all()
    want = np.full((n_pages, po.page_bytes(kv_heads, d, page)), 0xA5, np.uint8)
    kept = there & (slots >= 0)
    _store_all(want, slots[kept], kk[kept], x[kept][:, heads + kv_heads:], page)
    assert np.array_equal(pages.cpu().numpy(), want)
    if rope:                                                            # q rotated where it is
        pages.fill_(0xA5)
        k.kvpr_paged_append(desc, qkv, x[0].size, i32(slots), i32(positions), rows, torch.from_numpy(table).cuda(), 500, qkv, x[0].size, pages)
        torch.cuda.synchronize()
        after = x.copy()
        after[there, :heads] = turned[there, :heads]
        assert np.array_equal(qkv.cpu().numpy().view(np.uint16), after.reshape(rows, -1).view(np.uint16)) and np.array_equal(pages.cpu().numpy(), want)


@pytest.mark.parametrize("kv_heads,d,page,rows", [(4, 128, 16, 8203), (7, 64, 32, 9501), (12, 128, 64, 2741), (1, 128, 16, 32770), (9, 64, 16, 7282)])
def test_read_many_rows(k, kv_heads, d, page, rows):
    assert (rows + 3) // 4 * ((2 * kv_heads * d + 127) // 128) >= 16384
    rng = np.random.default_rng(rows)
    n_pages, cols = 11, 2 * kv_heads * d
    kv = rng.standard_normal((n_pages * page, 2, kv_heads, d)).astype(np.float16)
    pages = np.zeros((n_pages, po.page_bytes(kv_heads, d, page)), np.uint8)
    _store_all(pages, np.arange(n_pages * page), kv[:, 0], kv[:, 1], page)
    slots = rng.integers(-2, n_pages * page + 2, rows)                  # the same slot many times, some outside the pool
    out = torch.full((rows + 1, cols + 16), 3.0, dtype=torch.float16, device="cuda")
    k.kvpr_paged_read(k.make_paged_desc(kv_heads, kv_heads, d, page, n_pages, 1), torch.from_numpy(pages).cuda(), i32(slots), rows, out, cols + 16)
    torch.cuda.synchronize()
    out = out.cpu().numpy()
    assert (out[rows:] == 3.0).all() and (out[:, cols:] == 3.0).all()
    there = (slots >= 0) & (slots < n_pages * page)
    want = io.roundtrip(kv.reshape(n_pages * page, -1))
    assert np.array_equal(out[:rows][there][:, :cols].view(np.uint16), want[slots[there]].view(np.uint16))
    assert (out[:rows][~there] == 3.0).all()


def test_the_oracles_two_ways_to_store():
    rng = np.random.default_rng(3)
    a, b = (np.zeros((3, po.page_bytes(2, 128, 16)), np.uint8) for _ in range(2))
    slots, kk, v = rng.permutation(48)[:20], *(rng.standard_normal((20, 2, 128)).astype(np.float16) for _ in range(2))
    _store_all(a, slots, kk, v, 16)
    for i, s in enumerate(slots):
        po.store(b, int(s), kk[i], v[i], 16)
    assert np.array_equal(a, b)


@pytest.mark.parametrize("d", [64, 128])
def test_nan_counts_as_the_smallest_of_its_group(k, d):
    """One NaN, several, all but one, all: code 0 beside the scale and minimum of the numbers; a group of NaN alone keeps NaN as its pair and codes 0.  With
    an infinity in the group no value comes back finite."""
    page, rows = 16, 9
    x = np.random.default_rng(4).standard_normal((rows, 3, d)).astype(np.float16)
    x[1, 1, 5], x[2, 2, d - 1], x[3, 1, :64:3], x[4, 2, 1:64], x[5, 1], x[6, 2, -64:] = (np.nan,) * 6
    x[7, 1, 3], x[7, 1, 4], x[8, 2, 0], x[8, 2, 1] = np.nan, np.inf, np.nan, -np.inf
    pages = torch.full((1, po.page_bytes(1, d, page)), 0xA5, dtype=torch.uint8, device="cuda")
    k.kvpr_paged_append(k.make_paged_desc(1, 1, d, page, 1, 1), torch.from_numpy(x.reshape(rows, -1)).cuda(), 3 * d, i32(np.arange(rows)), None, rows, None, 0, None, 0, pages)
    torch.cuda.synchronize()
    got = pages.cpu().numpy()
    for t in range(rows):
        for side, (codes, scale, mn) in enumerate(po.load(got, t, 1, d, page)):
            for g in range(d // 64):
                group = x[t, 1 + side, 64 * g:64 * g + 64]
                c, s, m = codes[0, 64 * g:64 * g + 64], scale[0, g], mn[0, g]
                if np.isnan(group).all():
                    assert np.isnan(s) and np.isnan(m) and (c == 0).all(), (t, side, g)
                elif np.isinf(group).any():
                    with np.errstate(all="ignore"):
                        assert not np.isfinite(c.astype(np.float64) * float(s) + float(m)).any(), (t, side, g)
                else:
                    filled = np.where(np.isnan(group), np.nanmin(group), group)
                    wc, ws, wm = io.quantize_rows(filled[None])
                    assert np.array_equal(c, wc[0]) and s == ws[0, 0] and m == wm[0, 0], (t, side, g)
                    assert (c[np.isnan(group)] == 0).all()
