"""Append and read-back of more rows than one launch takes: what lies at the borders of launches, against the oracle."""
import numpy as np
import pytest
import torch

from oracle import kvpr_int4_oracle as io
from oracle import kvpr_paged_oracle as po
from paged_testlib import i32

pytestmark = pytest.mark.gpu

D, PAGE, N_PAGES, BORDER = 64, 16, 4, 1 << 24


@pytest.fixture(scope="module")
def k():
    import paper_2411_17089_amd as k
    return k


def _rows_that_count(rows):
    """Some rows, among them two quads of positions that lie across the border, whole and with their last row elsewhere."""
    at = np.array([0, 1, 5, BORDER - 7, BORDER - 2, BORDER - 1, BORDER, BORDER + 1, BORDER + 2, BORDER + 3, BORDER + 4, BORDER + 5, rows - 1])
    slots = np.array([3, 4, 9, 30, 20, 21, 22, 23, 40, 41, 42, 43, 60])
    return at, slots


@pytest.mark.parametrize("rope", [False, True])
def test_append_across_launches(k, rope):
    rows = BORDER + 37
    rng = np.random.default_rng(1)
    at, where = _rows_that_count(rows)
    x = rng.standard_normal((len(at), 3 * D)).astype(np.float16)
    qkv = torch.empty((rows, 3 * D), dtype=torch.float16, device="cuda")
    slots, positions = (torch.full((rows,), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    index = torch.from_numpy(at).cuda()
    qkv[index], slots[index] = torch.from_numpy(x).cuda(), i32(where)
    near = at[4] - 1                                                    # a row that is turned but has no slot
    qkv[near] = 1.0
    pos = rng.integers(0, 50, len(at))
    positions[index], positions[near] = i32(pos), 7
    table = k.kvpr_rope_table(50, D)
    pages = torch.full((N_PAGES, po.page_bytes(1, D, PAGE)), 0xA5, dtype=torch.uint8, device="cuda")
    q = torch.full((rows, D), 3.0, dtype=torch.float16, device="cuda") if rope else None
    desc = k.make_paged_desc(1, 1, D, PAGE, N_PAGES, 1)
    k.kvpr_paged_append(desc, qkv, 3 * D, slots, positions if rope else None, rows, torch.from_numpy(table).cuda() if rope else None, 50 if rope else 0, q, D if rope else 0, pages)
    torch.cuda.synchronize()
    h = x.reshape(-1, 3, D)
    kk, want_q = h[:, 1:2], None
    if rope:
        kk, want_q = (po.rotate(a, table, pos).astype(np.float16) for a in (h[:, 1:2], h[:, :1]))
    want = np.full((N_PAGES, po.page_bytes(1, D, PAGE)), 0xA5, np.uint8)
    for i, slot in enumerate(where):
        po.store(want, int(slot), kk[i], h[i, 2:], PAGE)
    assert np.array_equal(pages.cpu().numpy(), want)
    if rope:
        assert np.array_equal(q[index].cpu().numpy().view(np.uint16), want_q[:, 0].view(np.uint16))
        turned = po.rotate(np.ones((1, 1, D), np.float16), table, [7]).astype(np.float16)[0, 0]
        assert np.array_equal(q[near].cpu().numpy().view(np.uint16), turned.view(np.uint16))
        q[index] = 3.0
        q[near] = 3.0
        assert bool((q == 3.0).all())


def test_read_of_more_rows_than_a_grid_has_threads(k):
    rows = (1 << 26) + 9                                                # four rows a workgroup of 256: 2^32 threads
    rng = np.random.default_rng(2)
    kv = rng.standard_normal((N_PAGES * PAGE, 2, 1, D)).astype(np.float16)
    pages = np.zeros((N_PAGES, po.page_bytes(1, D, PAGE)), np.uint8)
    for slot in range(N_PAGES * PAGE):
        po.store(pages, slot, kv[slot, 0], kv[slot, 1], PAGE)
    at, where = _rows_that_count(rows)
    at, where = np.concatenate([at, [(1 << 26) - 1, 1 << 26, 3 * BORDER + 5]]), np.concatenate([where, [1, 2, 50]])
    out = torch.empty((rows, 2 * D), dtype=torch.float16, device="cuda")
    slots = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    index = torch.from_numpy(at).cuda()
    beside = index[4] - 1
    out[index], out[beside], slots[index] = 3.0, 3.0, i32(where)
    k.kvpr_paged_read(k.make_paged_desc(1, 1, D, PAGE, N_PAGES, 1), torch.from_numpy(pages).cuda(), slots, rows, out, 2 * D)
    torch.cuda.synchronize()
    want = np.stack([np.concatenate([io.roundtrip(kv[s, i].reshape(1, -1))[0] for i in (0, 1)]) for s in where])
    assert np.array_equal(out[index].cpu().numpy().view(np.uint16), want.view(np.uint16))
    assert bool((out[beside] == 3.0).all())
