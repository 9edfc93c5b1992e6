"""The plan of a ragged step against the oracle: whole arrays, what is left alone included."""
import numpy as np
import pytest
import torch

from oracle import kvpr_paged_oracle as po
from paged_testlib import i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def k():
    import paper_2411_17089_amd as k
    return k


def _state(rng, n, page, base_hi, new_hi, extra=0, spare=None, stale=0.2, idle=0.2):
    base = rng.integers(0, base_hi + 1, n)
    new = np.where(rng.random(n) < idle, 0, rng.integers(0, new_hi + 1, n))
    held = -(-base // page) + np.where(rng.random(n) < stale, rng.integers(0, 4, n), 0)
    gone = rng.random(n) < 0.1                                        # finished requests that still hold pages
    base[gone], new[gone] = 0, 0
    width = int(max(held.max(), (-(-(base + new) // page)).max())) + extra
    width = max(width, 1)
    need = int(np.maximum(-(-(base + new) // page) - held, 0).sum())
    spare = need + 3 if spare is None else spare
    n_pages = max(int(held.sum()) + spare, 1)
    order = rng.permutation(n_pages)
    table = np.full((n, width), -7, dtype=np.int64)
    at = 0
    for r in range(n):
        table[r, :held[r]] = order[at:at + held[r]]
        at += held[r]
    free = np.full(n_pages, -9, dtype=np.int64)
    free[:spare] = order[at:]
    return base, new, held, table, free, spare, n_pages


def _run(k, base, new, held, table, free, count, n_pages, page, max_rows, in_place=False):
    n = len(base)
    d = dict(base=i32(base), new=i32(new), held=i32(held), table=i32(table), free=i32(free), count=i32([count]))
    out = {name: torch.full((size,), -77, dtype=torch.int32, device="cuda") for name, size in
           (("held", n), ("count", 1), ("row_start", n + 1), ("seq_len", n), ("slots", max_rows + 5), ("positions", max_rows + 5), ("refused", 1))}
    if in_place:
        out["held"], out["count"] = d["held"], d["count"]
    desc = k.make_paged_desc(1, 1, 64, page, n_pages, table.shape[1])
    k.kvpr_paged_plan(desc, d["base"], d["new"], n, d["table"], d["held"], out["held"], d["free"], d["count"], out["count"], max_rows,
                      out["row_start"], out["seq_len"], out["slots"], out["positions"], out["refused"])
    torch.cuda.synchronize()
    assert (out["slots"][max_rows:] == -77).all() and (out["positions"][max_rows:] == -77).all()
    out["slots"], out["positions"] = out["slots"][:max_rows], out["positions"][:max_rows]
    out.update(table=d["table"], free=d["free"])
    assert np.array_equal(d["base"].cpu().numpy(), base) and np.array_equal(d["new"].cpu().numpy(), new)
    return {name: v.cpu().numpy() for name, v in out.items()}


def _check(got, want):
    for name, v in got.items():
        w = np.asarray(want[name]).reshape(v.shape)
        assert np.array_equal(v, w), (name, np.flatnonzero(v.ravel() != w.ravel())[:5])


@pytest.mark.parametrize("n,page,base_hi,new_hi", [(1, 16, 0, 1), (1, 16, 100, 700), (2, 256, 500, 3), (7, 32, 90, 5), (64, 16, 300, 9), (65, 64, 3000, 1),
                                                   (200, 16, 40, 200), (1023, 16, 64, 3), (1025, 128, 300, 2), (3000, 16, 50, 2), (8192, 16, 20, 1)])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan(k, n, page, base_hi, new_hi, in_place):
    rng = np.random.default_rng(n * 1000 + page)
    base, new, held, table, free, count, n_pages = _state(rng, n, page, base_hi, new_hi, extra=n % 3)
    total = int(new.sum())
    for max_rows in {total, total + 7}:
        want = po.plan(base, new, held, table, free, count, page, max_rows, n_pages)
        assert want["refused"] == 0
        _check(_run(k, base, new, held, table, free, count, n_pages, page, max_rows, in_place), want)


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("n", [3, 70, 1500])
def test_too_few_pages(k, n, seed):
    rng = np.random.default_rng(seed)
    base, new, held, table, free, count, n_pages = _state(rng, n, 16, 60, 90, extra=2, spare=[0, 1, 2, n, n + n // 2, 3 * n][seed])
    want = po.plan(base, new, held, table, free, count, 16, int(new.sum()) + 1, n_pages)
    _check(_run(k, base, new, held, table, free, count, n_pages, 16, int(new.sum()) + 1), want)


def test_longer_than_the_table_and_fewer_rows_than_tokens(k):
    rng = np.random.default_rng(3)
    base, new, held, table, free, count, n_pages = _state(rng, 40, 16, 60, 20, extra=0)
    new[11], new[30] = 16 * table.shape[1] + 1 - base[11], 16 * table.shape[1] - base[30]
    want = po.plan(base, new, held, table, free, count, 16, 50, n_pages)
    assert want["refused"] >= 1 and want["seq_len"][11] == 0
    _check(_run(k, base, new, held, table, free, count, n_pages, 16, 50), want)
    _check(_run(k, base, new, held, table, free, count, n_pages, 16, 0), po.plan(base, new, held, table, free, count, 16, 0, n_pages))


def test_nothing_new_and_negative_lengths(k):
    rng = np.random.default_rng(4)
    base, new, held, table, free, count, n_pages = _state(rng, 9, 32, 100, 0)
    new[:] = 0
    new[4], base[6] = -5, -1
    _check(_run(k, base, new, held, table, free, count, n_pages, 32, 3), po.plan(base, new, held, table, free, count, 32, 3, n_pages))


def test_lengths_beyond_32_bits_in_sum_are_refused_not_wrapped(k):
    big = 0x7fffffff
    base, new, held = np.array([big, 5, 3]), np.array([big, big, 2]), np.array([0, 1, 1])
    table, free = np.array([[-7, -7], [2, -7], [0, -7]]), np.array([1, 3, -9, -9])
    got = _run(k, base, new, held, table, free, 2, 4, 16, 4)
    assert got["refused"][0] == 2 and got["seq_len"].tolist() == [0, 0, 5] and got["held"].tolist() == [0, 1, 1] and got["count"][0] == 2
    assert got["row_start"].tolist() == [0, big, big, big] and (got["slots"] == -1).all()
    assert np.array_equal(got["table"], table) and np.array_equal(got["free"], free)


def test_steps_in_a_row_keep_every_page_once(k):
    """Grow, shrink and finish requests over many steps, in place; pages in use and on the stack are always a partition."""
    rng = np.random.default_rng(9)
    n, page, width, n_pages = 37, 16, 12, 150
    held, count = np.zeros(n, int), n_pages
    table, free = np.full((n, width), -7), rng.permutation(n_pages)
    base = np.zeros(n, int)
    for step in range(12):
        new = rng.integers(0, 40, n)
        base = np.where(rng.random(n) < 0.15, 0, np.maximum(base - rng.integers(0, 30, n), 0))
        new = np.where((base + new) > width * page, 0, new)
        want = po.plan(base, new, held, table, free, count, page, int(new.sum()), n_pages)
        got = _run(k, base, new, held, table, free, count, n_pages, page, int(new.sum()), in_place=True)
        _check(got, want)
        held, table, free, count = got["held"], got["table"], got["free"], int(got["count"][0])
        used = np.concatenate([table[r, :held[r]] for r in range(n)] + [free[:count]])
        assert np.array_equal(np.sort(used), np.arange(n_pages))
        base = np.where(got["seq_len"] > 0, base + new, base)
        base = np.minimum(base, held * page)
