"""Pins of the paged oracle: pages against the codec oracle, hand-made plans and verifications."""
import numpy as np
import pytest

from oracle import kvpr_int4_oracle as io
from oracle import kvpr_paged_oracle as po


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
def test_pages_hold_what_was_stored_and_every_byte_once(d, page):
    rng = np.random.default_rng(d + page)
    heads, n_pages = 3, 2
    pages = np.zeros((n_pages, po.page_bytes(heads, d, page)), np.uint8)
    touched = np.zeros_like(pages, dtype=int)
    rows = {}
    for slot in rng.permutation(n_pages * page):
        k, v = (rng.standard_normal((heads, d)).astype(np.float16) for _ in range(2))
        po.store(pages, slot, k, v, page)
        rows[int(slot)] = (k, v)
        for h in range(heads):
            for is_key in (True, False):
                codes, pair = po._addresses(h, slot % page, d, page, is_key)
                touched[slot // page][codes] += 1
                touched[slot // page][pair:pair + d // 64 * 4] += 1
    assert (touched == 1).all()
    for slot, (k, v) in rows.items():
        for got, x in zip(po.load(pages, slot, heads, d, page), (k, v)):
            want = io.quantize_rows(x)
            assert all(np.array_equal(a, b) for a, b in zip(got, want))


def test_plan_by_hand():
    table = np.array([[3, -1, -1], [5, 6, 7], [-1, -1, -1], [-1, -1, -1], [9, -1, -1]])
    free = np.array([1, 2, 0, 0, 0, 0, 0, 0, 0, 0])
    #        grows by one page, gives two back, takes one, finds none left, needs none
    got = po.plan([16, 4, 0, 0, 3], [1, 1, 10, 40, 2], [1, 3, 0, 0, 1], table, free, 2, 16, 60, 10)
    assert got["held"] == [2, 1, 1, 0, 1] and got["refused"] == 1 and got["count"] == 2
    assert got["free"][:4].tolist() == [1, 2, 6, 7]
    assert got["table"][0, 1] == 7 and got["table"][2, 0] == 6
    assert got["seq_len"] == [17, 5, 10, 0, 5]
    assert got["row_start"].tolist() == [0, 1, 2, 12, 52, 54]
    assert got["slots"][0] == 7 * 16 and got["slots"][1] == 5 * 16 + 4 and got["slots"][2] == 96 and (got["slots"][12:52] == -1).all()
    assert got["slots"][52:54].tolist() == [9 * 16 + 3, 9 * 16 + 4] and (got["slots"][54:] == -1).all()


def test_verification_by_hand():
    ln = lambda *p: np.log(np.array(p))                                                 # noqa: E731
    target = np.stack([ln(.5, .25, .25), ln(.1, .6, .3), ln(.2, .2, .6)])
    draft = np.stack([ln(1 / 3, 1 / 3, 1 / 3), ln(.25, .5, .25), ln(.6, .3, .1)])
    tok, start = [0, 1, 0], [0, 3]
    # draft 1: p/q = .5; draft 0: p/q = 1/6
    run = lambda u, s: po.verify(target, draft, tok, start, [1.0], [0, *u], [s], 3)      # noqa: E731
    assert run((.49, .16), .3) == ([1, 0, 1], [3])          # both stand; behind them cdf .2, .4, 1
    assert run((.49, .17), .3) == ([1, 1, -1], [2])         # residual of row 1: 0, .3, .2
    assert run((.49, .17), .61) == ([1, 2, -1], [2])
    assert run((.51, .0), .99) == ([0, -1, -1], [1])        # residual of row 0: .25, 0, 0
    assert po.verify(target, None, tok, start, [1.0], [0, .24, .09], [.1], 3) == ([1, 0, 0], [3])
    assert po.verify(target, None, tok, start, [1.0], [0, .26, .09], [.7], 3) == ([2, -1, -1], [1])   # .5, -, .25
    assert po.verify(target, draft, [9, 0, 1], start, [0.0], [0, 0, 0], [0], 3) == ([0, 1, 2], [3])


def test_attention_by_hand():
    d, page = 64, 16
    pages = np.zeros((2, po.page_bytes(1, d, page)), np.uint8)
    k = np.zeros((1, d), np.float16)
    for t, c in enumerate((1.0, 3.0)):
        po.store(pages, 16 + t, k, np.full((1, d), c, np.float16), page)
    q = np.ones((2, 2 * d))
    z, tol, done = po.attention(q, pages, np.array([[1]]), [0, 2], [2], 2, 1, d, page, 2)
    assert done.all() and np.allclose(z[0], 1.0) and np.allclose(z[1], 2.0) and (tol < 2e-3).all()
    z, _, _ = po.attention(q, pages, np.array([[1]]), [0, 2], [1], 2, 1, d, page, 2)
    assert np.allclose(z[0], 0.0) and np.allclose(z[1], 1.0)
