"""Verification of drafted tokens against the oracle: whole numbers, all equal."""
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


def _inputs(rng, new, vocab, dtype, greedy=0.25, near=0.5):
    n, rows = len(new), int(np.sum(new))
    target = rng.standard_normal((rows, vocab)) * 2
    target[np.arange(rows), rng.integers(0, vocab, rows)] += 6
    target = target.astype(dtype)
    draft = np.zeros_like(target)
    draft[1:] = (target[:-1].astype(np.float64) + near * rng.standard_normal((max(rows - 1, 0), vocab))).astype(dtype)
    x = draft.astype(np.float64) + rng.gumbel(size=draft.shape)
    tokens = x.argmax(-1)
    temperature = np.where(rng.random(n) < greedy, 0.0, rng.uniform(0.4, 1.5, n)).astype(np.float32)
    start = np.concatenate([[0], np.cumsum(new)])
    for r in range(n):                                                  # greedy drafts: mostly the target's own choice
        if temperature[r] == 0:
            for i in range(start[r] + 1, start[r + 1]):
                if rng.random() < 0.7:
                    tokens[i] = int(target[i - 1].argmax())
    return target, draft, tokens, start, temperature, rng.random(rows).astype(np.float32), rng.random(n).astype(np.float32)


def _run(k, target, draft, tokens, start, temperature, ua, us, n_rows=None, ld=0, len_in=None, same=False):
    n, vocab = len(temperature), target.shape[1]
    n_rows = target.shape[0] if n_rows is None else n_rows

    def up(a):
        if a is None:
            return None
        t = torch.full((max(a.shape[0], 1), vocab + ld), 50.0, dtype=torch.float16 if a.dtype == np.float16 else torch.float32, device="cuda")
        t[:a.shape[0], :vocab] = torch.from_numpy(a).cuda()
        return t

    f32 = lambda a: torch.from_numpy(np.asarray(a, np.float32)).cuda()                  # noqa: E731
    t, d = up(target), up(draft)
    kept = torch.full((n,), -77, dtype=torch.int32, device="cuda")
    out = torch.full((max(target.shape[0], 1),), -77, dtype=torch.int32, device="cuda")
    li = None if len_in is None else i32(len_in)
    lo = li if same else None if li is None else torch.zeros_like(li)
    ws = torch.full((k.kvpr_verify_workspace_bytes(n, n_rows, vocab),), 0xFF, dtype=torch.uint8, device="cuda")
    k.kvpr_verify_drafts(t, d, k.KVPR_F16 if target.dtype == np.float16 else k.KVPR_F32, vocab + ld, vocab + ld, vocab, i32(tokens), i32(start), n, n_rows,
                         f32(temperature), f32(ua), f32(us), li, lo, kept, out, ws, ws.numel())
    torch.cuda.synchronize()
    return out.cpu().numpy()[:target.shape[0]], kept.cpu().numpy(), None if lo is None else lo.cpu().numpy()


def _check(got, want):
    out, kept, lens = got
    w_out, w_kept = want
    assert kept.tolist() == w_kept
    assert out.tolist() == [-77 if v is None else v for v in w_out]


@pytest.mark.parametrize("vocab", [1, 2, 63, 64, 65, 1000, 4095, 4096, 4097, 9001, 32000, 50272])
@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("with_draft", [True, False])
def test_verify(k, vocab, dtype, with_draft):
    rng = np.random.default_rng(vocab)
    new = [1, 5, 2, 8, 3, 0, 1, 4, 6, 2, 3]
    target, draft, *rest = _inputs(rng, new, vocab, dtype)
    draft = draft if with_draft else None
    print("verify", vocab, dtype.__name__, with_draft, flush=True)
    for ld in (0, 3):
        _check(_run(k, target, draft, *rest, ld=ld), po.verify(target, draft, *rest, n_rows=target.shape[0]))


@pytest.mark.parametrize("rows,vocab", [(200, 9001), (330, 9001), (6, 700001)])
def test_sizes_of_chunks(k, rows, vocab):
    """The first launch in chunks of 4096 and of 8192 logits, and a vocabulary of more chunks than a workgroup has threads."""
    rng = np.random.default_rng(rows)
    new = [3] * (rows // 3) + [1] * (rows % 3)
    for dtype in (np.float16, np.float32):
        target, draft, *rest = _inputs(rng, new, vocab, dtype)
        _check(_run(k, target, draft, *rest), po.verify(target, draft, *rest, n_rows=target.shape[0]))


@pytest.mark.parametrize("seed", range(20))
def test_many_requests(k, seed):
    rng = np.random.default_rng(seed + 50)
    new = rng.integers(0, 9, 60)
    new[0] = 2
    target, draft, *rest = _inputs(rng, new, 300, np.float32, near=[0.05, 0.5, 2.0][seed % 3])
    lens = rng.integers(0, 5000, 60)
    want = po.verify(target, draft, *rest, n_rows=target.shape[0])
    got = _run(k, target, draft, *rest, len_in=lens, same=seed % 2 == 0)
    _check(got, want)
    assert got[2].tolist() == (lens + np.array(want[1])).tolist()


def test_more_rows_than_threads(k):
    rng = np.random.default_rng(1)
    target, draft, tokens, start, temperature, ua, us = _inputs(rng, [1500, 3, 1100], 70, np.float32, greedy=0, near=0.0)
    ua[:] = 0.0                                                         # every draft of positive probability stands
    ua[1400], tokens[2000] = 0.5, -1
    _check(_run(k, target, draft, tokens, start, temperature, ua, us), po.verify(target, draft, tokens, start, temperature, ua, us, target.shape[0]))
    _check(_run(k, target, draft, tokens, start, np.zeros(3, np.float32), ua, us), po.verify(target, draft, tokens, start, np.zeros(3), ua, us, target.shape[0]))


def test_rows_behind_the_last_and_fewer_rows_than_tokens(k):
    rng = np.random.default_rng(2)
    target, draft, tokens, start, temperature, ua, us = _inputs(rng, [3, 4, 5], 500, np.float32)
    start = np.array([0, 3, 7, 9])                                       # rows 9 .. 11 belong to nobody
    _check(_run(k, target, draft, tokens, start, temperature, ua, us), po.verify(target, draft, tokens, start, temperature, ua, us, 12))
    start = np.array([0, 3, 7, 12])
    got = _run(k, target, draft, tokens, start, temperature, ua, us, n_rows=5)
    want = po.verify(target, draft, tokens, start, temperature, ua, us, 5)
    assert got[1].tolist() == want[1] and got[0][:5].tolist() == want[0] and (got[0][5:] == -77).all()


def test_masked_infinite_and_nan_logits(k):
    rng = np.random.default_rng(3)
    inf, nan = np.inf, np.nan
    for dtype in (np.float32, np.float16):
        target, draft, tokens, start, temperature, ua, us = _inputs(rng, [4] * 12, 700, dtype)
        target[:, ::3] = -inf                                            # a third of the vocabulary is masked
        draft[:, 1::5] = -inf
        target[0], target[5], draft[9] = -inf, nan, -inf                 # rows without a distribution
        target[12, 7], target[13, 8], target[17, 4] = inf, nan, inf
        target[20], target[24, :] = 3.0, np.finfo(dtype).min             # ties throughout; the type's lowest value throughout
        target[28, 10:] = np.finfo(dtype).min
        draft[30, 5], draft[34, 6] = inf, nan
        tokens[37], tokens[41], tokens[45] = 700, -1, 2 ** 31 - 1
        for t in (temperature, np.zeros(12, np.float32), np.full(12, 1e-3, np.float32), np.full(12, 1e30, np.float32), np.full(12, np.nan, np.float32),
                  np.full(12, -1, np.float32)):
            for d in (draft, None):
                _check(_run(k, target, d, tokens, start, t, ua, us), po.verify(target, d, tokens, start, t, ua, us, 48))


def test_uniform_numbers_at_their_ends(k):
    rng = np.random.default_rng(4)
    top = np.float32(1) - np.float32(2) ** -24
    for d in (True, False):
        target, draft, tokens, start, temperature, ua, us = _inputs(rng, [3, 1, 6, 2, 4], 5000, np.float32, greedy=0)
        for a in (0.0, top):
            for s in (0.0, top):
                ua[:], us[:] = a, s
                _check(_run(k, target, draft if d else None, tokens, start, temperature, ua, us),
                       po.verify(target, draft if d else None, tokens, start, temperature, ua, us, 16))


def test_equal_models_accept_everything(k):
    rng = np.random.default_rng(5)
    target, draft, tokens, start, temperature, ua, us = _inputs(rng, [6] * 9, 4000, np.float32, greedy=0, near=0.0)
    out, kept, _ = _run(k, target, draft, tokens, start, temperature, ua, us)
    assert kept.tolist() == [6] * 9
    _check((out, kept, None), po.verify(target, draft, tokens, start, temperature, ua, us, 54))


def test_shares_of_drawn_tokens(k):
    """The tokens that come out are distributed as the target's: 4096 requests over 8 tokens with uniform numbers; each count is
    binomial, so within 6 standard deviations (chance of a miss below 10^-8)."""
    rng = np.random.default_rng(6)
    n, vocab = 4096, 8
    logits, guess = rng.standard_normal(vocab), rng.standard_normal(vocab)
    target, draft = np.tile(logits, (2 * n, 1)).astype(np.float32), np.tile(guess, (2 * n, 1)).astype(np.float32)
    q = np.exp(guess) / np.exp(guess).sum()
    tokens = rng.choice(vocab, 2 * n, p=q)
    start = np.arange(n + 1) * 2
    out, kept, _ = _run(k, target, draft, tokens, start, np.ones(n, np.float32), rng.random(2 * n), rng.random(n))
    p = np.exp(logits) / np.exp(logits).sum()
    counts = np.bincount(out[0::2], minlength=vocab)
    assert (np.abs(counts - n * p) < 6 * np.sqrt(n * p * (1 - p))).all()
