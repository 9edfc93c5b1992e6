"""Steps of a ragged batch in which the plan refuses requests: nothing of a refused request is kept, its length stays, and it goes on
when pages come back.  Each stage against the oracle on its own inputs, and the same steps from a graph, bit for bit."""
import numpy as np
import pytest
import torch

from oracle import kvpr_paged_oracle as po
from paged_testlib import i32

pytestmark = pytest.mark.gpu

VOCAB, H, HEADS, KV, D, PAGE = 320, 128, 4, 1, 64, 16
NEW = [1, 3, 5, 2, 4, 3]                                                # rows of each request in a step
N, ROWS, COLS, WIDTH = len(NEW), sum(NEW), (HEADS + 2 * KV) * D, 5
STEPS, LEAVES = 12, {6: 2, 9: 4}                                        # steps before which a request ends


@pytest.fixture(scope="module")
def k():
    import paper_2411_17089_amd as k
    return k


class Server:
    def __init__(self, k, seed, n_pages):
        self.k, self.n_pages = k, n_pages
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device="cuda") * scale).half()     # noqa: E731
        z = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype, device="cuda")                      # noqa: E731
        self.emb, self.wqkv, self.wlm = normal(VOCAB, H), normal(COLS, H, scale=0.1), normal(VOCAB, HEADS * D, scale=0.3)
        self.rope = torch.from_numpy(k.kvpr_rope_table(WIDTH * PAGE, D)).cuda()
        self.desc = k.make_paged_desc(HEADS, KV, D, PAGE, n_pages, WIDTH)
        self.pages = z(n_pages, k.kvpr_page_bytes(self.desc), dtype=torch.uint8)
        self.base, self.new, self.held = i32([12, 9, 14, 0, 15, 11]), i32(NEW), i32([0] * N)
        self.table = torch.full((N, WIDTH), -1, dtype=torch.int32, device="cuda")
        self.free, self.count = torch.randperm(n_pages, generator=g, device="cuda").int(), i32([n_pages])
        self.row_start, self.seq_len, self.slots, self.positions, self.refused = z(N + 1), z(N), z(ROWS), z(ROWS), z(1)
        self.tokens = torch.randint(0, VOCAB, (ROWS,), generator=g, device="cuda", dtype=torch.int32)
        self.qkv, self.q, self.z = (z(ROWS, c, dtype=torch.float16) for c in (COLS, HEADS * D, HEADS * D))
        self.logits, self.draft_logits = z(ROWS, VOCAB, dtype=torch.float32), z(ROWS, VOCAB, dtype=torch.float32)
        self.kept, self.out = z(N), z(ROWS)
        self.temperature = torch.tensor([0.0, 0.7, 1.0, 3.0, 0.0, 1.3], device="cuda")
        self.ws = z(k.kvpr_paged_attention_workspace_bytes(self.desc, N, ROWS, max(NEW), WIDTH * PAGE), dtype=torch.uint8)
        self.ws_v = z(k.kvpr_verify_workspace_bytes(N, ROWS, VOCAB), dtype=torch.uint8)
        self.drafts = torch.randint(0, VOCAB, (STEPS, ROWS), generator=g, device="cuda", dtype=torch.int32)
        self.guesses = torch.randn((STEPS, ROWS, VOCAB), generator=g, device="cuda")
        self.u = torch.rand((STEPS, ROWS + N), generator=g, device="cuda")
        self.step_no = z(1, dtype=torch.int64)
        # owner and place of every row while all requests are there
        self.owner = torch.repeat_interleave(torch.arange(N, device="cuda"), torch.tensor(NEW, device="cuda"))
        self.first = torch.tensor(np.cumsum([0] + NEW[:-1]), device="cuda")

    def forward(self):
        k = self.k
        k.kvpr_paged_plan(self.desc, self.base, self.new, N, self.table, self.held, self.held, self.free, self.count, self.count, ROWS, self.row_start,
                          self.seq_len, self.slots, self.positions, self.refused)
        k.kvpr_recompute_gemm(self.emb[self.tokens.long()], self.wqkv, None, self.qkv, ROWS, COLS, H, COLS)
        k.kvpr_paged_append(self.desc, self.qkv, COLS, self.slots, self.positions, ROWS, self.rope, self.rope.shape[0], self.q, HEADS * D, self.pages)
        k.kvpr_paged_attention(self.desc, self.q, k.KVPR_F16, HEADS * D, self.pages, self.table, self.row_start, self.seq_len, N, ROWS, max(NEW), WIDTH * PAGE,
                               self.z, HEADS * D, self.ws, self.ws.numel())
        k.kvpr_token_gemm(self.z, self.wlm, None, self.logits, None, ROWS, VOCAB, HEADS * D, VOCAB, VOCAB)
        u = self.u.index_select(0, self.step_no)[0]
        self.ua, self.us = u[:ROWS].contiguous(), u[ROWS:].contiguous()
        self.draft_logits.copy_(self.guesses.index_select(0, self.step_no)[0])
        k.kvpr_verify_step(self.logits, self.draft_logits, k.KVPR_F32, VOCAB, VOCAB, VOCAB, self.tokens, self.row_start, self.seq_len, None, N, ROWS,
                           self.temperature,
                           self.ua, self.us, self.base, self.base, self.kept, self.out, self.ws_v, self.ws_v.numel())

    def advance(self):
        """Row 0 of a request: the token behind what was kept, or the one that could not be fed; the others: new drafts."""
        first = self.row_start[:-1].long().clamp(max=ROWS - 1)
        last = self.out[(first + self.kept - 1).clamp(min=0)]
        last = torch.where(self.kept > 0, last, self.tokens[first])
        row = torch.arange(ROWS, device="cuda")
        owner = torch.searchsorted(self.row_start[1:].contiguous(), row.int(), right=True).clamp(max=N - 1)
        self.tokens.copy_(torch.where(row == first[owner], last[owner], self.drafts.index_select(0, self.step_no)[0]))
        self.step_no.add_(1).remainder_(STEPS)

    def leave(self, step):
        """A request that ends: its pages go back with the next plan, and its place has no rows."""
        if step in LEAVES:
            self.base[LEAVES[step]] = 0
            self.new[LEAVES[step]] = 0
            start = torch.cumsum(torch.cat([self.new.new_zeros(1), self.new]), 0)
            row = torch.arange(ROWS, device="cuda")
            owner = torch.searchsorted(start[1:].contiguous(), row, right=True).clamp(max=N - 1)
            old = (self.row_start[:-1][owner] + row - start[owner]).clamp(max=ROWS - 1)
            self.tokens.copy_(torch.where(row < start[-1], self.tokens[old.long()], 0))

    def state(self):
        return [t.clone() for t in (self.base, self.held, self.table, self.free, self.count, self.pages, self.tokens, self.out, self.kept, self.z, self.logits, self.refused)]


N_PAGES = 9                                                             # six requests want up to three pages each


def test_steps_with_refused_requests(k):
    s = Server(k, 1, N_PAGES)
    n = lambda t: t.cpu().numpy()                                                       # noqa: E731
    refused_before, went_on, refusals = set(), set(), 0
    for step in range(STEPS):
        s.leave(step)
        before = {name: n(getattr(s, name)).copy() for name in ("base", "new", "held", "table", "free", "count", "pages", "tokens")}
        s.forward()
        torch.cuda.synchronize()
        want = po.plan(before["base"], before["new"], before["held"], before["table"], before["free"], int(before["count"][0]), PAGE, ROWS, N_PAGES)
        for name, got in (("table", s.table), ("free", s.free), ("held", s.held), ("count", s.count), ("row_start", s.row_start), ("seq_len", s.seq_len),
                          ("slots", s.slots), ("positions", s.positions), ("refused", s.refused)):
            assert np.array_equal(n(got).ravel(), np.asarray(want[name]).ravel()), (step, name)
        heads = n(s.qkv).reshape(ROWS, -1, D)
        kk = po.rotate(heads[:, HEADS:HEADS + KV], n(s.rope), want["positions"]).astype(np.float16)
        pages = before["pages"].copy()
        for i in range(ROWS):
            if want["slots"][i] >= 0:
                po.store(pages, int(want["slots"][i]), kk[i], heads[i, HEADS + KV:], PAGE)
        assert np.array_equal(n(s.pages), pages), step
        z, tol, done = po.attention(n(s.q), pages, n(s.table), n(s.row_start), n(s.seq_len), HEADS, KV, D, PAGE, ROWS)
        assert (np.abs(n(s.z).astype(np.float64) - z) <= tol)[done].all(), step
        out, kept = po.verify(n(s.logits), n(s.draft_logits), before["tokens"], n(s.row_start), n(s.temperature), n(s.ua), n(s.us), ROWS, want["seq_len"])
        assert n(s.kept).tolist() == kept
        assert [a for a, w in zip(n(s.out).tolist(), out) if w is not None] == [w for w in out if w is not None]
        assert n(s.base).tolist() == (before["base"] + np.array(kept)).tolist()
        for r in range(N):
            if before["new"][r] and not want["seq_len"][r]:
                refusals += 1
                refused_before.add(r)
                a, b = want["row_start"][r:r + 2]
                assert kept[r] == 0 and n(s.base)[r] == before["base"][r] and n(s.held)[r] == before["held"][r]
                assert (n(s.out)[a:b] == -1).all() and (n(s.z)[a:b] == 0).all()
            elif r in refused_before and kept[r]:
                went_on.add(r)
        s.advance()
    assert refusals > 3 and went_on                                     # the pool is made for both


def test_steps_with_refused_requests_from_a_graph(k):
    want, eager = Server(k, 2, N_PAGES), []
    for step in range(STEPS):
        want.leave(step)
        want.forward()
        want.advance()
        eager.append(want.state())
    s = Server(k, 2, N_PAGES)
    first = {name: t.clone() for name, t in vars(s).items() if torch.is_tensor(t)}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.forward()                                                                     # warm-up of what is not ours
        s.advance()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.forward()
        s.advance()
    for name, t in first.items():
        getattr(s, name).copy_(t)
    for step in range(STEPS):
        s.leave(step)
        g.replay()
        torch.cuda.synchronize()
        for got, w in zip(s.state(), eager[step]):
            assert torch.equal(got.view(torch.uint8), w.view(torch.uint8)), step


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("with_draft", [True, False])
def test_verification_of_refused_requests(k, dtype, with_draft):
    rng = np.random.default_rng(7)
    new, vocab = [3, 1, 0, 4, 2, 5, 1, 3, 2], 700
    n, rows = len(new), sum(new)
    start = np.concatenate([[0], np.cumsum(new)])
    target, draft = (rng.standard_normal((rows, vocab)).astype(dtype) * 2 for _ in range(2))
    draft = draft if with_draft else None
    tokens, temperature = rng.integers(0, vocab, rows), np.where(rng.random(n) < 0.4, 0.0, 1.0).astype(np.float32)
    ua, us, lens = rng.random(rows).astype(np.float32) * 0.3, rng.random(n).astype(np.float32), rng.integers(0, 90, n)
    up = lambda a: None if a is None else torch.from_numpy(a).cuda()                    # noqa: E731
    for seq in (np.where(np.arange(n) % 2, 0, lens + new), np.zeros(n, int), lens + new + 1, None):
        want, kept = po.verify(target, draft, tokens, start, temperature, ua, us, rows, seq)
        got_kept, out, after = i32([-7] * n), i32([-7] * rows), i32(lens)
        ws = torch.full((k.kvpr_verify_workspace_bytes(n, rows, vocab),), 0xFF, dtype=torch.uint8, device="cuda")
        k.kvpr_verify_step(up(target), up(draft), k.KVPR_F16 if dtype == np.float16 else k.KVPR_F32, vocab, vocab, vocab, i32(tokens), i32(start),
                           None if seq is None else i32(seq), None, n, rows, up(temperature), up(ua), up(us), after, after, got_kept, out, ws, ws.numel())
        torch.cuda.synchronize()
        assert got_kept.tolist() == kept and out.tolist() == want
        assert after.tolist() == (lens + np.array(kept)).tolist()
