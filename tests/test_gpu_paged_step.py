"""Steps of a ragged batch as they are used: plan, projection, append, attention, output logits, verification, and the next plan from
what was kept.  Each stage against the oracle on its own inputs, and the same steps replayed from a graph, bit for bit."""
import numpy as np
import pytest
import torch

from oracle import kvpr_paged_oracle as po
from paged_testlib import i32

pytestmark = pytest.mark.gpu

VOCAB, H, HEADS, KV, D, PAGE, N, M, STEPS = 640, 256, 4, 2, 64, 16, 5, 3, 5
ROWS, COLS, WIDTH, N_PAGES = N * M, (HEADS + 2 * KV) * D, 6, 40


@pytest.fixture(scope="module")
def k():
    import paper_2411_17089_amd as k
    return k


class Server:
    """One attention layer between an embedding and an output matrix, N requests, a certain token and M - 1 drafts each a step."""

    def __init__(self, k, seed):
        self.k = k
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device="cuda") * scale).half()     # noqa: E731
        self.emb, self.wqkv, self.wlm = normal(VOCAB, H), normal(COLS, H, scale=0.08), normal(VOCAB, HEADS * D, scale=0.3)
        self.rope = torch.from_numpy(k.kvpr_rope_table(WIDTH * PAGE, D)).cuda()
        self.desc = k.make_paged_desc(HEADS, KV, D, PAGE, N_PAGES, WIDTH)
        self.pages = torch.zeros((N_PAGES, k.kvpr_page_bytes(self.desc)), dtype=torch.uint8, device="cuda")
        self.base, self.new = i32([0] * N), i32([M] * N)
        self.held, self.table = i32([0] * N), torch.full((N, WIDTH), -1, dtype=torch.int32, device="cuda")
        self.free, self.count = torch.randperm(N_PAGES, generator=g, device="cuda").int(), i32([N_PAGES])
        z = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype, device="cuda")                      # noqa: E731
        self.row_start, self.seq_len, self.slots, self.positions, self.refused = z(N + 1), z(N), z(ROWS), z(ROWS), z(1)
        self.tokens = torch.randint(0, VOCAB, (ROWS,), generator=g, device="cuda", dtype=torch.int32)
        self.qkv, self.q, self.z = (z(ROWS, c, dtype=torch.float16) for c in (COLS, HEADS * D, HEADS * D))
        self.logits, self.draft_logits = z(ROWS, VOCAB, dtype=torch.float32), z(ROWS, VOCAB, dtype=torch.float32)
        self.kept, self.out = z(N), z(ROWS)
        self.temperature = torch.tensor([0.0, 0.7, 1.0, 3.0, 0.0], device="cuda")
        self.ws = z(k.kvpr_paged_attention_workspace_bytes(self.desc, N, ROWS, M, WIDTH * PAGE), dtype=torch.uint8)
        self.ws_v = z(k.kvpr_verify_workspace_bytes(N, ROWS, VOCAB), dtype=torch.uint8)
        # what the draft model would give: drafts and their logits of every step, and the random numbers
        self.drafts = torch.randint(0, VOCAB, (STEPS, N, M - 1), generator=g, device="cuda", dtype=torch.int32)
        self.guesses = torch.randn((STEPS, ROWS, VOCAB), generator=g, device="cuda")
        self.u = torch.rand((STEPS, ROWS + N), generator=g, device="cuda")
        self.step_no = torch.zeros(1, dtype=torch.int64, device="cuda")

    def plan(self):
        k = self.k
        k.kvpr_paged_plan(self.desc, self.base, self.new, N, self.table, self.held, self.held, self.free, self.count, self.count, ROWS, self.row_start,
                          self.seq_len, self.slots, self.positions, self.refused)

    def layer(self):
        k = self.k
        x = self.emb[self.tokens.long()]
        k.kvpr_recompute_gemm(x, self.wqkv, None, self.qkv, ROWS, COLS, H, COLS)
        k.kvpr_paged_append(self.desc, self.qkv, COLS, self.slots, self.positions, ROWS, self.rope, self.rope.shape[0], self.q, HEADS * D, self.pages)
        k.kvpr_paged_attention(self.desc, self.q, k.KVPR_F16, HEADS * D, self.pages, self.table, self.row_start, self.seq_len, N, ROWS, M, WIDTH * PAGE,
                               self.z, HEADS * D, self.ws, self.ws.numel())
        k.kvpr_token_gemm(self.z, self.wlm, None, self.logits, None, ROWS, VOCAB, HEADS * D, VOCAB, VOCAB)

    def verify(self):
        k = self.k
        u = self.u.index_select(0, self.step_no)[0]
        self.ua, self.us = u[:ROWS].contiguous(), u[ROWS:].contiguous()
        self.draft_logits.copy_(self.guesses.index_select(0, self.step_no)[0])
        k.kvpr_verify_drafts(self.logits, self.draft_logits, k.KVPR_F32, VOCAB, VOCAB, VOCAB, self.tokens, self.row_start, N, ROWS, self.temperature,
                             self.ua, self.us, self.base, self.base, self.kept, self.out, self.ws_v, self.ws_v.numel())

    def advance(self):
        last = self.out.view(N, M).gather(1, (self.kept.long() - 1)[:, None])
        self.tokens.copy_(torch.cat([last, self.drafts.index_select(0, self.step_no)[0]], 1).reshape(-1))
        self.step_no.add_(1).remainder_(STEPS)

    def step(self):
        self.plan()
        self.layer()
        self.verify()
        self.advance()

    def state(self):
        return [t.clone() for t in (self.base, self.held, self.table, self.free, self.count, self.pages, self.tokens, self.out, self.kept, self.z, self.logits)]


def test_stages_of_steps_in_a_row(k):
    s = Server(k, 1)
    n = lambda t: t.cpu().numpy()                                                       # noqa: E731
    for step in range(STEPS):
        before = {name: n(getattr(s, name)).copy() for name in ("base", "held", "table", "free", "count", "pages", "tokens")}
        s.plan()
        s.layer()
        s.verify()
        torch.cuda.synchronize()
        want = po.plan(before["base"], [M] * N, before["held"], before["table"], before["free"], int(before["count"][0]), PAGE, ROWS, N_PAGES)
        assert want["refused"] == 0
        for name, got in (("table", s.table), ("free", s.free), ("held", s.held), ("count", s.count), ("row_start", s.row_start), ("seq_len", s.seq_len),
                          ("slots", s.slots), ("positions", s.positions)):
            assert np.array_equal(n(got).ravel(), np.asarray(want[name]).ravel()), (step, name)
        heads = n(s.qkv).reshape(ROWS, -1, D)
        q, kk = (po.rotate(a, n(s.rope), want["positions"]).astype(np.float16) for a in (heads[:, :HEADS], heads[:, HEADS:HEADS + KV]))
        pages = before["pages"].copy()
        for i in range(ROWS):
            po.store(pages, int(want["slots"][i]), kk[i], heads[i, HEADS + KV:], PAGE)
        assert np.array_equal(n(s.pages), pages) and np.array_equal(n(s.q), q.reshape(ROWS, -1))
        z, tol, done = po.attention(n(s.q), pages, n(s.table), n(s.row_start), n(s.seq_len), HEADS, KV, D, PAGE, ROWS)
        assert done.all() and (np.abs(n(s.z).astype(np.float64) - z) <= tol).all(), step
        out, kept = po.verify(n(s.logits), n(s.draft_logits), before["tokens"], n(s.row_start), n(s.temperature), n(s.ua), n(s.us), ROWS)
        assert n(s.out).tolist() == out and n(s.kept).tolist() == kept
        assert n(s.base).tolist() == (before["base"] + np.array(kept)).tolist()
        s.advance()


def test_steps_from_a_graph(k):
    """Three graphs of a step that share every buffer, replayed in turn with eager work between, against the same steps run eagerly."""
    want = Server(k, 2)
    eager = []
    for _ in range(STEPS):
        want.step()
        eager.append(want.state())
    s = Server(k, 2)
    first = {name: t.clone() for name, t in vars(s).items() if torch.is_tensor(t)}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.step()                                                                        # warm-up of what is not ours
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(3):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.step()
        graphs.append(g)
    for name, t in first.items():
        getattr(s, name).copy_(t)
    noise = torch.randn(512, 512, device="cuda")
    for i in range(STEPS):
        graphs[i % 3].replay()
        noise = (noise @ noise).clamp_(-1, 1)
        torch.cuda.synchronize()
        for got, w in zip(s.state(), eager[i]):
            assert torch.equal(got.view(torch.uint8), w.view(torch.uint8)), i


def test_two_streams_at_once(k):
    """Two servers with buffers of their own, their steps enqueued in turn on two streams."""
    alone = []
    for seed in (3, 4):
        s = Server(k, seed)
        for _ in range(STEPS):
            s.step()
        alone.append(s.state())
    both, streams = [Server(k, 3), Server(k, 4)], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(STEPS):
        for s, st in zip(both, streams):
            with torch.cuda.stream(st):
                s.step()
    torch.cuda.synchronize()
    for s, want in zip(both, alone):
        for got, w in zip(s.state(), want):
            assert torch.equal(got.view(torch.uint8), w.view(torch.uint8))
