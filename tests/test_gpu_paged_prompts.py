"""Steps in which some requests bring prompt chunks and others drafts: each stage against the oracle on its own inputs."""
import numpy as np
import pytest
import torch

from oracle import kvpr_paged_oracle as po
from paged_testlib import i32

pytestmark = pytest.mark.gpu

VOCAB, H, HEADS, KV, D, PAGE, WIDTH, N_PAGES = 320, 128, 8, 2, 64, 16, 8, 16
COLS = (HEADS + 2 * KV) * D
# of each step and request: (prompt tokens, drafts).  Request 0 has a prompt of 45 + 1 tokens in three chunks; request 1 decodes; request 2 comes
# later, with drafts right behind its prompt; request 3 finds no page in the first two steps
STEPS = [[(20, 0), (5, 2), (0, 0), (90, 0)],
         [(20, 0), (0, 3), (0, 0), (90, 0)],
         [(6, 0), (0, 1), (30, 2), (17, 0)],
         [(0, 2), (0, 0), (0, 4), (0, 1)],
         [(0, 3), (0, 2), (0, 1), (0, 2)]]


@pytest.fixture(scope="module")
def k():
    import paper_2411_17089_amd as k
    return k


@pytest.mark.parametrize("seed", [1, 2])
@pytest.mark.parametrize("with_draft", [True, False])
def test_prompts_and_drafts_in_one_step(k, seed, with_draft):
    rng = np.random.default_rng(seed)
    N = 4
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()                    # noqa: E731
    n = lambda t: t.cpu().numpy()                                                       # noqa: E731
    emb, wqkv, wlm = (dev((rng.standard_normal(s) * c).astype(np.float16)) for s, c in (((VOCAB, H), 1), ((COLS, H), .1), ((VOCAB, HEADS * D), .3)))
    rope = k.kvpr_rope_table(WIDTH * PAGE, D)
    desc = k.make_paged_desc(HEADS, KV, D, PAGE, N_PAGES, WIDTH)
    pages = torch.zeros((N_PAGES, k.kvpr_page_bytes(desc)), dtype=torch.uint8, device="cuda")
    base, held, table = i32([0] * N), i32([0] * N), torch.full((N, WIDTH), -1, dtype=torch.int32, device="cuda")
    free, count = i32(rng.permutation(N_PAGES)), i32([N_PAGES - 8])
    temperature = np.array([0.0, 1.0, 0.8, 0.0], np.float32)
    last, asked = [None] * N, [0] * N
    for step, plan_of_step in enumerate(STEPS):
        if step == 2:
            count += 8                                                  # pages come back from elsewhere
        new = [p + d + (last[r] is not None) for r, (p, d) in enumerate(plan_of_step)]
        new = [m if p + d or last[r] is not None else 0 for r, ((p, d), m) in enumerate(zip(plan_of_step, new))]
        certain = [p + (last[r] is not None) for r, (p, d) in enumerate(plan_of_step)]
        rows = sum(new)
        tokens = np.concatenate([[t for t in [last[r]] if t is not None] + list(rng.integers(0, VOCAB, p + d)) for r, (p, d) in enumerate(plan_of_step)]).astype(np.int64)
        assert len(tokens) == rows
        before = {name: n(t).copy() for name, t in (("base", base), ("held", held), ("table", table), ("free", free), ("count", count), ("pages", pages))}
        z = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype, device="cuda")                      # noqa: E731
        row_start, seq_len, slots, positions, refused = z(N + 1), z(N), z(rows), z(rows), z(1)
        k.kvpr_paged_plan(desc, base, i32(new), N, table, held, held, free, count, count, rows, row_start, seq_len, slots, positions, refused)
        qkv, q, out_z = (z(rows, c, dtype=torch.float16) for c in (COLS, HEADS * D, HEADS * D))
        k.kvpr_recompute_gemm(emb[dev(tokens)], wqkv, None, qkv, rows, COLS, H, COLS)
        k.kvpr_paged_append(desc, qkv, COLS, slots, positions, rows, dev(rope), len(rope), q, HEADS * D, pages)
        ws = z(k.kvpr_paged_attention_workspace_bytes(desc, N, rows, max(new), WIDTH * PAGE), dtype=torch.uint8)
        k.kvpr_paged_attention(desc, q, k.KVPR_F16, HEADS * D, pages, table, row_start, seq_len, N, rows, max(new), WIDTH * PAGE, out_z, HEADS * D, ws, ws.numel())
        logits = z(rows, VOCAB, dtype=torch.float32)
        for a in range(0, rows, 64):                                    # the product takes 64 rows at most
            k.kvpr_token_gemm(out_z[a:], wlm, None, logits[a:], None, min(rows - a, 64), VOCAB, HEADS * D, VOCAB, VOCAB)
        draft = torch.randn((rows, VOCAB), device="cuda") if with_draft else None
        ua, us = rng.random(rows).astype(np.float32) * 0.2, rng.random(N).astype(np.float32)
        kept, out = i32([-7] * N), i32([-7] * rows)
        ws = z(k.kvpr_verify_workspace_bytes(N, rows, VOCAB), dtype=torch.uint8)
        k.kvpr_verify_step(logits, draft, k.KVPR_F32, VOCAB, VOCAB, VOCAB, i32(tokens), row_start, seq_len, i32(certain), N, rows, dev(temperature), dev(ua), dev(us),
                           base, base, kept, out, ws, ws.numel())
        torch.cuda.synchronize()
        want = po.plan(before["base"], new, before["held"], before["table"], before["free"], int(before["count"][0]), PAGE, rows, N_PAGES)
        assert want["refused"] == (1 if step < 2 else 0)
        for name, got in (("table", table), ("free", free), ("held", held), ("count", count), ("row_start", row_start), ("seq_len", seq_len), ("slots", slots),
                          ("positions", positions), ("refused", refused)):
            assert np.array_equal(n(got).ravel(), np.asarray(want[name]).ravel()), (step, name)
        heads = n(qkv).reshape(rows, -1, D)
        kk = po.rotate(heads[:, HEADS:HEADS + KV], rope, want["positions"]).astype(np.float16)
        stored = before["pages"].copy()
        for i in range(rows):
            if want["slots"][i] >= 0:
                po.store(stored, int(want["slots"][i]), kk[i], heads[i, HEADS + KV:], PAGE)
        assert np.array_equal(n(pages), stored)
        wz, tol, done = po.attention(n(q), stored, n(table), want["row_start"], want["seq_len"], HEADS, KV, D, PAGE, rows)
        assert (np.abs(n(out_z).astype(np.float64) - wz) <= tol)[done].all(), step
        w_out, w_kept = po.verify(n(logits), None if draft is None else n(draft), tokens, want["row_start"], temperature, ua, us, rows, want["seq_len"], certain)
        assert n(kept).tolist() == w_kept and n(out).tolist() == w_out
        assert n(base).tolist() == (before["base"] + np.array(w_kept)).tolist()
        for r, (p, d) in enumerate(plan_of_step):
            a = int(want["row_start"][r])
            if new[r] and want["seq_len"][r]:
                assert w_kept[r] >= max(certain[r], 1)
                assert w_out[a:a + certain[r] - 1] == tokens[a + 1:a + certain[r]].tolist()
                last[r] = w_out[a + w_kept[r] - 1]
                if (r, step) in ((0, 0), (0, 1)):                       # the prompt goes on: its next token is certain, not what the model says
                    last[r] = None
            asked[r] += w_kept[r]
    assert asked[0] >= 46 and min(asked) > 0


@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("with_draft", [True, False])
@pytest.mark.parametrize("vocab", [300, 9001])
def test_verification_with_certain_rows(k, dtype, with_draft, vocab):
    rng = np.random.default_rng(vocab)
    new = [3, 1, 0, 40, 2, 25, 1, 3, 9, 130]
    n, rows = len(new), sum(new)
    start = np.concatenate([[0], np.cumsum(new)])
    target = (rng.standard_normal((rows, vocab)) * 2).astype(dtype)
    draft = np.zeros_like(target)
    draft[1:] = target[:-1] + 0.2 * rng.standard_normal((rows - 1, vocab)).astype(dtype)
    tokens = (draft.astype(np.float64) + rng.gumbel(size=draft.shape)).argmax(-1)
    draft = draft if with_draft else None
    temperature = np.array([0, 1, 1, 0.7, 0, 1.2, 0, 1, 0.9, 1], np.float32)
    ua, us, lens = rng.random(rows).astype(np.float32), rng.random(n).astype(np.float32), rng.integers(0, 90, n)
    up = lambda a: None if a is None else torch.from_numpy(a).cuda()                    # noqa: E731
    for certain in ([3, 1, 0, 40, 1, 20, 1, 2, 1, 130], [0, -5, 7, 39, 2 ** 31 - 1, 1, 9, -2 ** 31, 8, 100], [1] * n):
        for seq in (None, np.where(np.arange(n) % 3 == 2, 0, lens + new)):
            for n_rows in (rows, rows - 60):                            # the last request's certain rows may pass the arrays' end
                want, kept = po.verify(target, draft, tokens, start, temperature, ua, us, n_rows, seq, certain)
                got_kept, out, after = i32([-7] * n), i32([-7] * rows), i32([-7] * n)
                ws = torch.full((k.kvpr_verify_workspace_bytes(n, n_rows, vocab),), 0xFF, dtype=torch.uint8, device="cuda")
                k.kvpr_verify_step(up(target), up(draft), k.KVPR_F16 if dtype == np.float16 else k.KVPR_F32, vocab, vocab, vocab, i32(tokens), i32(start),
                                   None if seq is None else i32(seq), i32(certain), n, n_rows, up(temperature), up(ua), up(us), i32(lens), after, got_kept, out,
                                   ws, ws.numel())
                torch.cuda.synchronize()
                assert got_kept.tolist() == kept and out.tolist()[:n_rows] == want and (out[n_rows:] == -7).all()
                assert after.tolist() == (lens + np.array(kept)).tolist()
