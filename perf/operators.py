"""What the operators for ragged batches over a paged 4-bit cache are measured on.

A server that holds the KV cache of many requests of different lengths in 4-bit pages, and lets a small model draft a few
tokens ahead, goes through four operators for each step: a plan (pages, row offsets, slots and positions of the new tokens
from the requests' lengths), the append of the new tokens' rows (rotation, packing, and reading slots back), the attention of
the new tokens over the pages, and the verification of the drafted tokens.  Head shapes, vocabularies and contexts are
those of the bench and the tests (widths 768 to 7168, vocabularies 32000 and 50272, contexts up to 4096) and, for shared
key/value heads and long contexts, generic ones.

A case is a dict of plain values; "kind" says which operator it takes.  The requests' lengths follow from the case alone,
everything else from the seed.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

GROUP = 64                      # columns that share one scale and minimum
ROPE_BASE = 10000.0


def listed():
    return [
        # one verification step of eight requests at the bench's context: last token and up to four drafts each
        {"name": "plan_8_verify", "kind": "plan", "mix": 1, "n": 8, "page": 16, "base_lo": 700, "base_hi": 1400, "new_lo": 1, "new_hi": 5, "prompts": 0, "prompt": 0},
        # a busy server with chunked prompts: 512 requests, some idle, 24 with a prompt chunk of up to 2047 tokens
        {"name": "plan_512_prompts", "kind": "plan", "mix": 2, "n": 512, "page": 16, "base_lo": 16, "base_hi": 16000, "new_lo": 0, "new_hi": 6, "prompts": 24, "prompt": 2047},
        # a decode step's rows of the rotary 4096-wide family, batch 32, four drafts each
        {"name": "append_rope_4096_r160", "kind": "append", "mix": 3, "rows": 160, "pad": 0, "heads": 32, "kv_heads": 32, "d": 128, "page": 16, "rope": True},
        # prompts of the widest family, an odd number of rows and some padding behind them
        {"name": "append_7168_r8191", "kind": "append", "mix": 4, "rows": 8191, "pad": 65, "heads": 56, "kv_heads": 56, "d": 128, "page": 32, "rope": False},
        # the smallest attention: one short sequence of the 768-wide family, one token
        {"name": "attention_768_b1_s97", "kind": "attention", "mix": 5, "n": 1, "heads": 12, "kv_heads": 12, "d": 64, "page": 16, "base_lo": 96, "base_hi": 96, "new_lo": 1, "new_hi": 1, "q": "f16"},
        # the bench's decode batch: 32 sequences around 1024 positions, one token each, no shared heads
        {"name": "attention_4096_b32_s1024", "kind": "attention", "mix": 6, "n": 32, "heads": 32, "kv_heads": 32, "d": 128, "page": 16, "base_lo": 900, "base_hi": 1100, "new_lo": 1, "new_hi": 1, "q": "f32"},
        # long contexts with shared key/value heads, five rows a request (last token and four drafts)
        {"name": "attention_gqa8_b4_s32768", "kind": "attention", "mix": 7, "n": 4, "heads": 64, "kv_heads": 8, "d": 128, "page": 64, "base_lo": 20000, "base_hi": 32763, "new_lo": 5, "new_hi": 5, "q": "f16"},
        # a ragged batch: 64 requests from a few positions to 8192, one to eight rows, groups of five heads
        {"name": "attention_gqa5_ragged", "kind": "attention", "mix": 8, "n": 64, "heads": 40, "kv_heads": 8, "d": 128, "page": 32, "base_lo": 1, "base_hi": 8192, "new_lo": 1, "new_hi": 8, "q": "f32"},
        # prompt chunks over what is cached already
        {"name": "attention_chunk_2x1000", "kind": "attention", "mix": 9, "n": 2, "heads": 32, "kv_heads": 8, "d": 128, "page": 64, "base_lo": 2000, "base_hi": 4096, "new_lo": 1000, "new_hi": 1000, "q": "f16"},
        # interactive: one request, four drafts of a smaller model
        {"name": "verify_1x5_v50272", "kind": "verify", "mix": 10, "n": 1, "new_lo": 5, "new_hi": 5, "vocab": 50272, "type": "f32", "draft": True},
        # a batch of 64, one to six rows each, logits kept in 16 bits
        {"name": "verify_64_v32000_f16", "kind": "verify", "mix": 11, "n": 64, "new_lo": 1, "new_hi": 6, "vocab": 32000, "type": "f16", "draft": True},
        # drafts that a lookup made (no probabilities of their own), a generic large vocabulary of odd size
        {"name": "verify_48_v131071_lookup", "kind": "verify", "mix": 12, "n": 48, "new_lo": 2, "new_hi": 8, "vocab": 131071, "type": "f32", "draft": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _span(rng, name, most):
    lo, hi = sorted([_log(rng, 1, most), _log(rng, 1, most)])
    return {name + "_lo": lo, name + "_hi": hi}


def draw(rng):
    """One more case of the listed ranges, no dearer than the largest listed one of its kind."""
    kind = rng.choice(["plan", "append", "attention", "attention", "attention", "verify", "verify"])
    case = {"kind": kind, "mix": rng.randrange(1, 1 << 30)}
    heads, kv_heads, d = rng.choice([(12, 12, 64), (32, 32, 128), (40, 40, 128), (56, 56, 128), (32, 8, 128), (40, 8, 128), (64, 8, 128), (28, 4, 128), (16, 2, 64)])
    if kind == "plan":
        n = _log(rng, 1, 512)
        prompts = min(n, rng.choice([0, 0, 1, rng.randint(1, 24)]))
        return {**case, "n": n, "page": rng.choice([16, 32, 64, 128]), **_span(rng, "base", 16000), "new_lo": rng.randint(0, 1), "new_hi": rng.randint(1, 8),
                "prompts": prompts, "prompt": _log(rng, 8, 2047) if prompts else 0}
    if kind == "append":
        rows = min(_log(rng, 1, 8191), 8191 * 56 * 128 // (heads * d))
        return {**case, "rows": rows, "pad": rng.choice([0, 0, rng.randint(1, 70)]), "heads": heads, "kv_heads": kv_heads, "d": d,
                "page": rng.choice([16, 32, 64, 128]), "rope": rng.random() < 0.5}
    if kind == "attention":
        if rng.random() < 0.2:
            n, new = rng.randint(1, 3), _log(rng, 16, 1000)
            spans = {**_span(rng, "base", 4096), "new_lo": new, "new_hi": new}
            heads, kv_heads, d = rng.choice([(32, 8, 128), (32, 32, 128), (12, 12, 64)])
        else:
            n = _log(rng, 1, 64)
            most = max(64, min(32768, 64 * 8192 * 8 // (n * kv_heads)))
            spans = {**_span(rng, "base", most), **_span(rng, "new", 8)}
        return {**case, "n": n, "heads": heads, "kv_heads": kv_heads, "d": d, "page": rng.choice([16, 32, 64, 128]), **spans,
                "q": rng.choice(["f16", "f32"])}
    vocab = rng.choice([32000, 50272, 131071, _log(rng, 500, 131071)])
    most = max(1, min(64, 48 * 5 * 131071 // (9 * vocab)))
    return {**case, "n": _log(rng, 1, most), **_span(rng, "new", 8), "vocab": vocab, "type": rng.choice(["f16", "f32"]),
            "draft": rng.random() < 0.6}


def _lengths(case):
    """(cached positions, new tokens) of each request."""
    rng = random.Random(case["mix"])
    base = [_log(rng, case["base_lo"], case["base_hi"]) if "base_lo" in case else 0 for _ in range(case["n"])]
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["n"])]
    for r in rng.sample(range(case["n"]), case.get("prompts", 0)):
        base[r], new[r] = 0, rng.randint((case["prompt"] + 1) // 2, case["prompt"])
    return base, new


def _starts(new):
    return [0] + list(np.cumsum(new, dtype=np.int64).tolist())


def work(case):
    kind = case["kind"]
    if kind == "plan":
        base, new = _lengths(case)
        taken = sum(-(-m // case["page"]) for m in new)
        return {"bytes": 4 * (6 * case["n"] + 2 * taken + 2 * sum(new)), "flops": 0}
    if kind == "append":
        q, kv = case["heads"] * case["d"], 2 * case["kv_heads"] * case["d"]
        a_row = (q if case["rope"] else 0) * 4 + kv * 2 + 2 * (kv * 9 // 16) + kv * 2
        return {"bytes": case["rows"] * a_row, "flops": 0}
    if kind == "attention":
        base, new = _lengths(case)
        cache = sum(b + m for b, m in zip(base, new)) * 2 * case["kv_heads"] * case["d"] * 9 // 16
        seen = sum(m * b + m * (m + 1) // 2 for b, m in zip(base, new))
        width = case["heads"] * case["d"]
        return {"bytes": cache + sum(new) * width * ((2 if case["q"] == "f16" else 4) + 2), "flops": 4 * seen * width}
    new = _lengths(case)[1]
    rows = sum(new) + (sum(new) - case["n"] if case["draft"] else 0)
    return {"bytes": rows * case["vocab"] * (2 if case["type"] == "f16" else 4), "flops": 0}


# ---- the 4-bit pages in plain operations ----
# A page holds `page` positions; for each key/value head one block of page * 9 d / 8 bytes:
#   key codes    [page][d / 2 bytes]: the row's words of 8 columns, word 4 s + g stored at place g * (d / 32) + s
#   value codes  [page / 4][d / 2][4]: the bytes of four positions side by side; byte 32 u + 2 m + w of a row stored at
#                place m * (d / 32) + 2 u + w
#   key pairs    [page][d / 64] of (scale, minimum) in float16, then the same of the values
# Column 2 k of a row is in the low four bits of its byte k, column 2 k + 1 in the high ones.

def _codes(x):
    """x [..., c] float16 -> codes [..., c] uint8, scale and minimum [..., c / 64] float16."""
    g = x.float().unflatten(-1, (-1, GROUP))
    mn, mx = g.amin(-1), g.amax(-1)
    scale = ((mx - mn) / 15.0).half()
    s = scale.float()[..., None]
    code = torch.where(s > 0, torch.round((g - mn[..., None]) / torch.where(s > 0, s, 1.0)), 0.0).clamp_(0, 15)
    return code.to(torch.uint8).flatten(-2), scale, mn.half()


def _values(codes, scale, mn):
    v = codes.float().unflatten(-1, (-1, GROUP)) * scale.float()[..., None] + mn.float()[..., None]
    return v.flatten(-2)


def _pack(k, v):
    """k, v [pages, heads, page, d] float16 -> pages [pages, heads * page * 9 d / 8] uint8."""
    n, h, p, d = k.shape
    parts, pairs = [], []
    for x, is_key in ((k, True), (v, False)):
        c, scale, mn = _codes(x)
        b = c[..., 0::2] | (c[..., 1::2] << 4)                                            # [n, h, p, d / 2]
        if is_key:
            b = b.reshape(n, h, p, d // 32, 4, 4).transpose(3, 4)
        else:
            b = b.reshape(n, h, p // 4, 4, d // 64, 16, 2).permute(0, 1, 2, 5, 4, 6, 3)
        parts.append(b.reshape(n, h, -1))
        pairs.append(torch.stack([scale, mn], -1).reshape(n, h, -1).view(torch.uint8))
    return torch.cat(parts + pairs, -1).reshape(n, -1)


def _unpack(pages, h, p, d):
    """pages [pages, bytes] -> (codes, scale, mn) of k and of v, [pages, heads, page, ...]."""
    n = pages.shape[0]
    block = pages.reshape(n, h, -1)
    half, pair = p * d // 2, p * (d // 64) * 4
    out = []
    for i, is_key in ((0, True), (1, False)):
        b = block[..., i * half:(i + 1) * half]
        if is_key:
            b = b.reshape(n, h, p, 4, d // 32, 4).transpose(3, 4).reshape(n, h, p, d // 2)
        else:
            b = b.reshape(n, h, p // 4, 16, d // 64, 2, 4).permute(0, 1, 2, 6, 4, 3, 5).reshape(n, h, p, d // 2)
        m = block[..., 2 * half + i * pair:2 * half + (i + 1) * pair].contiguous().view(torch.float16).reshape(n, h, p, d // 64, 2)
        out.append((torch.stack([b & 15, b >> 4], -1).flatten(-2), m[..., 0], m[..., 1]))
    return out


def _random_pages(g, n, h, p, d):
    """Pages of a cache of N(0, 1) keys and values, a part of the keys' columns larger than the rest, as keys have them."""
    pages = torch.empty((n, h * p * 9 * d // 8), dtype=torch.uint8, device="cuda")
    gain = torch.where(torch.rand((h, 1, d), generator=g, device="cuda") < 0.05, 3.0, 0.9)
    at_once = max(1, (1 << 26) // (h * p * d))
    for a in range(0, n, at_once):
        b = min(n, a + at_once)
        k = (torch.randn((b - a, h, p, d), generator=g, device="cuda") * gain).half()
        v = torch.randn((b - a, h, p, d), generator=g, device="cuda").half()
        pages[a:b] = _pack(k, v)
    return pages


# ---- inputs ----

def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _rope_table(n, d):
    """float32 (cos, sin) of position * base^(-2 i / d), from angles in 64 bits."""
    angle = np.arange(n, dtype=np.float64)[:, None] * ROPE_BASE ** (-2.0 * np.arange(d // 2) / d)
    return torch.from_numpy(np.stack([np.cos(angle), np.sin(angle)], -1).astype(np.float32)).cuda()


def _prepare_plan(st, case, g):
    base, new = _lengths(case)
    n, p = case["n"], case["page"]
    # pages that a request holds: what its positions need, here and there some that rejected drafts left behind
    held = [-(-b // p) + (r % 7 == 3) * 2 for r, b in enumerate(base)]
    need = [-(-(b + m) // p) for b, m in zip(base, new)]
    width = max(max(held), max(need)) + 3
    take = sum(max(0, b - a) for a, b in zip(held, need))
    spare = take + 17
    n_pages = sum(held) + spare
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    table = np.full((n, width), -1, dtype=np.int64)
    at = 0
    for r, m in enumerate(held):
        table[r, :m] = np.arange(at, at + m)
        at += m
    ids = torch.from_numpy(table).cuda()
    st["table"] = torch.where(ids >= 0, order[ids.clamp(min=0)], -1).int().contiguous()
    st["free"] = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    st["free"][:spare] = order[at:]
    st.update(base=_ints(base), new=_ints(new), held=_ints(held), count=_ints([spare]), max_rows=sum(new) + 13, n_pages=n_pages, width=width)
    i32 = lambda k: torch.zeros(k, dtype=torch.int32, device="cuda")                    # noqa: E731
    st.update(held_out=i32(n), count_out=i32(1), row_start=i32(n + 1), seq_len=i32(n), slots=i32(st["max_rows"]),
              positions=i32(st["max_rows"]), refused=i32(1))


def _prepare_append(st, case, g):
    rows, total, p, d = case["rows"], case["rows"] + case["pad"], case["page"], case["d"]
    width = (case["heads"] + 2 * case["kv_heads"]) * d
    rng = random.Random(case["mix"])
    # requests of 1 to 300 rows at consecutive positions, page by page
    slots, positions, n_pages = [], [], rows // p + rows + 8
    page_ids = list(range(n_pages))
    rng.shuffle(page_ids)
    while len(slots) < rows:
        m = min(rng.choice([1, 3, 5, rng.randint(1, 300)]), rows - len(slots))
        start = rng.randint(0, 3000)
        page = -1
        for t in range(start, start + m):
            if page < 0 or t % p == 0:
                page = page_ids.pop()
            slots.append(page * p + t % p)
            positions.append(t)
    used = sorted({s // p for s in slots})
    small = {page: i for i, page in enumerate(rng.sample(used, len(used)))}              # only pages that are in use are kept
    slots = [small[s // p] * p + s % p for s in slots]
    st.update(total=total, n_pages=len(used), slots=_ints(slots + [-1] * case["pad"]), positions=_ints(positions + [0] * case["pad"]))
    st["qkv"] = torch.randn((total, width), generator=g, device="cuda", dtype=torch.float16)
    st["pages"] = torch.zeros((len(used), case["kv_heads"] * p * 9 * d // 8), dtype=torch.uint8, device="cuda")
    st["back"] = torch.zeros((total, 2 * case["kv_heads"] * d), dtype=torch.float16, device="cuda")
    if case["rope"]:
        st["rope"] = _rope_table(4096, d)
        st["q_out"] = torch.zeros((total, case["heads"] * d), dtype=torch.float16, device="cuda")


def _prepare_attention(st, case, g):
    base, new = _lengths(case)
    p, d, h = case["page"], case["d"], case["kv_heads"]
    lens = [b + m for b, m in zip(base, new)]
    need = [-(-L // p) for L in lens]
    n_pages, width = sum(need) + 5, max(need) + 2
    st["pages"] = _random_pages(g, n_pages, h, p, d)
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    st["table"] = torch.full((case["n"], width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for r, m in enumerate(need):
        st["table"][r, :m] = order[at:at + m]
        at += m
    rows = sum(new)
    q = torch.randn((rows, case["heads"] * d), generator=g, device="cuda") * 1.5
    st["q"] = q.half() if case["q"] == "f16" else q
    st["z"] = torch.zeros((rows, case["heads"] * d), dtype=torch.float16, device="cuda")
    st.update(lens=lens, new_host=new, row_start=_ints(_starts(new)), seq_len=_ints(lens), n_pages=n_pages, width=width, rows=rows)


def _prepare_verify(st, case, g):
    new = _lengths(case)[1]
    n, vocab, rows = case["n"], case["vocab"], sum(new)
    dtype = torch.float16 if case["type"] == "f16" else torch.float32
    start = _starts(new)
    # a few likely tokens above a long tail; the draft model sees it a little differently
    logits = torch.randn((rows, vocab), generator=g, device="cuda") * 1.8
    top = torch.randint(0, vocab, (rows, 12), generator=g, device="cuda")
    logits.scatter_add_(1, top, torch.rand((rows, 12), generator=g, device="cuda") * 9.0 + 4.0)
    temperature = torch.tensor([0.0 if r % 5 == 4 else 0.6 + 0.1 * (r % 6) for r in range(n)], dtype=torch.float32, device="cuda")
    owner = torch.repeat_interleave(torch.arange(n, device="cuda"), _ints(new).long())
    t_row = temperature[owner]
    # row i of a request holds the logits after its token i; the draft row of token i + 1 is made from the same context
    guess = logits + torch.randn((rows, vocab), generator=g, device="cuda") * 0.7
    draft = torch.zeros_like(guess)
    draft[1:] = guess[:-1]
    t_safe = torch.where(t_row > 0, t_row, 0.05)
    noise = -torch.log(-torch.log(torch.rand((rows, vocab), generator=g, device="cuda").clamp_(1e-20, 1 - 1e-7)))
    st["tokens"] = (draft / t_safe[:, None] + noise).argmax(-1).int()
    del noise, guess
    st["target"] = logits.to(dtype)
    if case["draft"]:
        st["draft"] = draft.to(dtype)
    st["u_accept"] = torch.rand((rows,), generator=g, device="cuda")
    st["u_sample"] = torch.rand((n,), generator=g, device="cuda")
    st.update(temperature=temperature, row_start=_ints(start), rows=rows, most=max(new), len_in=torch.randint(1, 4000, (n,), generator=g, device="cuda", dtype=torch.int32))
    i32 = lambda k: torch.zeros(k, dtype=torch.int32, device="cuda")                    # noqa: E731
    st.update(len_out=i32(n), kept=i32(n), out=i32(rows))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = {"case": case}
    {"plan": _prepare_plan, "append": _prepare_append, "attention": _prepare_attention, "verify": _prepare_verify}[case["kind"]](st, case, g)
    if own:
        import paper_2411_17089_amd as kv
        if case["kind"] == "verify":
            st["ws"] = torch.zeros(kv.kvpr_verify_workspace_bytes(case["n"], st["rows"], case["vocab"]), dtype=torch.uint8, device="cuda")
        else:
            st["desc"] = kv.make_paged_desc(case.get("heads", 1), case.get("kv_heads", 1), case.get("d", 128), case["page"], st["n_pages"], st.get("width", 1))
        if case["kind"] == "attention":
            st["ws"] = torch.zeros(kv.kvpr_paged_attention_workspace_bytes(st["desc"], case["n"], st["rows"], max(st["new_host"]), max(st["lens"])),
                                   dtype=torch.uint8, device="cuda")
    return st


# ---- plain forms ----

def _plain_plan(st, case):
    n, p, width, n_pages = case["n"], case["page"], st["width"], st["n_pages"]
    base, new, held = st["base"].long(), st["new"].long(), st["held"].long()
    need = (base + new + p - 1) // p
    col = torch.arange(width, device="cuda")[None]
    gives = (col >= need[:, None]) & (col < held[:, None])
    rank = torch.cumsum(gives.flatten(), 0) - 1
    count = st["count"].long()
    free = torch.cat([st["free"], st["free"].new_zeros(1)])
    place = torch.where(gives.flatten(), count + rank, n_pages)
    free.scatter_(0, place, torch.where(gives.flatten(), st["table"].flatten(), 0))
    avail = count + gives.sum()
    takes = torch.where(need <= width, (need - held).clamp(min=0), 0)
    after = torch.cumsum(takes, 0)
    granted = (need <= width) & ((takes == 0) | (after <= avail))
    left = avail - torch.where(granted, takes, 0).sum()
    got = (col >= held[:, None]) & (col < need[:, None]) & granted[:, None]
    source = (avail - 1 - ((after - takes)[:, None] + col - held[:, None])).clamp(0, n_pages - 1)
    table = torch.where(got, free[source], st["table"])
    row_start = torch.cat([torch.zeros(1, dtype=torch.long, device="cuda"), torch.cumsum(new, 0)])
    t = torch.arange(st["max_rows"], device="cuda")
    r = torch.searchsorted(row_start[1:].contiguous(), t, right=True).clamp(max=n - 1)
    real = t < row_start[-1]
    position = torch.where(real, base[r] + t - row_start[r], 0)
    page = table[r, (position // p).clamp(max=width - 1)].long()
    slot = torch.where(real & granted[r], page * p + position % p, -1)
    return {"table": table, "held": torch.where(granted, need, held).int(), "free": free[:-1], "count": left.int(), "row_start": row_start.int(),
            "seq_len": torch.where(granted, base + new, 0).int(), "slots": slot.int(), "positions": position.int(), "refused": (~granted).sum().int().reshape(1)}


def _to_half(x):
    """float64 -> float16 in one rounding: to float32 with an odd last bit where that is inexact, which keeps the second rounding right."""
    f = x.float()
    rest = x - f.double()
    bits = f.view(torch.int32)
    step = torch.where((rest > 0) == (f > 0), 1, -1).int()
    odd = torch.where((rest != 0) & (bits & 1 == 0), bits + step, bits)
    return odd.view(torch.float32).half()


def _rotate(x, table, positions):
    """x [rows, heads, d] float16; element i of a head goes with element i + d / 2."""
    cs = table[positions.long()].double()[:, None]
    a, b = x.double().chunk(2, -1)
    return _to_half(torch.cat([a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]], -1))


def _plain_append(st, case):
    heads, h, d, rows = case["heads"], case["kv_heads"], case["d"], case["rows"]
    x = st["qkv"].unflatten(-1, (-1, d))
    q, k, v = x[:, :heads], x[:, heads:heads + h], x[:, heads + h:]
    out = {}
    if case["rope"]:
        out["q"] = _rotate(q, st["rope"], st["positions"]).flatten(1)
        k = _rotate(k, st["rope"], st["positions"])
    there = (st["slots"] >= 0)[:, None]
    kv = torch.cat([k.flatten(1), v.flatten(1)], 1)
    out["rows"] = torch.where(there, _values(*_codes(kv)).half(), st["back"])
    return out


def _plain_attention(st, case):
    p, d, h = case["page"], case["d"], case["kv_heads"]
    group = case["heads"] // h
    z, at = [], 0
    for r, (L, m) in enumerate(zip(st["lens"], st["new_host"])):
        pages = st["pages"][st["table"][r, :-(-L // p)].long()]
        k, v = (_values(*x).transpose(0, 1).reshape(h, -1, d)[:, :L] for x in _unpack(pages, h, p, d))
        q = st["q"][at:at + m].float().reshape(m, h, group, d).permute(1, 2, 0, 3).reshape(h, group * m, d)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)
        hidden = torch.arange(L, device="cuda")[None] > torch.arange(L - m, L, device="cuda")[:, None]
        s = s.reshape(h, group, m, L).masked_fill_(hidden, -math.inf)
        s = torch.exp(s - s.amax(-1, keepdim=True))
        o = torch.matmul(s.reshape(h, group * m, L), v.contiguous()) / s.sum(-1).reshape(h, group * m, 1)
        z.append(o.reshape(h, group, m, d).permute(2, 0, 1, 3).reshape(m, -1))
        at += m
    return torch.cat(z).half()


def _shares(logits, t):
    """softmax(logits / t) in 64 bits."""
    x = logits.double()
    e = torch.exp((x - x.amax(-1, keepdim=True)) / t[:, None].double())
    return e / e.sum(-1, keepdim=True)


def _plain_verify(st, case):
    n, vocab, rows = case["n"], case["vocab"], st["rows"]
    start = st["row_start"].long()
    first, m = start[:-1], start[1:] - start[:-1]
    row = torch.arange(rows, device="cuda")
    owner = torch.searchsorted(start[1:].contiguous(), row, right=True)
    temperature = st["temperature"][owner]
    greedy = temperature <= 0
    t = torch.where(greedy, 1.0, temperature)
    token = st["tokens"].long()
    target = _shares(st["target"], t)
    best = st["target"].float().argmax(-1)
    before = (row - 1).clamp(min=0)                        # the row whose target distribution a draft is held against
    p = target[before, token]
    q = _shares(st["draft"], t)[row, token] if case["draft"] else torch.ones_like(p)
    good = torch.where(greedy, best[before] == token, st["u_accept"].double() * q < p)
    # accepted in a row from the first draft on
    i = torch.arange(1, st["most"] + 1, device="cuda")[None]
    at = (first[:, None] + i).clamp(max=rows - 1)
    run_on = (good[at] & (i < m[:, None])).long().cumprod(1)
    accepted = run_on.sum(1)
    last = first + accepted
    p = target[last]
    rejected = accepted < m - 1
    drafted = (last + 1).clamp(max=rows - 1)
    if case["draft"]:
        q = _shares(st["draft"][drafted], t[drafted])
    else:
        q = torch.zeros_like(p).scatter_(1, token[drafted][:, None], 1.0)
    rest = torch.where(rejected[:, None], (p - q).clamp(min=0), p)
    rest = torch.where(rest.sum(-1, keepdim=True) > 0, rest, p)
    summed = rest.cumsum(-1)
    pick = (summed > st["u_sample"].double()[:, None] * summed[:, -1:]).long().argmax(-1)
    pick = torch.where(greedy[last], best[last], pick)
    offset = row - first[owner]
    following = (row + 1).clamp(max=rows - 1)
    out = torch.where(offset < accepted[owner], token[following], torch.where(offset == accepted[owner], pick[owner], -1))
    return {"tokens": out.int(), "kept": (accepted + 1).int(), "len": st["len_in"] + (accepted + 1).int()}


# ---- the framework's calls ----

def _own(st, case):
    import paper_2411_17089_amd as kv
    kind = case["kind"]
    if kind == "plan":
        kv.kvpr_paged_plan(st["desc"], st["base"], st["new"], case["n"], st["table"], st["held"], st["held_out"], st["free"], st["count"], st["count_out"],
                           st["max_rows"], st["row_start"], st["seq_len"], st["slots"], st["positions"], st["refused"])
        return {"table": st["table"], "held": st["held_out"], "free": st["free"], "count": st["count_out"], "row_start": st["row_start"],
                "seq_len": st["seq_len"], "slots": st["slots"], "positions": st["positions"], "refused": st["refused"]}
    if kind == "append":
        rope = st.get("rope")
        kv.kvpr_paged_append(st["desc"], st["qkv"], st["qkv"].shape[1], st["slots"], st["positions"], st["total"], rope, 0 if rope is None else rope.shape[0],
                             st.get("q_out"), case["heads"] * case["d"], st["pages"])
        kv.kvpr_paged_read(st["desc"], st["pages"], st["slots"], st["total"], st["back"], st["back"].shape[1])
        return {**({"q": st["q_out"]} if case["rope"] else {}), "rows": st["back"]}
    if kind == "attention":
        width = case["heads"] * case["d"]
        kv.kvpr_paged_attention(st["desc"], st["q"], kv.KVPR_F16 if case["q"] == "f16" else kv.KVPR_F32, width, st["pages"], st["table"], st["row_start"],
                                st["seq_len"], case["n"], st["rows"], max(st["new_host"]), max(st["lens"]), st["z"], width, st["ws"], st["ws"].numel())
        return st["z"]
    kv.kvpr_verify_drafts(st["target"], st.get("draft"), kv.KVPR_F16 if case["type"] == "f16" else kv.KVPR_F32, case["vocab"], case["vocab"], case["vocab"], st["tokens"],
                          st["row_start"], case["n"], st["rows"], st["temperature"], st["u_accept"], st["u_sample"], st["len_in"], st["len_out"], st["kept"],
                          st["out"], st["ws"], st["ws"].numel())
    return {"tokens": st["out"], "kept": st["kept"], "len": st["len_out"]}


def run(st):
    case = st["case"]
    if own:
        return _own(st, case)
    return {"plan": _plain_plan, "append": _plain_append, "attention": _plain_attention, "verify": _plain_verify}[case["kind"]](st, case)


# ---- the definitions in 64 bits, request by request ----

def _exact_plan(st, case):
    p, width = case["page"], st["width"]
    base, new, held = (st[k].tolist() for k in ("base", "new", "held"))
    table, stack = st["table"].cpu().numpy().copy(), st["free"].cpu().numpy().copy()
    count = int(st["count"])
    need = [-(-(b + m) // p) for b, m in zip(base, new)]
    for r in range(case["n"]):
        for e in range(need[r], held[r]):
            stack[count] = table[r, e]
            count += 1
    held_out, seq_len, refused, full = list(held), [0] * case["n"], 0, False
    for r in range(case["n"]):
        more = need[r] - held[r]
        full = full or (need[r] <= width and more > count)
        if need[r] > width or (more > 0 and full):
            refused += 1
            continue
        for e in range(held[r], need[r]):
            count -= 1
            table[r, e] = stack[count]
        held_out[r], seq_len[r] = need[r], base[r] + new[r]
    slots, positions = np.full(st["max_rows"], -1), np.zeros(st["max_rows"], dtype=np.int64)
    row = 0
    for r in range(case["n"]):
        for i in range(new[r]):
            t = base[r] + i
            positions[row] = t
            if seq_len[r]:
                slots[row] = table[r, t // p] * p + t % p
            row += 1
    return {"table": table, "held": np.array(held_out), "free": stack, "count": np.array([count]), "row_start": np.array(_starts(new)),
            "seq_len": np.array(seq_len), "slots": slots, "positions": positions, "refused": np.array([refused])}


def _nearest_half(x):
    """float64 rounded to 11 significant bits (fewer below 2^-14), still in float64."""
    step = torch.exp2((torch.frexp(x)[1] - 11).clamp(min=-24).double())
    return torch.round(x / step) * step


def _exact_append(st, case):
    heads, h, d = case["heads"], case["kv_heads"], case["d"]
    width = (heads + 2 * h) * d
    out = {"rows": torch.zeros((st["total"], 2 * h * d), dtype=torch.float64, device="cuda")}
    if case["rope"]:
        out["q"] = torch.zeros((st["total"], heads * d), dtype=torch.float64, device="cuda")
    for a in range(0, st["total"], 1024):
        sl = slice(a, min(st["total"], a + 1024))
        x = st["qkv"][sl].double().reshape(-1, width // d, d)
        if case["rope"]:
            at = st["positions"][sl].long()
            cos, sin = st["rope"][at][:, None, :, 0].double(), st["rope"][at][:, None, :, 1].double()
            turned = torch.empty_like(x)
            turned[..., :d // 2] = x[..., :d // 2] * cos - x[..., d // 2:] * sin
            turned[..., d // 2:] = x[..., d // 2:] * cos + x[..., :d // 2] * sin
            out["q"][sl] = turned[:, :heads].reshape(-1, heads * d)
            x = torch.cat([_nearest_half(turned[:, heads:heads + h]), x[:, heads + h:]], 1)
        else:
            x = x[:, heads:]
        grouped = x.reshape(x.shape[0], -1, GROUP)
        low, high = grouped.min(-1, keepdim=True)[0], grouped.max(-1, keepdim=True)[0]
        scale = _nearest_half((high - low) / 15)
        code = torch.round((grouped - low) / torch.where(scale > 0, scale, 1.0)).clamp(0, 15) * (scale > 0)
        value = (code * scale + low).reshape(x.shape[0], -1)
        out["rows"][sl] = value * (st["slots"][sl] >= 0)[:, None]
    return out


def _exact_attention(st, case):
    p, d, h = case["page"], case["d"], case["kv_heads"]
    group = case["heads"] // h
    z = torch.zeros((st["rows"], case["heads"], d), dtype=torch.float64, device="cuda")
    at = 0
    for r, (L, m) in enumerate(zip(st["lens"], st["new_host"])):
        ids = st["table"][r, :(L + p - 1) // p].long()
        for j in range(h):
            block = p * 9 * d // 8
            one = st["pages"][ids][:, j * block:(j + 1) * block]
            cache = []
            for codes, scale, low in _unpack(one, 1, p, d):
                value = codes.double() * scale.double().repeat_interleave(GROUP, -1) + low.double().repeat_interleave(GROUP, -1)
                cache.append(value.reshape(-1, d)[:L])
            for i in range(group):
                head = j * group + i
                score = st["q"][at:at + m, head * d:(head + 1) * d].double() @ cache[0].t().contiguous() / d ** 0.5
                score += torch.full((m, L), -math.inf, dtype=torch.float64, device="cuda").triu(L - m + 1)
                z[at:at + m, head] = torch.softmax(score, -1) @ cache[1]
        at += m
    return z.reshape(st["rows"], -1)


def _exact_verify(st, case):
    start, tokens = st["row_start"].tolist(), st["tokens"].tolist()
    temperature, u, us, len_in = (st[k].double().tolist() for k in ("temperature", "u_accept", "u_sample", "len_in"))
    out, kept = [-1] * st["rows"], []

    def share(logits, t):
        x = logits.double().cpu().numpy()
        e = np.exp((x - x.max()) / t)
        return e / e.sum()

    for r in range(case["n"]):
        t, a, b = temperature[r], start[r], start[r + 1]
        row, pick = a, None
        while pick is None:
            logits = st["target"][row]
            drafted = tokens[row + 1] if row + 1 < b else None
            if t == 0:
                best = int(np.argmax(logits.float().cpu().numpy()))
                ok, rest = drafted == best, None
                pick = None if ok else best
            else:
                p = share(logits, t)
                ok, rest = False, p
                if drafted is not None:
                    q = share(st["draft"][row + 1], t) if case["draft"] else np.eye(1, case["vocab"], drafted)[0]
                    ok = u[row + 1] * q[drafted] < p[drafted]
                    rest = np.maximum(p - q, 0.0)
                    rest = rest if rest.sum() > 0 else p
                if not ok:
                    summed = np.cumsum(rest)
                    pick = int(np.argmax(summed > us[r] * summed[-1]))
            out[row] = drafted if ok else pick
            row += ok
        kept.append(row - a + 1)
    return {"tokens": np.array(out), "kept": np.array(kept), "len": np.array([int(x) + k for x, k in zip(len_in, kept)])}


def exact(case, seed):
    st = prepare(case, seed)
    return {"plan": _exact_plan, "append": _exact_append, "attention": _exact_attention, "verify": _exact_verify}[case["kind"]](st, case)
