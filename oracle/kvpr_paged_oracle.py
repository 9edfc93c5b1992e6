"""CPU oracle for ragged batches over a paged 4-bit cache, in float64.  TEST INFRASTRUCTURE ONLY.

It shares no code with the HIP library and never imports it.  What it implements is stated request by request, without any of
the library's order of work:

  * plan: what a request needs is ceil((base + new) / page) pages; requests that hold more give pages back, in order, onto a stack; then
    requests that need more take pages off it, in order, refused from the first that does not find enough;
  * append: k (rotated by the position: element i of a head with element i + d/2, one rounding to float16) and v of a token, packed with the codec of
    kvpr_int4_oracle (groups of 64 columns of one head) into a page;
  * page: for each key/value head the bytes of `key codes | value codes | key pairs | value pairs`; words of 4 bytes of a key row in the order
    [g][s] of columns 8 (4 s + g); value bytes of four positions side by side, byte 32 u + 2 m + w of a row at place [m][u][w];
  * attention: softmax(q k^T / sqrt(d)) v over the positions that a row sees, query head i with key/value head i / group; k as
    code * scale + minimum, v rounded to float16;
  * verification: a draft x stands if u q(x) < p(x); behind the first that does not, the token at which the running sum of max(p - q, 0)
    passes u times its total.
"""
from __future__ import annotations

import numpy as np

from oracle import kvpr_int4_oracle as io


def plan(base, new, held, table, free, count, page, max_rows, n_pages):
    """All lists / arrays of ints; returns a dict of the outputs (table and free as copies)."""
    n, width = len(base), table.shape[1]
    table, free = table.copy(), free.copy()
    base, new = [max(int(b), 0) for b in base], [max(int(m), 0) for m in new]
    need = [(b + m + page - 1) // page for b, m in zip(base, new)]
    held_out, seq_len, refused = [int(h) for h in held], [0] * n, 0
    for r in range(n):
        for e in range(need[r], held_out[r]):
            free[count] = table[r, e]
            count += 1
    full = False
    for r in range(n):
        more = max(0, need[r] - held_out[r])
        if need[r] > width:
            refused += 1
            continue
        if more and (full or more > count):
            full = True
            refused += 1
            continue
        for e in range(held_out[r], need[r]):
            count -= 1
            table[r, e] = free[count]
        held_out[r], seq_len[r] = need[r], base[r] + new[r]
    row_start = np.concatenate([[0], np.cumsum(new)])
    slots, positions = np.full(max_rows, -1), np.zeros(max_rows, dtype=np.int64)
    for r in range(n):
        for i in range(new[r]):
            row, t = int(row_start[r]) + i, base[r] + i
            if row >= max_rows:
                break
            positions[row] = t
            if t < seq_len[r] and 0 <= table[r, t // page] < n_pages:
                slots[row] = table[r, t // page] * page + t % page
    return {"table": table, "free": free, "held": held_out, "seq_len": seq_len, "count": count, "refused": refused,
            "row_start": row_start, "slots": slots, "positions": positions}


def rotate(x, table, positions):
    """x [rows, heads, d], table [n_pos, d/2, 2] -> float64, not rounded."""
    d = x.shape[-1]
    cs = table[np.asarray(positions)].astype(np.float64)[:, None]
    a, b = x[..., :d // 2].astype(np.float64), x[..., d // 2:].astype(np.float64)
    return np.concatenate([a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]], -1)


def _places(d):
    key = np.empty(d // 2, dtype=np.int64)
    value = np.empty(d // 2, dtype=np.int64)
    for k in range(d // 2):
        word, in_word = divmod(k, 4)
        s, g = divmod(word, 4)
        key[k] = (g * (d // 32) + s) * 4 + in_word
        u, rest = divmod(k, 32)
        m, w = divmod(rest, 2)
        value[k] = m * (d // 32) + 2 * u + w
    return key, value


def page_bytes(kv_heads, d, page):
    return kv_heads * page * 9 * d // 8


def _addresses(head, t, d, page, is_key):
    """(byte addresses of a row's code bytes 0 .. d/2 - 1, address of its first pair) inside a page."""
    key, value = _places(d)
    block = head * page * 9 * d // 8
    codes = block + t * (d // 2) + key if is_key else block + page * d // 2 + (t // 4) * (2 * d) + value * 4 + t % 4
    return codes, block + page * d + (0 if is_key else page * (d // 64) * 4) + t * (d // 64) * 4


def store(pages, slot, k, v, page):
    """k, v [kv_heads, d] float16 into pages [n_pages, page_bytes] uint8."""
    d = k.shape[-1]
    for x, is_key in ((k, True), (v, False)):
        codes, scale, mn = io.quantize_rows(x)
        nib = codes[:, 0::2] | codes[:, 1::2] << 4
        for h in range(k.shape[0]):
            at, pair = _addresses(h, slot % page, d, page, is_key)
            pages[slot // page][at] = nib[h]
            pages[slot // page][pair:pair + d // 64 * 4] = np.stack([scale[h], mn[h]], -1).astype(np.float16).reshape(-1).view(np.uint8)


def load(pages, slot, kv_heads, d, page):
    """(codes [kv_heads, d], scale, mn [kv_heads, d / 64]) of k, then of v."""
    out = []
    for is_key in (True, False):
        codes, scale, mn = np.empty((kv_heads, d), np.uint8), np.empty((kv_heads, d // 64), np.float16), np.empty((kv_heads, d // 64), np.float16)
        for h in range(kv_heads):
            at, pair = _addresses(h, slot % page, d, page, is_key)
            b = pages[slot // page][at]
            codes[h, 0::2], codes[h, 1::2] = b & 15, b >> 4
            pairs = pages[slot // page][pair:pair + d // 64 * 4].copy().view(np.float16).reshape(-1, 2)
            scale[h], mn[h] = pairs[:, 0], pairs[:, 1]
        out.append((codes, scale, mn))
    return out


def values(codes, scale, mn):
    """float64, not rounded."""
    spread = lambda a: np.repeat(a.astype(np.float64), io.GROUP, -1)                    # noqa: E731
    return codes.astype(np.float64) * spread(scale) + spread(mn)


def attention(q, pages, table, row_start, seq_len, heads, kv_heads, d, page, n_rows):
    """q [n_rows, heads * d] -> (z float64, bound float64): z per row, and what a kernel may be off by that rounds
    its weights and its result to float16 once each (half a step, 2^-11) and sums in float32."""
    z = np.zeros((n_rows, heads, d))
    tol = np.zeros((n_rows, heads, d))
    done = np.zeros(n_rows, bool)
    group = heads // kv_heads
    for r in range(len(row_start) - 1):
        m, L = int(row_start[r + 1] - row_start[r]), int(seq_len[r])
        span = min(L, table.shape[1] * page)
        ts = [t for t in range(span) if 0 <= table[r, t // page] < len(pages)]
        cache = [load(pages, table[r, t // page] * page + t % page, kv_heads, d, page) for t in ts]
        for i in range(m):
            row = int(row_start[r]) + i
            if row >= n_rows:
                break
            done[row] = True
            see = [j for j, t in enumerate(ts) if t < L - m + i + 1]
            if not see:
                continue
            for h in range(heads):
                g = h // group
                k = np.stack([values(*(a[g] for a in cache[j][0])) for j in see])
                v = np.stack([values(*(a[g] for a in cache[j][1])) for j in see]).astype(np.float16).astype(np.float64)
                ks = np.stack([np.repeat(15 * cache[j][0][1][g].astype(np.float64) + np.abs(cache[j][0][2][g].astype(np.float64)), io.GROUP) for j in see])
                x = q[row, h * d:(h + 1) * d].astype(np.float64)
                s = k @ x / np.sqrt(d)
                p = np.exp(s - s.max())
                p /= p.sum()
                z[row, h] = p @ v
                # a score passes about 16 roundings of 2^-24 of sums of |q| (15 scale + |minimum|); so do a weight and the sum of weights
                off = 16 * 2.0 ** -24 * ((ks @ np.abs(x) / np.sqrt(d)).max() + 1)
                tol[row, h] = 2.0 ** -11 * (p @ np.abs(v) + np.abs(z[row, h])) + 2 * off * (p @ np.abs(v)) + 2.0 ** -25
    return z.reshape(n_rows, -1), tol.reshape(n_rows, -1), done


def _share(logits, t):
    x = np.where(np.isnan(logits.astype(np.float64)), -np.inf, logits.astype(np.float64))
    top = x.max()
    if top == -np.inf:
        return None
    with np.errstate(invalid="ignore"):
        e = np.where(x == top, 1.0, np.exp((x - top) / t))
    return e / e.sum()


def verify(target, draft, tokens, row_start, temperature, u_accept, u_sample, n_rows, seq_len=None, certain=None):
    """-> (out_tokens, kept); rows outside every request are given as None.  A request whose seq_len is 0 was refused: nothing of it counts.
    certain: rows of each request, from its first on, that hold certain tokens; a token that is certain stands."""
    out, kept = [None] * n_rows, []
    vocab = target.shape[1]
    for r in range(len(row_start) - 1):
        a, b = int(row_start[r]), min(int(row_start[r + 1]), n_rows)
        if a >= b:
            kept.append(0)
            continue
        if seq_len is not None and seq_len[r] <= 0:
            out[a:b] = [-1] * (b - a)
            kept.append(0)
            continue
        t = float(temperature[r])
        greedy = not t > 0
        row, pick = a, None
        sure = a + (1 if certain is None else max(int(certain[r]), 1))
        while pick is None:
            if row + 1 < min(sure, b):
                out[row] = int(tokens[row + 1])
                row += 1
                continue
            x = int(tokens[row + 1]) if row + 1 < b else None
            p = _share(target[row], 1.0 if greedy else t)
            ok = False
            if p is None:
                pick = -1
            elif greedy:
                best = int(np.argmax(np.where(np.isnan(target[row]), -np.inf, target[row].astype(np.float64))))
                ok = x == best
                pick = None if ok else best
            else:
                s = p
                if x is not None and 0 <= x < vocab:
                    if draft is None:
                        q = np.zeros(vocab)
                        q[x] = 1.0
                    else:
                        q = _share(draft[row + 1], t)
                        q = np.zeros(vocab) if q is None else q
                    ok = float(u_accept[row + 1]) * q[x] < p[x]
                    s = np.maximum(p - q, 0)
                    s = s if s.sum() > 0 else p
                if not ok:
                    c = np.cumsum(s)
                    above = np.nonzero(c > float(u_sample[r]) * c[-1])[0]
                    pick = int(above[0])
            if ok:
                out[row] = x
                row += 1
        out[row] = pick
        out[row + 1:b] = [-1] * (b - row - 1)
        kept.append(row - a + 1)
    return out, kept
