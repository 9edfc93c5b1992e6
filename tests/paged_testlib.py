"""Inputs of the paged tests: pages, tables and ragged batches, on host and device."""
import numpy as np
import torch

from oracle import kvpr_paged_oracle as po


def i32(a):
    return torch.from_numpy(np.asarray(a, dtype=np.int32)).cuda()


class Batch:
    """Requests of given (length, new tokens) over a pool of random pages; page ids are a random permutation."""

    def __init__(self, lens, new, heads, kv_heads, d, page, seed, spare=3, extra_width=1, spread=1.0):
        self.lens, self.new, self.heads, self.kv_heads, self.d, self.page = list(lens), list(new), heads, kv_heads, d, page
        rng = self.rng = np.random.default_rng(seed)
        need = [-(-L // page) for L in self.lens]
        self.n_pages, self.width = sum(need) + spare, max(max(need), 1) + extra_width
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(self.lens), self.width), -1, dtype=np.int64)
        at = 0
        for r, m in enumerate(need):
            self.table[r, :m] = order[at:at + m]
            at += m
        # any bytes are codes; scales and minima as values of N(0, spread) have them
        block = page * 9 * d // 8
        pages = rng.integers(0, 256, (self.n_pages, kv_heads, block), dtype=np.uint8)
        pairs = np.empty((self.n_pages, kv_heads, 2 * page * (d // 64), 2), np.float16)
        pairs[..., 0] = rng.uniform(0.2, 0.4, pairs.shape[:-1]) * spread
        pairs[..., 1] = -rng.uniform(1.8, 2.6, pairs.shape[:-1]) * spread
        pages[..., page * d:] = pairs.reshape(self.n_pages, kv_heads, -1).view(np.uint8)
        self.pages = pages.reshape(self.n_pages, -1)
        self.row_start = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int64)
        self.rows = int(self.row_start[-1])

    def q(self, q_type, rows=None, scale=1.5):
        q = (self.rng.standard_normal((self.rows if rows is None else rows, self.heads * self.d)) * scale).astype(np.float32)
        return q.astype(np.float16) if q_type == "f16" else q

    def desc(self, k):
        return k.make_paged_desc(self.heads, self.kv_heads, self.d, self.page, self.n_pages, self.width)

    def attention(self, k, q, rows=None, max_new=None, max_len=None, ldq=None, ldz=None, stream=None, fill=7.0):
        """z of the library as float64 numpy, [rows, heads * d]; untouched elements hold `fill`."""
        cols = self.heads * self.d
        rows = q.shape[0] if rows is None else rows
        ldq, ldz = ldq or cols, ldz or cols
        qd = torch.zeros((max(q.shape[0], 1), ldq), dtype=torch.float16 if q.dtype == np.float16 else torch.float32, device="cuda")
        qd[:q.shape[0], :cols] = torch.from_numpy(q).cuda()
        z = torch.full((max(q.shape[0], 1), ldz), fill, dtype=torch.float16, device="cuda")
        max_new, max_len = max_new or max(max(self.new), 1), max_len or max(max(self.lens), 1)
        desc, n = self.desc(k), len(self.lens)
        ws = torch.full((k.kvpr_paged_attention_workspace_bytes(desc, n, rows, max_new, max_len),), 0xFF, dtype=torch.uint8, device="cuda")
        pages, table, start, lens = torch.from_numpy(self.pages).cuda(), i32(self.table), i32(self.row_start), i32(self.lens)
        k.kvpr_paged_attention(desc, qd, k.KVPR_F16 if q.dtype == np.float16 else k.KVPR_F32, ldq, pages, table, start, lens, n, rows, max_new, max_len,
                               z, ldz, ws, ws.numel(), stream=stream)
        torch.cuda.synchronize()
        assert (z[:, cols:] == fill).all()
        return z[:q.shape[0], :cols].double().cpu().numpy()

    def oracle(self, q, rows=None):
        return po.attention(q, self.pages, self.table, self.row_start, self.lens, self.heads, self.kv_heads, self.d, self.page,
                            q.shape[0] if rows is None else rows)
