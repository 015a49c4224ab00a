"""The paged cache and the attention over it, written out from their definitions (float64), for the tests of the library's kernels.

Sequences are kept whole here, k and v [rows, Hkv, d] in augmented order (Eq. 1); `build` lays them out in pages."""
import math

import numpy as np
import torch

import paper_2604_24432_amd as K

BF16, E4M3 = 2.0 ** -8, 2.0 ** -4      # a rounding's largest relative error


def kinds(n_rows, c, m):
    """Per augmented row: its chunk, whether it is text, and its text index or summary ordinal."""
    a = np.arange(n_rows)
    j, r = a // (c + m), a % (c + m)
    return j, r < c, np.where(r < c, j * c + r, j * m + r - c)


def mask(rows, n_rows, c, m, C, self_only=False):
    """[len(rows), n_rows]: what the augmented rows see, key by key."""
    j, text, idx = kinds(n_rows, c, m)
    jq, tq, iq = j[rows][:, None], text[rows][:, None], idx[rows][:, None]
    by_text = np.where(text, (j >= jq - C) & (idx <= iq), j < jq - C)
    by_summary = np.where(text, j == jq, (idx == iq) if self_only else ((j == jq) & (idx <= iq)))
    return np.where(tq, by_text, by_summary)


def attend(q, k, v, rows, p):
    """Rows `rows` of a sequence whose whole k and v (float64) are given -> o, lse, and how far a kernel may be off each.

    Off the output: half a step of bf16 for the output and for every weight, which carries |v|; the score's float32 sum of d products
    is off by (d + 8) 2^-24 sum |q k| at most and a weight by twice that (it and the row's maximum), all other float32 steps, the exponential's
    among them, by 2^-21 together; a sum of n weights by n 2^-24."""
    dev = k.device
    see = torch.from_numpy(mask(np.asarray(rows), k.shape[0], p.chunk_len, p.n_summary, p.window_chunks, bool(p.flags & 1))).to(dev)
    scale = p.softmax_scale if p.softmax_scale > 0 else 1 / math.sqrt(p.head_dim)
    G = p.n_q_heads // p.n_kv_heads
    o, lse = torch.empty(q.shape, dtype=torch.float64, device=dev), torch.empty(q.shape[:2], dtype=torch.float64, device=dev)
    o_off, lse_off = torch.empty_like(o), torch.empty_like(lse)
    n = see.sum(1).double()
    for h in range(p.n_q_heads):
        kh, vh = k[:, h // G], v[:, h // G]
        s = (q[:, h] @ kh.T * scale).masked_fill(~see, -math.inf)
        size = ((q[:, h].abs() @ kh.abs().T) * abs(scale)).masked_fill(~see, 0).amax(1)
        w = torch.softmax(s, 1)
        o[:, h], lse[:, h] = w @ vh, torch.logsumexp(s, 1)
        score_off = (p.head_dim + 8) * 2.0 ** -24 * size
        o_off[:, h] = (BF16 + 2 * score_off + 2.0 ** -21 + n * 2.0 ** -24)[:, None] * (w @ vh.abs()) * 1.01 + BF16 * o[:, h].abs()
        lse_off[:, h] = score_off + 2.0 ** -21 * (1 + lse[:, h].abs()) + n * 2.0 ** -24
    return o, lse, o_off, lse_off


def e4m3(x):
    """Rows x (float64, last dimension) as the 8-bit cache holds them -> values they stand for, biased exponents."""
    fine = torch.isfinite(x)
    most = torch.where(fine, x.abs(), 0.0).amax(-1, keepdim=True)
    e = torch.full_like(most, -117.0)
    for n in range(-116, 120):
        e = torch.where(most > 448.0 * 2.0 ** (n - 1), float(n), e)
    y = (torch.where(fine, x, 0.0) * torch.exp2(-e)).clamp(-448, 448)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    y = torch.round(y / step) * step * torch.exp2(e)
    return torch.where(fine, y, math.nan), (e[..., 0] + 127).to(torch.uint8)


class Pages:
    """A pool and tables for sequences of up to n_rows[b] augmented rows, pages in random order, filled with `fill`."""

    def __init__(self, p, n_rows, page, fp8, seed=0, fill=math.nan, device="cuda", spare=2, order="phsd"):
        g = torch.Generator().manual_seed(seed)
        self.p, self.page, self.fp8 = p, page, fp8
        need = [K.paged_pages(p, page, n) for n in n_rows]
        cols_t, cols_s = max(max(t for t, _ in need), 1), max(max(s for _, s in need), 1)
        n_pages = sum(t + s for t, s in need) + spare
        order_of = torch.randperm(n_pages, generator=g).to(torch.int32)
        self.text, self.sums, at = torch.full((p.batch, cols_t), -1, dtype=torch.int32), torch.full((p.batch, cols_s), -1, dtype=torch.int32), 0
        for b, (t, s) in enumerate(need):
            self.text[b, :t], self.sums[b, :s] = order_of[at:at + t], order_of[at + t:at + t + s]
            at += t + s
        shape = (n_pages, p.n_kv_heads, page, p.head_dim)

        def pool():
            x = torch.full(shape, fill, device=device)
            x = x.to(torch.float8_e4m3fn if fp8 else torch.bfloat16)
            return x if order == "phsd" else x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)   # rows outside the heads
        self.k, self.v = pool(), pool()
        self.k_exp = torch.full(shape[:3], 127, dtype=torch.uint8, device=device) if fp8 else None
        self.v_exp = self.k_exp.clone() if fp8 else None
        self.text_dev, self.sums_dev = self.text.to(device), self.sums.to(device)
        self.cache = K.PagedCache(p, self.k, self.v, self.text_dev, self.sums_dev if p.n_summary else None, self.k_exp, self.v_exp)

    def places(self, b, first, n):
        """Page and slot of augmented rows first .. first + n - 1 of sequence b."""
        _, text, idx = kinds(first + n, self.p.chunk_len, self.p.n_summary)
        text, idx = text[first:], idx[first:]
        page = np.where(text, self.text[b].numpy()[np.minimum(idx // self.page, self.text.shape[1] - 1)],
                        self.sums[b].numpy()[np.minimum(idx // self.page, self.sums.shape[1] - 1)])
        return torch.from_numpy(page).long(), torch.from_numpy(idx % self.page).long()

    def put(self, b, first, k, v):
        """Rows k, v [n, Hkv, d] (bf16) into the pages by index, without the library."""
        at, slot = (x.to(self.k.device) for x in self.places(b, first, k.shape[0]))
        for pool, exp, x in ((self.k, self.k_exp, k), (self.v, self.v_exp, v)):
            if self.fp8:
                y, e = e4m3(x.double())
                y = torch.where(torch.isfinite(y), y * torch.exp2(127 - e.double())[..., None], math.nan).float().to(torch.float8_e4m3fn)
                pool.view(torch.uint8)[at, :, slot] = y.view(torch.uint8)
                exp[at, :, slot] = e
            else:
                pool[at, :, slot] = x


def batch_of(first, count, device="cuda"):
    cu = np.concatenate([[0], np.cumsum(count)])
    return torch.tensor(cu, dtype=torch.int32, device=device), torch.tensor(first, dtype=torch.int32, device=device)


def randn(*shape, seed=0, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, generator=g) * torch.exp2(torch.randn(*shape[:-1], 1, generator=g))
    return x.to(torch.bfloat16).to(device)


def stands_for(x, fp8):
    """float64 values that bf16 rows x stand for in the cache."""
    return e4m3(x.double())[0] if fp8 else x.double()
