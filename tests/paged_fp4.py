"""The 4-bit paged cache from its definition (float64), for the tests of the library's kernels."""
import math

import torch

import paper_2604_24432_amd as K
from tests.paged import Pages

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def e2m1(x):
    """Rows x (float64, last dimension) as the 4-bit cache holds them -> values they stand for, codes (one to a byte), biased exponents.

    The nearest level by its distance, of two as near the one with the even code; a group of 32 has the least power of two with max |x| <= 7 * 2^e."""
    levels = LEVELS.to(x.device)
    g = x.unflatten(-1, (-1, 32))
    fine = torch.isfinite(g).all(-1, keepdim=True)
    most = torch.where(fine, g.abs(), 0.0).amax(-1, keepdim=True)
    e = torch.full_like(most, -125.0)
    for n in range(-124, 126):
        e = torch.where(most > 7.0 * 2.0 ** (n - 1), float(n), e)
    y = torch.where(fine, g, 0.0) * torch.exp2(-e)
    off = (y.abs()[..., None] - levels).abs()
    off = off * 2 + (torch.arange(8, device=x.device) % 2) * 1e-12     # (halfway to the even code: distances are multiples of 2^-9 or so apart)
    code = off.argmin(-1)
    value = levels[code] * torch.exp2(e)
    negative = torch.signbit(y)
    value = torch.where(negative, -value, value)
    code = code + 8 * negative
    value = torch.where(fine, value, math.nan)
    code = torch.where(fine, code, 0)
    exps = torch.where(fine[..., 0], e[..., 0] + 127, 255.0)
    return value.flatten(-2), code.flatten(-2).to(torch.uint8), exps.to(torch.uint8)


def packed(code):
    return code[..., ::2] | code[..., 1::2] << 4


class Pages4(Pages):
    """A 4-bit pool and its tables; slots nobody has written hold NaN groups."""

    def __init__(self, p, n_rows, page, seed=0, device="cuda", spare=2, order="phsd", exponent=255, byte=0x77):
        super().__init__(p, n_rows, page, False, seed, device=device, spare=spare)
        n_pages, d = self.k.shape[0], p.head_dim

        def pool():
            x = torch.full((n_pages, p.n_kv_heads, page, d // 2), byte, dtype=torch.uint8, device=device)
            return x if order == "phsd" else x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)   # rows outside the heads
        self.k, self.v = pool(), pool()
        self.k_exp = torch.full((n_pages, p.n_kv_heads, page, d // 32), exponent, dtype=torch.uint8, device=device)
        self.v_exp = self.k_exp.clone()
        self.cache = K.PagedCache(p, self.k, self.v, self.text_dev, self.sums_dev if p.n_summary else None, self.k_exp, self.v_exp)

    def put(self, b, first, k, v):
        """Rows k, v [n, Hkv, d] (bf16) into the pages by index, without the library."""
        at, slot = (x.to(self.k.device) for x in self.places(b, first, k.shape[0]))
        for pool, exp, x in ((self.k, self.k_exp, k), (self.v, self.v_exp, v)):
            _, code, e = e2m1(x.double())
            pool[at, :, slot], exp[at, :, slot] = packed(code), e
