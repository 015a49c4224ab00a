"""Rotary positions from their definition in 64 bits, for the tests of the library's kernels."""
import math

import numpy as np
import torch

import paper_2604_24432_amd as K
from tests.paged import BF16

RULES = [dict(dim=128), dict(dim=64, base=1e6, interleaved=True), dict(dim=32, base=5e5, scaling="linear", factor=4.0),
         dict(dim=64, scaling="by_parts", factor=8.0, original=2048.0), dict(dim=20), dict(dim=2, base=100.0), dict(dim=36, interleaved=True, scaling="by_parts", factor=2.0,
         original=64.0, slow=0.5, fast=4.0), dict(dim=46, base=1e6, magnitude=0.7), dict(dim=128, interleaved=True), dict(dim=16), dict(dim=6, interleaved=True)]


def name(rule):
    return "-".join(f"{k}{v}" for k, v in rule.items())


def frequencies(rule):
    """Radians per position (Python floats) and the magnitude."""
    dim, base, factor = rule["dim"], rule.get("base", 1e4), rule.get("factor", 1.0)
    out = []
    for i in range(dim // 2):
        f = base ** (-2 * i / dim)
        if rule.get("scaling") == "linear":
            f /= factor
        if rule.get("scaling") == "by_parts":
            slow, fast = rule.get("slow", 1.0), rule.get("fast", 32.0)
            s = min(max((rule["original"] * f / (2 * math.pi) - slow) / (fast - slow), 0.0), 1.0)
            f *= s + (1 - s) / factor
        out.append(f)
    magnitude = 0.1 * math.log(factor) + 1 if rule.get("scaling") == "by_parts" else 1.0
    return out, rule.get("magnitude", magnitude)


def positions(rows, c, m):
    """Rotary positions of augmented rows."""
    a = np.asarray(rows)
    return a // (c + m) * c + np.minimum(a % (c + m), c - 1)


def turn(x, rule, at, back=False):
    """Rows x [.., rows, heads, d] (float64) at positions `at` -> turned, and how far a kernel may be off.

    A cosine and a sine are off by 2^-22 at most (32 bits of a turn, the series, roundings), each of the two products and their sum by 2^-24 of its size; the
    output is rounded to bf16 once."""
    f, magnitude = frequencies(rule)
    dim = rule["dim"]
    pairs = [(2 * i, 2 * i + 1) if rule.get("interleaved") else (i, i + dim // 2) for i in range(dim // 2)]
    angle = torch.tensor(at, dtype=torch.float64, device=x.device)[:, None, None] * torch.tensor(f, dtype=torch.float64, device=x.device)
    c, s = angle.cos() * magnitude, angle.sin() * magnitude * (-1 if back else 1)
    i, j = ([p[k] for p in pairs] for k in (0, 1))
    a, b = x[..., i], x[..., j]
    y, off = x.clone(), torch.zeros_like(x)
    y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    size = (a.abs() + b.abs()) * magnitude * 2.0 ** -21
    off[..., i] = off[..., j] = size
    turned = torch.zeros(x.shape[-1], dtype=torch.bool, device=x.device)
    turned[:dim] = True
    return y, torch.where(turned, off + BF16 * y.abs() + 2.0 ** -133, 0.0)


def handle(rule, device="cuda"):
    r = dict(rule)
    return K.Rotary(r.pop("dim"), device=device, **r)
