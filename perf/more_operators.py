"""More operators of a serving step and of training, and the cases that their performance is measured on.

Four operators over augmented sequences (chunks of c text rows, each followed by m summary rows): the paged cache in 4 bits (`write`: rows in and back
out, `attend`: new rows attend to what they see), rotary positions (`turn`: q and k of whole sequences and the gradients back through it, `place`: new rows of
a ragged batch are turned, k and v go into a cache in pages) and `advance`, which from the sequences' lengths works out a step's rows and gives and takes pages.

The cache in 4 bits holds a row of one KV head in groups of 32 elements: values 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives times a power of two
2^e per group, e the least integer in [-125, 125] with max |x| <= 7 * 2^e, every element rounded to the nearest (ties to the even code).

A row's rotary position is its text index, a summary row's that of its chunk's last text.  Pair i of the first `rot` elements, (2i, 2i + 1) or
(i, i + rot / 2), turns by position * base^(-2i / rot); for long contexts all frequencies are divided by `factor` ("linear") or those with few turns over
`original` positions are ("by_parts"), which then also scales the turned part.

A case is a dict of plain values; its "kind" is one of the words above.  `rows` is the largest number of new rows of a sequence and `n` the context in text
tokens; with `ragged` both differ from sequence to sequence.  `own` chooses between the plain forms below and the library's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False


def _attend(name, kind, batch, heads, kv_heads, d, n, rows, c, m, C, page, ragged=False):
    return _named(name, dict(kind=kind, batch=batch, heads=heads, kv_heads=kv_heads, d=d, n=n, rows=rows, c=c, m=m, C=C, page=page, ragged=ragged))


def _turn(name, kind, batch, heads, kv_heads, d, n, rows, c, m, page, rot, pairs, base, scaling="none", factor=1.0, original=4096, ragged=False):
    return _named(name, dict(kind=kind, batch=batch, heads=heads, kv_heads=kv_heads, d=d, n=n, rows=rows, c=c, m=m, C=1, page=page, rot=rot, pairs=pairs,
                             base=base, scaling=scaling, factor=factor, original=original, ragged=ragged))


def _advance(name, batch, n, c, m, C, page, prompts):
    return _named(name, dict(kind="advance", batch=batch, n=n, c=c, m=m, C=C, page=page, prompts=prompts))


def _named(name, case):
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # the smallest step of a generate loop over a 4-bit cache: launches and latency
        _attend("fp4_decode_tiny", "attend", 1, 8, 1, 64, 700, 1, 8, 1, 32, 16),
        # serving at a long context: 64 sequences at 128K, a quarter of the bytes of bf16
        _attend("fp4_decode_128k_b64", "attend", 64, 32, 8, 128, 131072 + 63, 1, 64, 8, 1, 64),
        # up to eight drafted tokens per sequence are checked in one pass, the paper's own form
        _attend("fp4_draft_64k_b16", "attend", 16, 32, 8, 128, 65536, 8, 8, 1, 128, 32, True),
        # a chunk of a 128K prompt in a summary layer; text and summary rows
        _attend("fp4_chunk_128k", "attend", 1, 32, 8, 128, 131072, 4608, 64, 8, 1, 64),
        # single tokens beside pieces of prompts in one batch; three query heads per KV head, odd chunks, short pages
        _attend("fp4_mixed_b6", "attend", 6, 12, 4, 64, 20011, 1031, 48, 6, 2, 16, True),
        # a whole prompt goes into the 4-bit cache and comes back as what it stands for
        _attend("fp4_write_32k", "write", 1, 32, 8, 128, 32768, 36864, 64, 8, 1, 64),
        # a training step's positions, there and back
        _turn("rotary_train_32k", "turn", 1, 32, 8, 128, 32768, 0, 64, 8, 16, 128, "half", 1e6),
        # half of the head, interleaved pairs, a context four times as long as the original, an incomplete last chunk
        _turn("rotary_train_odd", "turn", 2, 12, 4, 64, 6011, 0, 48, 6, 16, 32, "interleaved", 1e4, "by_parts", 4.0, 2048),
        # one new row of each of 64 sequences: positions and cache in one call
        _turn("rotary_decode_b64", "place", 64, 32, 8, 128, 131072, 1, 64, 8, 16, 128, "half", 1e6, ragged=True),
        # pieces of prompts at far positions
        _turn("rotary_chunk_b3", "place", 3, 32, 8, 128, 1048576, 4608, 64, 8, 64, 128, "half", 1e6, "linear", 8.0, 131072, ragged=True),
        # the step of 64 generate loops: most get one token, some end, some wait
        _advance("advance_decode_b64", 64, 131072, 64, 8, 1, 64, False),
        # prompts of many lengths come in beside others that go on
        _advance("advance_prompts_b200", 200, 8192, 64, 8, 1, 16, True),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choice(["attend", "attend", "attend", "write", "turn", "turn", "place", "place", "advance", "advance"])
        heads, kv_heads = rng.choice([(32, 8), (32, 8), (32, 8), (16, 16), (16, 4), (8, 1), (8, 4), (12, 4)])
        d = rng.choice([128, 128, 128, 64])
        c, m, C = rng.choice([(64, 8, 1), (64, 8, 1), (128, 16, 1), (8, 1, 128), (8, 1, 32), (16, 2, 64), (32, 4, 3), (64, 8, 0), (48, 6, 2),
                              (20, 5, 2), (1, 0, 255), (1, 0, 1023), (8, 0, 128), (64, 0, 4096)])
        page = rng.choice([16, 32, 64, 64, 128])
        batch = size(1, 64)
        ragged = batch > 1 and rng.random() < 0.6
        if kind in ("attend", "write"):
            n = size(256, 131072)
            rows = rng.choice([1, 1, rng.randint(2, 8), size(9, 4608)]) if kind == "attend" else size(1, 36864)
            case = _attend(None, kind, batch, heads, kv_heads, d, n, min(rows, _augmented(n, c, m)), c, m, C, page, ragged)
            seen = _lists(case)
            room = batch * max(x["n_sum"] + x["n_txt"] for x in seen)
            if work(case)["flops"] > 2e12 or work(case)["bytes"] > 1.2e9 or room * case["rows"] * heads > 4e9 or room * kv_heads * d > 1.1e9:
                continue
            if kind == "write" and sum(_starts(case)[1]) * kv_heads * d > 4e7:
                continue
        elif kind == "advance":
            batch = size(1, 256)
            case = _advance(None, batch, size(256, 131072), c, m, C, page, rng.random() < 0.5)
            if sum(_lengths(case)[1]) > 1.5e6 or batch * sum(_columns(case)) > 4e5 or _pool(case) > 4e5:
                continue
        else:
            n = size(1, 32768) if kind == "turn" else size(256, 1048576)
            rows = rng.choice([1, 1, rng.randint(2, 8), size(9, 4608)])
            rot = rng.choice([d, d, d, d // 2, d // 4, 48, 20])
            scaling = rng.choice(["none", "none", "linear", "by_parts"])
            case = _turn(None, kind, batch, heads, kv_heads, d, n, min(rows, _augmented(n, c, m)) if kind == "place" else 0, c, m, page, rot,
                         rng.choice(["half", "half", "interleaved"]), rng.choice([1e4, 5e5, 1e6]), scaling,
                         rng.choice([2.0, 4.0, 8.0]) if scaling != "none" else 1.0, rng.choice([2048, 4096, 32768]), ragged)
            if work(case)["bytes"] > 1.6e9:
                continue
        return case


# ---- sizes, on the host -------------------------------------------------------------------------------------------------

def _augmented(n, c, m):
    return n // c * (c + m) + n % c


def _text_of(a, c, m):
    """Text rows among the first a augmented rows."""
    return a // (c + m) * c + min(a % (c + m), c)


def _starts(case):
    """First new row (augmented) and number of new rows of every sequence."""
    B, L, rows = case["batch"], _augmented(case["n"], case["c"], case["m"]), case["rows"]
    start, count = [], []
    for b in range(B):
        k, end = rows, L
        if case["ragged"]:
            k = max(1, rows - rows * 3 * b // (4 * B) if b % 2 == 0 else rows // 4 ** min(b, 20))
            end = max(k, L * (B + 3 * ((5 * b) % B) + 3) // (4 * B) - 11 * b)
        if case["kind"] == "write":
            end = k      # whole sequences, or their beginnings
        start.append(min(end, L) - k), count.append(k)
    return start, count


def _seen(a, case):
    """Summaries [lo_s, hi_s) and text [lo_t, hi_t) that augmented row a sees."""
    c, m, C = case["c"], case["m"], case["C"]
    j, r = divmod(a, c + m)
    if r < c:
        first = max(j - C, 0)
        return 0, first * m, first * c, j * c + r + 1
    return j * m, j * m + r - c + 1, j * c, j * c + c


def _lists(case):
    """Per sequence: how many summaries and text rows its new rows see together, from which on, and the (row, key) pairs."""
    out = []
    for a0, k in zip(*_starts(case)):
        v = [_seen(a, case) for a in range(a0, a0 + k)]
        out.append(dict(n_sum=max(x[1] for x in v), t0=min(x[2] for x in v), n_txt=max(x[3] for x in v) - min(x[2] for x in v),
                        sums=max(x[1] for x in v) - min([x[0] for x in v if x[1] > x[0]], default=0), pairs=sum(x[1] - x[0] + x[3] - x[2] for x in v)))
    return out


def _lengths(case):
    """Text tokens that every sequence holds, and those that come: -1 where it has ended."""
    B, n = case["batch"], case["n"]
    held, new = [], []
    for b in range(B):
        if case["prompts"]:      # a third goes on from somewhere, the others begin; lengths over a factor of 64
            h = n // 2 * ((5 * b) % 7) // 7 if b % 3 == 2 else 0
            t = max(1, (n - h) * (1 + (11 * b) % 13) // (13 << (b % 7)) - b % 5)
        else:
            h = n // 4 + (n - 1 - n // 4) * ((7 * b) % 61) // 60
            t = -1 if b % 17 == 16 else 0 if b % 13 == 12 else 1
        held.append(h), new.append(min(t, n - h))
    return held, new


def _columns(case):
    c, m, page, n = case["c"], case["m"], case["page"], case["n"]
    return -(-n // page), -(-(n // c * m) // page) if m else 0


def _pages_of(case, h, t):
    """Columns of text and of summaries, from .. to, that hold something a sequence of h + t text tokens still needs when the t come."""
    c, m, C, page = case["c"], case["m"], case["C"], case["page"]
    return max(h // c - C, 0) * c // page, -(-(h + t) // page), -(-((h + t) // c * m) // page)


def _pool(case):
    total = 0
    for h, t in zip(*_lengths(case)):
        lo, text, sums = _pages_of(case, h, max(t, 0))
        total += text - lo + 2 + sums + 1
    return total + total // 4 + 3


def work(case):
    kind = case["kind"]
    if kind == "advance":
        held, new = _lengths(case)
        rows = sum(_augmented(h + max(t, 0), case["c"], case["m"]) - _augmented(h, case["c"], case["m"]) for h, t in zip(held, new))
        tables = sum(sum(_pages_of(case, h, max(t, 0))[1:]) for h, t in zip(held, new))
        return {"bytes": 4 * tables + 4 * _pool(case) + 16 * case["batch"] + 16 * rows, "flops": 0}
    H, Hkv, d = case["heads"], case["kv_heads"], case["d"]
    if kind == "turn":
        rows = case["batch"] * _augmented(case["n"], case["c"], case["m"])
        return {"bytes": 8 * rows * (H + Hkv) * d, "flops": 6 * rows * (H + Hkv) * case["rot"]}
    total = sum(_starts(case)[1])
    if kind == "place":
        return {"bytes": 4 * total * (H + 2 * Hkv) * d, "flops": 3 * total * (H + Hkv) * case["rot"]}
    held = 2 * Hkv * (d // 2 + d // 32)                  # bytes of a row in the cache, K and V
    if kind == "write":
        return {"bytes": 2 * total * (held + 4 * Hkv * d), "flops": 0}
    v = _lists(case)
    read = sum(x["sums"] + x["n_txt"] for x in v) * held + total * H * (4 * d + 4)
    return {"bytes": read, "flops": 4 * d * H * sum(x["pairs"] for x in v)}


# ---- inputs -------------------------------------------------------------------------------------------------------------

_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _split(x):
    """Two 4-bit codes per byte and biased exponents of rows x (last dimension, float32), as the cache holds them."""
    x = x.unflatten(-1, (-1, 32))
    most = x.abs().amax(-1)
    f, e = torch.frexp(most)                             # most = f 2^e, 0.5 <= f < 1; 7 = 0.875 * 2^3
    e = torch.where(most > 0, e - 3 + (f > 0.875).to(e.dtype), -125).clamp(-125, 125)
    y = torch.ldexp(x, -e[..., None]).flatten(-2)
    a, code = y.abs(), (y < 0).to(torch.uint8) * 8
    for level, reached in ((0.25, torch.gt), (0.75, torch.ge), (1.25, torch.gt), (1.75, torch.ge), (2.5, torch.gt), (3.5, torch.ge), (5.0, torch.gt)):
        code += reached(a, level)                        # (halfway goes to the even code)
    return code[..., ::2] | code[..., 1::2] << 4, (e + 127).to(torch.uint8)


def _values(pool, exps):
    """What rows stand for, float32."""
    levels = torch.tensor(_LEVELS + tuple(-x for x in _LEVELS), device=pool.device)
    y = levels[torch.stack([pool & 15, pool >> 4], -1).flatten(-2).int()]
    return torch.ldexp(y.unflatten(-1, (-1, 32)), exps.int()[..., None] - 127).flatten(-2)


def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _rows(g, dev, *shape):
    x = torch.randn(*shape, generator=g, device=dev)
    return x * torch.exp2(0.5 * torch.randn(*shape[:-1], 1, generator=g, device=dev))


def _batch(s, case, dev):
    start, count = _starts(case)
    cu = [0]
    for k in count:
        cu.append(cu[-1] + k)
    s["cu_rows"] = torch.tensor(cu, dtype=torch.int32, device=dev)
    s["start"] = torch.tensor(start, dtype=torch.int32, device=dev)
    s["row_seq"] = torch.repeat_interleave(torch.arange(case["batch"]), torch.tensor(count)).to(dev)      # the sequence of a packed row
    s["row_at"] = torch.arange(cu[-1], device=dev) - s["cu_rows"].long()[s["row_seq"]]                     # ... and its place among the sequence's
    return cu[-1]


def _tables(case, g, dev, first_t, last_t, first_s, last_s):
    """Tables whose columns first .. last - 1 have a page each, in any order; how many pages there are."""
    B = case["batch"]

    def table(first, last, base):
        cols = max(int(last.max()), 1)
        need = (torch.arange(cols) >= first[:, None]) & (torch.arange(cols) < last[:, None])
        t = torch.full((B, cols), -1, dtype=torch.int32)
        t[need] = base + torch.arange(int(need.sum()), dtype=torch.int32)
        return t, base + int(need.sum())

    text, used = table(first_t, last_t, 0)
    sums, used = table(first_s, last_s, used) if case["m"] else (None, used)
    order = torch.randperm(used + 3, generator=g, device=dev).to(torch.int32)     # a pool that has been in use

    def placed(t):
        t = t.to(dev)
        return torch.where(t >= 0, order[t.clamp(min=0).long()], -1).to(torch.int32).contiguous()

    return placed(text), placed(sums) if sums is not None else None, used + 3


def prepare(case, seed):
    dev = _device()
    g = torch.Generator(device=dev).manual_seed(seed)
    s = dict(case=case)
    if case["kind"] == "advance":
        return _prepare_advance(s, case, g, dev)
    B, Hq, Hkv, d, c, m, page = (case[x] for x in ("batch", "heads", "kv_heads", "d", "c", "m", "page"))
    if case["kind"] == "turn":
        L = _augmented(case["n"], c, m)
        for name, heads in (("q", Hq), ("k", Hkv), ("dq", Hq), ("dk", Hkv)):
            s[name] = torch.randn(B, L, heads, d, generator=g, device=dev).to(torch.bfloat16)
        if own:      # the parameters and the frequencies that a training program keeps
            s["params"], s["rotary"] = _params(case), _rotary(case, dev)
        return s
    start, count = _starts(case)
    total = _batch(s, case, dev)
    ends = [a + k for a, k in zip(start, count)]
    if case["kind"] == "attend":      # pages for what the new rows see; text that has left the window has none any more (-1)
        lists = _lists(case)
        s["n_sum"], s["n_txt"] = max(x["n_sum"] for x in lists), max(x["n_txt"] for x in lists)
        s["t0"] = torch.tensor([x["t0"] for x in lists], device=dev)
        first_t, last_t = [x["t0"] for x in lists], [max(_text_of(e, c, m), x["t0"] + x["n_txt"]) for e, x in zip(ends, lists)]
        first_s = [0] * B
    else:                             # ... for the new rows
        first_t, last_t, first_s = [_text_of(a, c, m) for a in start], [_text_of(e, c, m) for e in ends], [a - _text_of(a, c, m) for a in start]
    last_s = [e - _text_of(e, c, m) for e in ends]
    down, up = (lambda x: torch.tensor(x) // page), (lambda x: -(-torch.tensor(x) // page))
    s["text_table"], s["sum_table"], n_pages = _tables(case, g, dev, down(first_t), up(last_t), down(first_s), up(last_s))
    if case["kind"] == "place":
        s["k"], s["v"] = (torch.zeros(n_pages, Hkv, page, d, dtype=torch.bfloat16, device=dev) for _ in range(2))
        s["q"] = torch.randn(total, Hq, d, generator=g, device=dev).to(torch.bfloat16)
    else:
        for x in ("k", "v"):
            parts = [_split(_rows(g, dev, min(4096, n_pages - i), Hkv, page, d).to(torch.bfloat16).float()) for i in range(0, n_pages, 4096)]
            s[x], s[x + "_exp"] = torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])
        if case["kind"] == "attend":
            s["q"] = torch.randn(total, Hq, d, generator=g, device=dev).to(torch.bfloat16)
    if case["kind"] != "attend":
        s["k_new"], s["v_new"] = _rows(g, dev, total, Hkv, d).to(torch.bfloat16), _rows(g, dev, total, Hkv, d).to(torch.bfloat16)
    if own:      # the handle of the cache, the frequencies and the scratch memory that a serving program keeps
        import paper_2604_24432_amd as K
        s["cache"] = K.PagedCache(_params(case), s["k"], s["v"], s["text_table"], s["sum_table"], s.get("k_exp"), s.get("v_exp"))
        if case["kind"] == "place":
            s["rotary"] = _rotary(case, dev)
        if case["kind"] == "attend":
            s["workspace"] = torch.empty(max(K.paged_workspace_bytes(s["cache"], total, case["rows"]), 1), dtype=torch.uint8, device=dev)
    return s


def _params(case):
    import paper_2604_24432_amd as K
    return K.make_params(case["batch"], case["n"], case["c"], case["m"], case["C"], case.get("heads", 1), case.get("kv_heads", 1), case.get("d", 64))


def _rotary(case, dev):
    import paper_2604_24432_amd as K
    scaling = None if case["scaling"] == "none" else case["scaling"]
    return K.Rotary(case["rot"], base=case["base"], interleaved=case["pairs"] == "interleaved", scaling=scaling, factor=case["factor"],
                    original=case["original"], device=dev)


def _prepare_advance(s, case, g, dev):
    B, c, m, page = (case[x] for x in ("batch", "c", "m", "page"))
    held, new = _lengths(case)
    cols_t, cols_s = _columns(case)
    n_pages = _pool(case)
    order = torch.randperm(n_pages, generator=g, device=dev).cpu().numpy()
    table = np.full((B, cols_t + cols_s), -1, np.int32)
    used = 0
    for b, h in enumerate(held):      # what it held after the step before: the window of that step's token, which may begin a page earlier
        lo, text, sums = _pages_of(case, max(h - 1, 0), min(h, 1))
        if h:
            table[b, lo:text] = order[used:used + text - lo]
            used += text - lo
            table[b, cols_t:cols_t + sums] = order[used:used + sums]
            used += sums
    refs = np.zeros(n_pages, np.int32)
    refs[order[:used]] = 1
    # one tensor for what a step changes: both tables and the pages' reference counts
    at = [B * cols_t, B * (cols_t + cols_s)]
    flat = np.concatenate([table[:, :cols_t].ravel(), table[:, cols_t:].ravel(), refs])
    s["before"] = torch.from_numpy(flat).to(dev)
    s["now"] = s["before"].clone()
    s["text"], s["sums"], s["refs"] = s["now"][:at[0]].view(B, cols_t), s["now"][at[0]:at[1]].view(B, cols_s) if m else None, s["now"][at[1]:]
    s["held"], s["new"] = (torch.tensor(x, dtype=torch.int32, device=dev) for x in (held, new))
    rows = sum(_augmented(h + max(t, 0), c, m) - _augmented(h, c, m) for h, t in zip(held, new))
    s["total"] = rows + rows // 32 + 3     # a step's tensors have room for more
    if own:
        import paper_2604_24432_amd as K
        pool = torch.empty(n_pages, 1, page, 64, dtype=torch.bfloat16, device=dev)
        s["cache"] = K.PagedCache(_params(case), pool, pool, s["text"], s["sums"])
        s["workspace"] = torch.empty(max(K.paged_advance_workspace_bytes(s["cache"]), 1), dtype=torch.uint8, device=dev)
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if kind == "advance":
        s["now"].copy_(s["before"])      # (the step before this one again)
    if own:
        import paper_2604_24432_amd as K
        if kind == "attend":
            return K.ksa_paged_fwd(s["cache"], s["q"], s["cu_rows"], s["start"], max_rows=s["case"]["rows"], workspace=s["workspace"])
        if kind == "write":
            K.ksa_paged_append(s["cache"], s["k_new"], s["v_new"], s["cu_rows"], s["start"])
            return K.ksa_paged_read(s["cache"], s["cu_rows"], s["start"], len(s["row_seq"]))
        if kind == "turn":
            q, k = K.ksa_rotary_fwd(s["params"], s["rotary"], s["q"], s["k"])
            dq, dk = K.ksa_rotary_bwd(s["params"], s["rotary"], s["dq"], s["dk"])
            return q, k, dq, dk
        if kind == "place":
            q = K.ksa_paged_rotary(s["cache"], s["rotary"], s["q"], s["k_new"], s["v_new"], s["cu_rows"], s["start"])
            return q, s["k"], s["v"]
        step = K.ksa_paged_advance(s["cache"], s["refs"], s["held"], s["new"], s["total"], workspace=s["workspace"])
        return (step.cu_rows, step.start, step.lacking, step.slots, step.positions, step.tokens, s["text"], s["refs"]) + ((s["sums"],) if s["case"]["m"] else ())
    if kind == "attend":
        return _plain_attend(s)
    if kind == "write":
        at, slot = _places(s)
        for x in ("k", "v"):
            y, e = _split(s[x + "_new"].float())
            s[x][at, :, slot], s[x + "_exp"][at, :, slot] = y, e
        return tuple(_values(s[x][at, :, slot], s[x + "_exp"][at, :, slot]).to(torch.bfloat16) for x in ("k", "v"))
    if kind == "turn":
        c, m = s["case"]["c"], s["case"]["m"]
        a = torch.arange(s["q"].shape[1], device=s["q"].device)
        cos, sin = _plain_angles(s["case"], a // (c + m) * c + (a % (c + m)).clamp(max=c - 1))
        return tuple(_plain_turn(s["case"], s[x], cos, -sin if x[0] == "d" else sin) for x in ("q", "k", "dq", "dk"))
    if kind == "place":
        c, m = s["case"]["c"], s["case"]["m"]
        a = s["start"].long()[s["row_seq"]] + s["row_at"]
        cos, sin = _plain_angles(s["case"], a // (c + m) * c + (a % (c + m)).clamp(max=c - 1))
        at, slot = _places(s)
        s["k"][at, :, slot] = _plain_turn(s["case"], s["k_new"], cos, sin)
        s["v"][at, :, slot] = s["v_new"]
        return _plain_turn(s["case"], s["q"], cos, sin), s["k"], s["v"]
    return _plain_advance(s)


def _frequencies(case, dev):
    """Radians per position of every pair, float64, and what the turned part is multiplied with."""
    theta = case["base"] ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device=dev) / case["rot"])
    if case["scaling"] == "linear":
        return theta / case["factor"], 1.0
    if case["scaling"] == "by_parts":
        turns = case["original"] * theta / (2 * math.pi)
        keep = ((turns - 1) / (32 - 1)).clamp(0, 1)
        return theta * (keep + (1 - keep) / case["factor"]), 0.1 * math.log(case["factor"]) + 1
    return theta, 1.0


def _plain_angles(case, positions):
    theta, magnitude = _frequencies(case, positions.device)
    angle = positions.double()[:, None] * theta
    return (angle.cos() * magnitude).float(), (angle.sin() * magnitude).float()


def _plain_turn(case, x, cos, sin):
    """Pairs of x [.., rows, heads, d] turned by the rows' angles [rows, rot / 2]."""
    rot = case["rot"]
    cos, sin = cos[:, None], sin[:, None]
    y = x.float()
    if case["pairs"] == "half":
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], -1).to(torch.bfloat16)


def _places(s):
    """Page and slot of every packed row."""
    c, m, page = s["case"]["c"], s["case"]["m"], s["case"]["page"]
    a = s["start"].long()[s["row_seq"]] + s["row_at"]
    j, r = a // (c + m), a % (c + m)
    i, u = j * c + r.clamp(max=c - 1), j * m + (r - c).clamp(min=0)
    if m == 0:
        return s["text_table"][s["row_seq"], i // page].long(), i % page
    text = r < c
    at = s["text_table"][s["row_seq"], torch.where(text, i, 0) // page]
    u = torch.where(text, 0, u)
    return torch.where(text, at, s["sum_table"][s["row_seq"], u // page]).long(), torch.where(text, i % page, u % page)


def _plain_attend(s):
    B, T, Hq, Hkv, d, c, m, C, page = (s["case"][x] for x in ("batch", "rows", "heads", "kv_heads", "d", "c", "m", "C", "page"))
    G, dev = Hq // Hkv, s["q"].device
    a = s["start"].long()[:, None] + torch.arange(T, device=dev)
    j, r = a // (c + m), a % (c + m)
    text, first = r < c, (j - C).clamp(min=0)
    i, u = j * c + r, j * m + r - c
    lo_s, hi_s = torch.where(text, 0, j * m), torch.where(text, first * m, u + 1)
    lo_t, hi_t = torch.where(text, first * c, j * c), torch.where(text, i + 1, j * c + c)
    # keys of every sequence: summaries from the first on, then text from the first visible one on
    ks = torch.arange(s["n_sum"], device=dev).expand(B, -1)
    kt = s["t0"][:, None] + torch.arange(s["n_txt"], device=dev)
    seen = torch.cat([(ks[:, None] >= lo_s[..., None]) & (ks[:, None] < hi_s[..., None]),
                      (kt[:, None] >= lo_t[..., None]) & (kt[:, None] < hi_t[..., None])], -1)                # [B, T, N]
    b = torch.arange(B, device=dev)[:, None]
    at = s["text_table"][b, (kt // page).clamp(max=s["text_table"].shape[1] - 1)]
    if s["n_sum"]:
        at = torch.cat([s["sum_table"][b, (ks // page).clamp(max=s["sum_table"].shape[1] - 1)], at], 1)
    at, slot = at.clamp(min=0).long(), torch.cat([ks % page, kt % page], 1)
    k = _values(s["k"][at, :, slot], s["k_exp"][at, :, slot]).permute(0, 2, 1, 3).contiguous()                # [B, Hkv, N, d]
    q = torch.zeros(B, T, Hq, d, device=dev)
    q[s["row_seq"], s["row_at"]] = s["q"].float()
    q = q.view(B, T, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, d)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(1 / math.sqrt(d)).view(B, Hkv, T, G, -1)
    del k
    x.masked_fill_(~seen[:, None, :, None], -math.inf)
    most = x.amax(-1, keepdim=True)
    x.sub_(most).exp_()
    total = x.sum(-1, keepdim=True)
    v = _values(s["v"][at, :, slot], s["v_exp"][at, :, slot]).permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(x.view(B, Hkv, T * G, -1), v).view(B, Hkv, T, G, d) / total
    lse = (most + total.log())[..., 0]
    o = o.permute(0, 2, 1, 3, 4).reshape(B, T, Hq, d)[s["row_seq"], s["row_at"]]
    return o.to(torch.bfloat16), lse.permute(0, 2, 1, 3).reshape(B, T, Hq)[s["row_seq"], s["row_at"]]


def _plain_advance(s):
    B, c, m, C, page = (s["case"][x] for x in ("batch", "c", "m", "C", "page"))
    dev, h, t, total = s["held"].device, s["held"].long(), s["new"].long(), s["total"]
    ended, t = t < 0, t.clamp(min=0)
    e = h + t
    start = h // c * (c + m) + h % c
    count = torch.where(ended, 0, e // c * (c + m) + e % c - start)
    start = torch.where(ended, 0, start)
    cu = torch.cat([count.new_zeros(1), count.cumsum(0)])
    # columns of both tables side by side: given back, and lacking a page
    n_t = s["text"].shape[1]
    table = torch.cat([s["text"], s["sums"]], 1) if m else s["text"].clone()
    col = torch.arange(table.shape[1], device=dev)
    is_text, col = col < n_t, torch.where(col < n_t, col, col - n_t)
    begin = ((h // c - C).clamp(min=0) * c // page)[:, None]
    first = torch.where(is_text, -(-h // page)[:, None], -(-(h // c * m) // page)[:, None])
    last = torch.where(is_text, -(-e // page)[:, None], -(-(e // c * m) // page)[:, None])
    has = table >= 0
    leaves = has & (ended[:, None] | (is_text & (col < begin)))
    s["refs"].index_add_(0, torch.where(leaves, table, 0).flatten().long(), -leaves.flatten().int())
    lacks = ~has & ~ended[:, None] & (col >= first) & (col < last)
    free = s["refs"] == 0
    rank = free.cumsum(0) - 1
    n_pages = len(free)
    pages = torch.full((n_pages + 1,), -1, dtype=torch.int32, device=dev)      # the free ones, in order
    pages.scatter_(0, torch.where(free, rank, n_pages), torch.arange(n_pages, dtype=torch.int32, device=dev))
    want = lacks.flatten().cumsum(0).view(B, -1) - 1
    n_free, n_want = rank[-1] + 1, want[-1, -1] + 1
    given = lacks & (want < n_free)
    page_of = pages[torch.where(given, want, 0)]
    table = torch.where(given, page_of, torch.where(leaves, -1, table)).int()
    s["refs"].index_add_(0, torch.where(given, page_of, 0).flatten().long(), given.flatten().int())
    s["text"].copy_(table[:, :n_t])
    if m:
        s["sums"].copy_(table[:, n_t:])
    # what every row is
    row = torch.arange(total, device=dev)
    seq = torch.searchsorted(cu[1:].contiguous(), row, right=True)
    any_ = seq < B
    seq = seq.clamp(max=B - 1)
    a = start[seq] + row - cu[seq]
    j, r = a // (c + m), a % (c + m)
    text = r < c
    i, u = j * c + r.clamp(max=c - 1), j * m + (r - c).clamp(min=0)
    idx = torch.where(text, i, u)
    column = idx // page + torch.where(text, 0, n_t)
    at = table[seq, torch.where(any_, column, 0)].long()
    slots = torch.where(any_ & (at >= 0), at * page + idx % page, -1)
    positions = torch.where(any_, i, 0).int()
    before = torch.cat([t.new_zeros(1), t.cumsum(0)])[seq] - h[seq]
    tokens = torch.where(any_, torch.where(text, before + i, c - 1 - r), -1).int()
    out = (cu.int(), start.int(), (n_want - n_free).clamp(min=0).int().view(1), slots, positions, tokens, s["text"], s["refs"])
    return out + ((s["sums"],) if m else ())


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------

def _held(codes, exps):
    """float64 values of 4-bit codes: a sign, two bits of exponent, one of mantissa."""
    x = torch.stack([codes % 16, codes // 16], -1).flatten(-2).double()
    size, sign = x % 8, 1 - 2 * torch.floor(x / 8)
    power = torch.floor(size / 2)
    y = torch.where(power > 0, (1 + (size % 2) / 2) * torch.exp2(power - 1), size / 2)
    return sign * y * torch.exp2(exps.double() - 127).repeat_interleave(32, -1)


def _rounded(x):
    """float64 values of x as the 4-bit cache holds them."""
    y = x.unflatten(-1, (-1, 32))
    most = y.abs().amax(-1, keepdim=True)
    e = torch.full_like(most, -125)
    for k in range(-124, 126):
        e = torch.where(most > 7.0 * 2.0 ** (k - 1), float(k), e)
    y = y * torch.exp2(-e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=1.0))) - 1)
    return ((torch.round(y / step) * step).clamp(-6, 6) * torch.exp2(e)).flatten(-2)


def _turned(case, x, positions, back):
    """Pairs as complex numbers times exp(i angle)."""
    rot, dev = case["rot"], x.device
    i = torch.arange(rot // 2, dtype=torch.float64, device=dev)
    angle = torch.exp(-2 * i / rot * math.log(case["base"]))
    scale = 1.0
    if case["scaling"] == "linear":
        angle = angle / case["factor"]
    if case["scaling"] == "by_parts":
        keep = torch.clamp((case["original"] * angle / (2 * math.pi) - 1) / 31, 0, 1)
        angle = torch.lerp(angle / case["factor"], angle, keep)
        scale = 1 + math.log(case["factor"]) / 10
    phase = positions.double()[:, None] * angle
    by = torch.polar(torch.full_like(phase, scale), -phase if back else phase)[:, None]
    part = x[..., :rot].double()
    if case["pairs"] == "half":
        z = by * torch.complex(part[..., :rot // 2], part[..., rot // 2:])
        part = torch.cat([z.real, z.imag], -1)
    else:
        part = torch.view_as_real(by * torch.view_as_complex(part.unflatten(-1, (-1, 2)).contiguous())).flatten(-2)
    return torch.cat([part, x[..., rot:].double()], -1)


def exact(case, seed):
    if case["kind"] == "advance":
        return None
    s = prepare(case, seed)
    c, m, dev = case["c"], case["m"], _device()

    def position(a):
        j, r = divmod(a, c + m)
        return j * c + min(r, c - 1)

    if case["kind"] == "turn":
        at = torch.tensor([position(a) for a in range(s["q"].shape[1])], device=dev)
        return tuple(_turned(case, s[x], at, x[0] == "d") for x in ("q", "k", "dq", "dk"))
    start, count = _starts(case)
    page = case["page"]
    if case["kind"] == "write":
        return _rounded(s["k_new"].double()), _rounded(s["v_new"].double())
    text, sums = s["text_table"].tolist(), s["sum_table"].tolist() if m else None
    if case["kind"] == "place":
        where, at = [], []
        for b in range(case["batch"]):
            for a in range(start[b], start[b] + count[b]):
                j, r = divmod(a, c + m)
                x, t = (j * c + r, text) if r < c else (j * m + r - c, sums)
                where.append((t[b][x // page], x % page)), at.append(position(a))
        pages, slots = torch.tensor([x[0] for x in where], device=dev), torch.tensor([x[1] for x in where], device=dev)
        at = torch.tensor(at, device=dev)
        pool = {x: s[x].double() for x in ("k", "v")}
        pool["k"][pages, :, slots], pool["v"][pages, :, slots] = _turned(case, s["k_new"], at, False), s["v_new"].double()
        return _turned(case, s["q"], at, False), pool["k"], pool["v"]
    G = case["heads"] // case["kv_heads"]
    pool = {x: _held(s[x], s[x + "_exp"]) for x in ("k", "v")}
    outs, lses, at = [], [], 0
    for b in range(case["batch"]):
        v = torch.tensor([_seen(a, case) for a in range(start[b], start[b] + count[b])], device=dev)
        hi_s, lo_t, hi_t = int(v[:, 1].max()), int(v[:, 2].min()), int(v[:, 3].max())
        us, ts = torch.arange(hi_s, device=dev), torch.arange(lo_t, hi_t, device=dev)
        pg = s["text_table"][b].long()[ts // page]
        if hi_s:
            pg = torch.cat([s["sum_table"][b].long()[us // page], pg])
        sl = torch.cat([us, ts]) % page
        mask = torch.cat([(us >= v[:, :1]) & (us < v[:, 1:2]), (ts >= v[:, 2:3]) & (ts < v[:, 3:4])], 1)       # [rows, N]
        q = s["q"][at:at + count[b]].double()
        at += count[b]
        o, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float64, device=dev)
        for h in range(case["kv_heads"]):
            k_h, v_h = pool["k"][pg, h, sl], pool["v"][pg, h, sl]
            for r0 in range(0, count[b], 1024):
                part = slice(r0, r0 + 1024)
                for x in range(h * G, h * G + G):
                    z = (q[part, x] @ k_h.T / math.sqrt(case["d"])).masked_fill(~mask[part], -math.inf)
                    lse[part, x] = torch.logsumexp(z, 1)
                    o[part, x] = torch.softmax(z, 1) @ v_h
        outs.append(o), lses.append(lse)
    return torch.cat(outs), torch.cat(lses)
