"""The operators of the paged KV cache, and the cases that their performance is measured on.

A cache in pages holds the K / V rows of a ragged batch of augmented sequences (chunks of c text rows, each followed by m summary rows);
text index i and summary ordinal u of a sequence lie in the pages that its rows of two tables name.  Three operators: new rows are written
(`append`, as bf16 or as 8-bit floats with a power of two per row and KV head), rows are read back (`read`), and the new rows attend
(`attend`) to what they see: a text row of chunk j to the summaries of the chunks before j - C and the text from chunk j - C up to itself, a
summary row to the text of its own chunk and that chunk's summaries up to itself.

A case is a dict of plain values; its "kind" says what makes up one pass:
  attend  the new rows of every sequence, already in the cache, attend: one row (decode), a few (drafted tokens), thousands (a chunk of a prompt);
  step    append, then attend: a step of a generate loop;
  append  append alone (a bf16 cache: what it holds comes back whole);
  write   append, then read the same rows back: what the cache stands for;
  read    rows are read back (moved out of the cache, handed to another one).
`rows` is the largest number of new rows of a sequence and `n` the context in text tokens; with `ragged` both differ from sequence to sequence.
`own` chooses between the plain forms below (float32, elementary operations) and the library's calls.
"""
from __future__ import annotations

import math

import torch

own = False


def _case(name, kind, batch, heads, kv_heads, d, n, rows, c, m, C, page, fp8, ragged=False):
    case = dict(kind=kind, batch=batch, heads=heads, kv_heads=kv_heads, d=d, n=n, rows=rows, c=c, m=m, C=C, page=page, fp8=fp8, ragged=ragged)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # the smallest step of a generate loop: one sequence, a few hundred rows; launches and latency
        _case("step_tiny", "step", 1, 8, 1, 64, 700, 1, 8, 1, 32, 16, False),
        # a small batch of generate loops of different lengths at a middle context
        _case("decode_32k_b4", "attend", 4, 32, 8, 128, 32768 + 40, 1, 64, 8, 1, 64, False, True),
        # serving at a long context from a cache of half the size: 64 sequences at 128K
        _case("decode_128k_b64_fp8", "attend", 64, 32, 8, 128, 131072 + 63, 1, 64, 8, 1, 64, True),
        # up to eight drafted tokens per sequence are checked in one pass, the paper's own form
        _case("draft_64k_b16_fp8", "attend", 16, 32, 8, 128, 65536, 8, 8, 1, 128, 32, True, True),
        # a chunk of a long prompt in a layer of full attention: the matrix unit's case
        _case("chunk_full_64k", "attend", 1, 32, 8, 128, 65536, 2048, 64, 0, 4096, 128, False),
        # a chunk of a 128K prompt in a summary layer, the cache in 8 bits; text and summary rows
        _case("chunk_128k_fp8", "attend", 1, 32, 8, 128, 131072, 4608, 64, 8, 1, 64, True),
        # single tokens beside pieces of prompts in one batch; three query heads per KV head, odd chunks, short pages
        _case("mixed_b6", "attend", 6, 12, 4, 64, 20011, 1031, 48, 6, 2, 16, False, True),
        # a sliding window without summaries, pieces of two prompts, no grouped heads
        _case("window_chunk_fp8", "attend", 2, 16, 16, 128, 16384, 1024, 1, 0, 1023, 64, True, True),
        # one new row of each of 64 sequences: latency
        _case("append_b64", "append", 64, 32, 8, 128, 2048, 1, 64, 8, 1, 16, False, True),
        # a whole prompt goes into the 8-bit cache and comes back as what it stands for
        _case("write_32k_fp8", "write", 1, 32, 8, 128, 32768, 36864, 64, 8, 1, 64, True),
        # the same for pieces of odd lengths
        _case("write_ragged_fp8", "write", 7, 12, 4, 64, 6011, 2500, 48, 6, 2, 32, True, True),
        # sequences of different lengths leave the cache
        _case("read_16k_b3", "read", 3, 16, 16, 128, 16384, 18432, 64, 8, 1, 16, False, True),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choice(["attend", "attend", "attend", "attend", "step", "append", "write", "read"])
        heads, kv_heads = rng.choice([(32, 8), (32, 8), (32, 8), (16, 16), (16, 4), (8, 1), (8, 4), (12, 4)])
        d = rng.choice([128, 128, 128, 64])
        c, m, C = rng.choice([(64, 8, 1), (64, 8, 1), (128, 16, 1), (8, 1, 128), (8, 1, 32), (16, 2, 64), (32, 4, 3), (64, 8, 0), (48, 6, 2),
                              (20, 5, 2), (1, 0, 255), (1, 0, 1023), (8, 0, 128), (64, 0, 4096)])
        batch = size(1, 64)
        n = size(256, 131072)
        rows = rng.choice([1, 1, rng.randint(2, 8), size(9, 4608)]) if kind in ("attend", "step", "append") else size(1, 36864)
        rows = min(rows, _augmented(n, c, m))
        case = _case(None, kind, batch, heads, kv_heads, d, n, rows, c, m, C, rng.choice([16, 32, 64, 64, 128]), kind not in ("append", "step") and rng.random() < 0.5,
                     batch > 1 and rng.random() < 0.6)
        seen = _lists(case)
        room = batch * max(x["n_sum"] + x["n_txt"] for x in seen)
        scores = room * case["rows"] * heads
        if work(case)["flops"] > 2e12 or work(case)["bytes"] > 2e9 or scores > 4e9 or room * kv_heads * d > 1.1e9:
            continue
        if kind not in ("attend", "step") and sum(_starts(case)[1]) * kv_heads * d > 2e8:
            continue
        return case


# ---- sizes, on the host -------------------------------------------------------------------------------------------------

def _augmented(n, c, m):
    return n // c * (c + m) + n % c


def _starts(case):
    """First new row (augmented) and number of new rows of every sequence."""
    B, L, rows = case["batch"], _augmented(case["n"], case["c"], case["m"]), case["rows"]
    start, count = [], []
    for b in range(B):
        k, end = rows, L
        if case["ragged"]:
            k = max(1, rows - rows * 3 * b // (4 * B) if b % 2 == 0 else rows // 4 ** min(b, 20))
            end = max(k, L * (B + 3 * ((5 * b) % B) + 3) // (4 * B) - 11 * b)
        if case["kind"] in ("write", "read"):
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


def work(case):
    H, Hkv, d, fp8 = case["heads"], case["kv_heads"], case["d"], case["fp8"]
    total = sum(_starts(case)[1])
    held = 2 * Hkv * (d + 1 if fp8 else 2 * d)           # bytes of a row in the cache, K and V
    plain = 2 * Hkv * 2 * d                              # ... of a new row
    move = total * (held + plain)
    if case["kind"] == "append" or case["kind"] == "read":
        return {"bytes": move, "flops": 0}
    if case["kind"] == "write":
        return {"bytes": 2 * move, "flops": 0}
    v = _lists(case)
    read = sum(x["sums"] + x["n_txt"] for x in v) * held + total * H * (4 * d + 4)
    return {"bytes": read + (move if case["kind"] == "step" else 0), "flops": 4 * d * H * sum(x["pairs"] for x in v)}


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _split(x):
    """e4m3 values and biased exponents of rows x (last dimension), as the cache holds them."""
    most = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    f, e = torch.frexp(most)                             # most = f 2^e, 0.5 <= f < 1; 448 = 0.875 * 2^9
    e = torch.where(most > 0, e - 9 + (f > 0.875).to(e.dtype), -117).clamp(-117, 119)
    y = torch.where(torch.isfinite(x), torch.ldexp(x, -e[..., None]), float("nan"))
    return y.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def prepare(case, seed):
    B, Hq, Hkv, d, c, m, page = (case[x] for x in ("batch", "heads", "kv_heads", "d", "c", "m", "page"))
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    g = torch.Generator(device=dev).manual_seed(seed)
    start, count = _starts(case)
    lists = _lists(case)

    # Pages for what the new rows see and for the rows themselves; text that has left the window has none any more (-1).
    whole = case["kind"] not in ("attend", "step")
    n_text = max(_text_of(a + k, c, m) for a, k in zip(start, count))
    cols_t, cols_s = -(-n_text // page), max(-(-max(a + k for a, k in zip(start, count)) // page), 1) if m else 0
    first_t = torch.tensor([_text_of(a, c, m) if whole else x["t0"] for a, x in zip(start, lists)]) // page
    last_t = torch.tensor([max(-(-_text_of(a + k, c, m) // page), -(-(x["t0"] + x["n_txt"]) // page)) for a, k, x in zip(start, count, lists)])
    ends = [a + k - _text_of(a + k, c, m) for a, k in zip(start, count)]
    first_s = torch.tensor([a - _text_of(a, c, m) if whole else 0 for a in start]) // page
    last_s = torch.tensor([-(-x // page) for x in ends])
    cols_s = min(cols_s, max(int(last_s.max()), 1)) if m else 0

    def table(first, last, cols, base):
        need = (torch.arange(cols) >= first[:, None]) & (torch.arange(cols) < last[:, None])
        t = torch.full((B, cols), -1, dtype=torch.int32)
        t[need] = base + torch.arange(int(need.sum()), dtype=torch.int32)
        return t, base + int(need.sum())

    text_table, used = table(first_t, last_t, cols_t, 0)
    sum_table, used = table(first_s, last_s, cols_s, used) if m else (None, used)
    n_pages = used + 3
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)     # a pool that has been in use: pages in any order

    def placed(t):
        t = t.to(dev)
        return torch.where(t >= 0, order[t.clamp(min=0).long()], -1).to(torch.int32).contiguous()

    def rows_of(*shape):
        x = torch.randn(*shape, d, generator=g, device=dev)
        return x * torch.exp2(0.5 * torch.randn(*shape, 1, generator=g, device=dev))

    s = dict(case=case, text_table=placed(text_table), sum_table=placed(sum_table) if m else None, k_exp=None, v_exp=None)
    for x in ("k", "v"):
        pool = rows_of(n_pages, Hkv, page)
        if case["fp8"]:
            s[x], s[x + "_exp"] = _split(pool.to(torch.bfloat16).float())
        else:
            s[x] = pool.to(torch.bfloat16)
        del pool
    total = sum(count)
    if case["kind"] in ("attend", "step"):
        s["q"] = torch.randn(total, Hq, d, generator=g, device=dev).to(torch.bfloat16)
    if case["kind"] in ("step", "append", "write"):
        s["k_new"], s["v_new"] = rows_of(total, Hkv).to(torch.bfloat16), rows_of(total, Hkv).to(torch.bfloat16)
    cu = [0]
    for k in count:
        cu.append(cu[-1] + k)
    s["cu_rows"] = torch.tensor(cu, dtype=torch.int32, device=dev)
    s["start"] = torch.tensor(start, dtype=torch.int32, device=dev)
    s["row_seq"] = torch.repeat_interleave(torch.arange(B), torch.tensor(count)).to(dev)      # the sequence of a packed row
    s["row_at"] = torch.arange(total, device=dev) - s["cu_rows"].long()[s["row_seq"]]         # ... and its place among the sequence's
    s["n_sum"], s["n_txt"] = max(x["n_sum"] for x in lists), max(x["n_txt"] for x in lists)
    s["t0"] = torch.tensor([x["t0"] for x in lists], device=dev)
    if own:      # the handle of the cache and the scratch memory that a serving program keeps
        import paper_2604_24432_amd as K
        p = K.make_params(B, case["n"], c, m, case["C"], Hq, Hkv, d)
        s["cache"] = K.PagedCache(p, s["k"], s["v"], s["text_table"], s["sum_table"], s["k_exp"], s["v_exp"])
        if "q" in s:
            s["workspace"] = torch.empty(max(K.paged_workspace_bytes(s["cache"], total, case["rows"]), 1), dtype=torch.uint8, device=dev)
    return s


def _text_of(a, c, m):
    """Text rows among the first a augmented rows."""
    return a // (c + m) * c + min(a % (c + m), c)


# ---- one pass -----------------------------------------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if own:
        import paper_2604_24432_amd as K
        if kind in ("step", "append", "write"):
            K.ksa_paged_append(s["cache"], s["k_new"], s["v_new"], s["cu_rows"], s["start"])
        if kind in ("write", "read"):
            return K.ksa_paged_read(s["cache"], s["cu_rows"], s["start"], len(s["row_seq"]))
        if kind == "append":
            return s["k"], s["v"]
        o, lse = K.ksa_paged_fwd(s["cache"], s["q"], s["cu_rows"], s["start"], max_rows=s["case"]["rows"], workspace=s["workspace"])
        return (o, lse) if kind == "attend" else (o, lse, s["k"], s["v"])
    if kind in ("step", "append", "write"):
        _plain_append(s)
    if kind in ("write", "read"):
        return _plain_read(s)
    if kind == "append":
        return s["k"], s["v"]
    o, lse = _plain_attend(s)
    return (o, lse) if kind == "attend" else (o, lse, s["k"], s["v"])


def _places(s):
    """Page and slot of every packed row."""
    c, m, page = s["case"]["c"], s["case"]["m"], s["case"]["page"]
    a = s["start"].long()[s["row_seq"]] + s["row_at"]
    j, r = a // (c + m), a % (c + m)
    i, u = j * c + r.clamp(max=c - 1), j * m + (r - c).clamp(min=0)
    at = s["text_table"][s["row_seq"], i // page]
    if m == 0:
        return at.long(), i % page
    text = r < c
    u = torch.where(text, 0, u)
    return torch.where(text, at, s["sum_table"][s["row_seq"], u // page]).long(), torch.where(text, i % page, u % page)


def _plain_append(s):
    at, slot = _places(s)
    if s["case"]["fp8"]:
        for x in ("k", "v"):
            y, e = _split(s[x + "_new"].float())
            s[x].view(torch.uint8)[at, :, slot] = y.view(torch.uint8)
            s[x + "_exp"][at, :, slot] = e
    else:
        s["k"][at, :, slot] = s["k_new"]
        s["v"][at, :, slot] = s["v_new"]


def _values(s, x, at, slot):
    """What rows (page at, slot) of k or v stand for, float32 [..., Hkv, d]."""
    if not s["case"]["fp8"]:
        return s[x][at, :, slot].float()
    y = s[x].view(torch.uint8)[at, :, slot].view(torch.float8_e4m3fn).float()
    return torch.ldexp(y, s[x + "_exp"][at, :, slot].int()[..., None] - 127)


def _plain_read(s):
    at, slot = _places(s)
    return _values(s, "k", at, slot).to(torch.bfloat16), _values(s, "v", at, slot).to(torch.bfloat16)


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
    k = _values(s, "k", at, slot).permute(0, 2, 1, 3).contiguous()                                            # [B, Hkv, N, d]
    q = torch.zeros(B, T, Hq, d, device=dev)
    q[s["row_seq"], s["row_at"]] = s["q"].float()
    q = q.view(B, T, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, d)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(1 / math.sqrt(d)).view(B, Hkv, T, G, -1)
    del k
    x.masked_fill_(~seen[:, None, :, None], -math.inf)
    most = x.amax(-1, keepdim=True)
    x.sub_(most).exp_()
    total = x.sum(-1, keepdim=True)
    v = _values(s, "v", at, slot).permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(x.view(B, Hkv, T * G, -1), v).view(B, Hkv, T, G, d) / total
    lse = (most + total.log())[..., 0]
    o = o.permute(0, 2, 1, 3, 4).reshape(B, T, Hq, d)[s["row_seq"], s["row_at"]]
    return o.to(torch.bfloat16), lse.permute(0, 2, 1, 3).reshape(B, T, Hq)[s["row_seq"], s["row_at"]]


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------

def _e4m3(x):
    """float64 values of x (finite rows) as the 8-bit cache holds them: round to nearest even with 4 significant bits, 2^-9 at the least."""
    most = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(most, -117)
    for k in range(-116, 120):
        e = torch.where(most > 448.0 * 2.0 ** (k - 1), float(k), e)
    y = x * torch.exp2(-e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * torch.exp2(e)


def exact(case, seed):
    s = prepare(case, seed)
    c, m, C, page, fp8, G = case["c"], case["m"], case["C"], case["page"], case["fp8"], case["heads"] // case["kv_heads"]
    start, count = _starts(case)

    def held(x):
        y = s[x].double()
        return y * torch.exp2(s[x + "_exp"].double() - 127)[..., None] if fp8 else y

    pool = {x: held(x) for x in ("k", "v")} if case["kind"] != "write" else None

    def place(b, a):      # page and slot of augmented row a
        j, r = divmod(a, c + m)
        x, t = (j * c + r, s["text"]) if r < c else (j * m + r - c, s["sums"])
        return t[b][x // page], x % page

    s["text"], s["sums"] = s["text_table"].tolist(), s["sum_table"].tolist() if m else None
    where = [place(b, a) for b in range(case["batch"]) for a in range(start[b], start[b] + count[b])]
    pages, slots = torch.tensor([x[0] for x in where], device=s["k"].device), torch.tensor([x[1] for x in where], device=s["k"].device)
    if case["kind"] in ("step", "append", "write"):
        new = {x: _e4m3(s[x + "_new"].double()) if fp8 else s[x + "_new"].double() for x in ("k", "v")}
        if case["kind"] == "write":
            return new["k"], new["v"]
        for x in ("k", "v"):
            pool[x][pages, :, slots] = new[x]
    if case["kind"] == "append":
        return pool["k"], pool["v"]
    if case["kind"] == "read":
        return pool["k"][pages, :, slots], pool["v"][pages, :, slots]

    outs, lses, at = [], [], 0
    for b in range(case["batch"]):
        v = torch.tensor([_seen(a, case) for a in range(start[b], start[b] + count[b])], device=s["k"].device)
        hi_s, lo_t, hi_t = int(v[:, 1].max()), int(v[:, 2].min()), int(v[:, 3].max())
        us, ts = torch.arange(hi_s, device=v.device), torch.arange(lo_t, hi_t, device=v.device)
        pg = s["text_table"][b].long()[ts // page]
        if hi_s:
            pg = torch.cat([s["sum_table"][b].long()[us // page], pg])
        sl = torch.cat([us, ts]) % page
        mask = torch.cat([(us >= v[:, :1]) & (us < v[:, 1:2]), (ts >= v[:, 2:3]) & (ts < v[:, 3:4])], 1)       # [rows, N]
        q = s["q"][at:at + count[b]].double()
        at += count[b]
        o, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float64, device=q.device)
        for h in range(case["kv_heads"]):
            k_h, v_h = pool["k"][pg, h, sl], pool["v"][pg, h, sl]
            for r0 in range(0, count[b], 1024):
                part = slice(r0, r0 + 1024)
                for x in range(h * G, h * G + G):
                    z = (q[part, x] @ k_h.T / math.sqrt(case["d"])).masked_fill(~mask[part], -math.inf)
                    lse[part, x] = torch.logsumexp(z, 1)
                    o[part, x] = torch.softmax(z, 1) @ v_h
        outs.append(o), lses.append(lse)
    o, lse = torch.cat(outs), torch.cat(lses)
    return (o, lse) if case["kind"] == "attend" else (o, lse, pool["k"], pool["v"])
