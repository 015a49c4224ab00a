"""GPU tests of a step's rows and pages from the sequences' lengths: every table entry, count and row map against a model in Python (tests/advance.py), and a
generate loop of all the paged operators together."""
import random

import pytest
import torch

import paper_2604_24432_amd as K
from tests.advance import advance
from tests.paged import attend, randn, stands_for
from tests.paged_fp4 import e2m1
from tests.rotary import frequencies, positions, turn
from tests.test_gpu_paged import bits, say

pytestmark = pytest.mark.gpu


class Books:
    """Tables and counts on the GPU and in Python."""

    def __init__(self, batch, n, c, m, C, page, n_pages, cols=None, garbage=False):
        self.shape = c, m, C, page, n
        self.p = K.make_params(batch, n, c, m, C, 1, 1, 64)
        ct, cs = cols or (-(-n // page), max(-(-(n // c * m) // page), 1))
        empty = -1 if not garbage else n_pages + 5                          # entries that are no page
        self.text, self.sums, self.refs = [[empty] * ct for _ in range(batch)], [[empty] * cs for _ in range(batch)], [0] * n_pages
        pool = torch.zeros(n_pages, 1, page, 64, dtype=torch.bfloat16, device="cuda")
        self.cache = K.PagedCache(self.p, pool, pool, self.dev(self.text), self.dev(self.sums) if m else None)
        self.refs_dev = self.dev(self.refs)
        if not m:
            self.sums = [[] for _ in range(batch)]

    @staticmethod
    def dev(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    def upload(self):
        self.cache.text_table.copy_(self.dev(self.text)), self.refs_dev.copy_(self.dev(self.refs))
        if self.cache.summary_table is not None:
            self.cache.summary_table.copy_(self.dev(self.sums))

    def check(self, step, want, total):
        cu, start, lacking, rows = want
        assert step.cu_rows.tolist() == cu and step.start.tolist() == start and step.lacking.tolist() == [lacking]
        assert self.cache.text_table.tolist() == self.text and self.refs_dev.tolist() == self.refs
        assert self.cache.summary_table is None or self.cache.summary_table.tolist() == self.sums
        rows = rows[:total] + [(-1, 0, -1)] * (total - len(rows))
        assert step.slots.tolist() == [r[0] for r in rows]
        assert step.positions.tolist() == [r[1] for r in rows]
        assert step.tokens.tolist() == [r[2] for r in rows]

    def step(self, held, new, total=None, **more):
        want = advance(*self.shape, self.text, self.sums, self.refs, held, new)
        total = len(want[3]) + 5 if total is None else total
        step = K.ksa_paged_advance(self.cache, self.refs_dev, self.dev(held), self.dev(new), total, **more)
        self.check(step, want, total)
        return step


# batch, text tokens, c, m, C, page, pages, most new tokens
LOOPS = [(1, 300, 8, 1, 2, 8, 100, 1), (5, 400, 16, 4, 0, 8, 24, 90), (7, 500, 12, 3, 1, 16, 400, 200), (3, 300, 1, 0, 30, 8, 200, 20), (40, 2000, 64, 8, 1, 64, 300, 700),
         (300, 200, 8, 8, 1, 8, 9000, 40), (3, 5000, 64, 0, 4096, 16, 5000, 3000), (2, 100, 200, 8, 1, 8, 30, 30)]


@pytest.mark.parametrize("case", LOOPS, ids=str)
def test_loops_of_steps(case):
    """Sequences grow by tokens and by pieces of prompts, wait, end and begin again; the pool runs out in some."""
    B, n, c, m, C, page, n_pages, most = case
    say(f"advance loop {case}")
    g = random.Random(str(case))
    books = Books(B, n, c, m, C, page, n_pages)
    held, ran_out = [0] * B, 0
    for i in range(25):
        new = [min(g.choice([1, 1, 1, 0, g.randint(1, most), -1]), n - h) for h in held]
        if i == 20:
            new[0], held[0] = 1, g.choice([-3, n])                          # out of place
        step = books.step(held, new)
        ran_out += int(step.lacking)
        held = [0 if t < 0 or not 0 <= h <= n - t else h + t for h, t in zip(held, new)]
        if g.random() < 0.3:
            books.step([h if t >= 0 else 0 for h, t in zip(held, new)], [0 if t >= 0 else -1 for t in new])
    assert n_pages != 24 or ran_out > 0


@pytest.mark.parametrize("B,n", [(2500, 3000), (5000, 700)])
def test_many_sequences_and_many_pages(B, n):
    """Counts added up by every workgroup, and from 4096 sequences on by one for all."""
    say(f"advance large {B}")
    g = random.Random(4)
    books = Books(B, n, 64, 8, 1, 64, 70001)
    held = [0] * B
    for most in (n, 1, 1, n // 6):
        new = [min(g.choice([0, 1, g.randint(1, most), -1 if held[0] else 1]), n - h) for h in held]
        books.step(held, new)
        held = [0 if t < 0 else h + t for h, t in zip(held, new)]


def test_one_long_sequence_takes_scattered_pages():
    say("advance scattered")
    g = random.Random(5)
    books = Books(1, 100000, 64, 8, 1, 8, 40000)
    for x in g.sample(range(40000), 24000):
        books.refs[x] = g.choice([1, 2, -1])
    books.upload()
    books.step([0], [100000])
    assert books.refs.count(0) > 0
    books.step([100000], [0])
    books.step([100000], [-1])


def test_shared_prompts():
    """Two sequences name the pages of one prompt: they stay until the last one gives them back."""
    say("advance shared")
    c, m, C, page = 16, 2, 1, 16
    books = Books(3, 400, c, m, C, page, 80)
    books.step([0, 0, 0], [128, 0, 0])
    books.text[1], books.sums[1] = list(books.text[0]), list(books.sums[0])
    for x in books.text[0] + books.sums[0]:
        if x >= 0:
            books.refs[x] += 1
    books.upload()
    books.step([128, 128, 0], [5, 40, 1])
    books.step([133, 168, 1], [1, -1, 7])
    books.step([134, 0, 8], [-1, 3, 1])
    assert sum(books.refs) == sum(x >= 0 for t in books.text + books.sums for x in t)


def test_entries_that_are_no_pages_narrow_tables_and_short_maps():
    say("advance odd tables")
    books = Books(4, 600, 16, 4, 2, 8, 100, cols=(20, 4), garbage=True)
    books.step([0, 10, 100, 0], [300, 30, 7, 0], total=100)                 # more rows than the maps hold, rows behind the last column
    books.step([300, 40, 107, 0], [1, 1, 1, 1], total=0)
    books.step([301, 41, 108, 1], [-1, 0, 492, 10], total=700)


def test_graph_replays_and_streams():
    say("advance graph")
    c, m, C, page, n, B = 16, 2, 1, 16, 300, 5
    books = Books(B, n, c, m, C, page, 60)
    held, new = books.dev([0] * B), books.dev([0] * B)
    total = 200
    ws = torch.empty(K.paged_advance_workspace_bytes(books.cache), dtype=torch.uint8, device="cuda")
    step = K.ksa_paged_advance(books.cache, books.refs_dev, held, new, total, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        K.ksa_paged_advance(books.cache, books.refs_dev, held, new, total, step=step, workspace=ws)
        held.add_(new.clamp(min=0))
    lengths = [0] * B
    g = random.Random(3)
    for i in range(12):
        t = [min(g.choice([0, 1, g.randint(1, 30)]), n - h) for h in lengths]
        if i == 6:
            t[2] = -1
        new.copy_(books.dev(t))
        want = advance(*books.shape, books.text, books.sums, books.refs, lengths, t)
        graph.replay()
        torch.cuda.synchronize()
        books.check(step, want, total)
        books.refs_dev.clone(), torch.cuda.synchronize()
        lengths = [h + max(x, 0) for h, x in zip(lengths, t)]
        if i == 6:
            lengths[2] = 0
            held[2] = 0
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    t = [min(3, n - h) for h in lengths]
    want = advance(*books.shape, books.text, books.sums, books.refs, lengths, t)
    other = K.ksa_paged_advance(books.cache, books.refs_dev, held, books.dev(t), 50, stream=stream)
    stream.synchronize()
    books.check(other, want, 50)


@pytest.mark.parametrize("kind", ["bf16", "fp8", "fp4"])
def test_a_generate_loop_of_all_operators(kind):
    """Lengths -> rows and pages -> q and k turned, k and v into pages -> attention: prompts, drafted tokens, single tokens, sequences that end and others that
    begin in their pages; every row's output against the definition over its whole sequence, every step replayed from a graph."""
    say(f"advance generate {kind}")
    c, m, C, page, n, B, Hq, Hkv, d = 16, 2, 2, 16, 400, 3, 8, 2, 128
    p = K.make_params(B, n, c, m, C, Hq, Hkv, d)
    rule = dict(dim=64, base=1e6, scaling="by_parts", factor=4.0, original=128.0)
    r = K.Rotary(64, base=1e6, scaling="by_parts", factor=4.0, original=128.0)
    n_pages, room, most = 40, 240, 150
    text, sums = torch.full((B, -(-n // page)), -1, dtype=torch.int32, device="cuda"), torch.full((B, -(-(n // c * m) // page)), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    if kind == "fp4":
        pools = [torch.full((n_pages, Hkv, page, d // 2), 0x77, dtype=torch.uint8, device="cuda") for _ in range(2)]
        exps = [torch.full((n_pages, Hkv, page, d // 32), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    else:
        pools = [torch.full((n_pages, Hkv, page, d), float("nan"), device="cuda").to(torch.float8_e4m3fn if kind == "fp8" else torch.bfloat16) for _ in range(2)]
        exps = [torch.full((n_pages, Hkv, page), 255, dtype=torch.uint8, device="cuda") for _ in range(2)] if kind == "fp8" else [None, None]
    cache = K.PagedCache(p, *pools, text, sums, *exps)
    held, new = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    q, k, v = (torch.zeros(room, h, d, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    q_out, o, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(room, Hq, device="cuda")
    aws = torch.empty(K.paged_advance_workspace_bytes(cache), dtype=torch.uint8, device="cuda")
    ws = {most_: torch.empty(max(K.paged_workspace_bytes(cache, room, most_), 1), dtype=torch.uint8, device="cuda") for most_ in (8, room)}
    step = K.ksa_paged_advance(cache, refs, held, new, room, workspace=aws)

    def run(most_):
        K.ksa_paged_advance(cache, refs, held, new, room, step=step, workspace=aws)
        K.ksa_paged_rotary(cache, r, q, k, v, step.cu_rows, step.start, q_out=q_out)
        K.ksa_paged_fwd(cache, q_out, step.cu_rows, step.start, max_rows=most_, o=o, lse=lse, workspace=ws[most_])

    side = torch.cuda.Stream()
    graphs = {}
    for most_ in (8, room):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run(most_)
        torch.cuda.current_stream().wait_stream(side)
        graphs[most_] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[most_]):
            run(most_)
    lengths, seqs = [0] * B, [([], []) for _ in range(B)]
    plan = [[100, 33, 0], [1, 1, 50], [1, 6, 1], [7, 1, 1], [1, -1, 1], [1, 130, 1], [1, 1, 7], [-1, 1, 1], [60, 1, 1], [1, 1, 1]]
    for i, t in enumerate(plan):
        held.copy_(torch.tensor(lengths, dtype=torch.int32)), new.copy_(torch.tensor(t, dtype=torch.int32))
        for x, s in ((q, 1), (k, 2), (v, 3)):
            x.copy_(randn(*x.shape, seed=100 * i + s))
        aug = [(h + h // c * m, h + max(x, 0) + (h + max(x, 0)) // c * m) for h, x in zip(lengths, t)]
        few = max(b - a for a, b in aug) <= 8
        o.fill_(7.0)
        graphs[8 if few else room].replay()
        torch.cuda.synchronize()
        assert int(step.lacking) == 0
        at = 0
        for b in range(B):
            if t[b] < 0:
                seqs[b], lengths[b] = ([], []), 0
                continue
            first, end = aug[b]
            rows, pos = slice(at, at + end - first), positions(range(first, end), c, m)
            assert step.positions[rows].tolist() == pos.tolist()
            if end > first:
                # what the cache holds is exactly what it stands for of the turned rows, rounded to bf16; those within a rounding of a border are taken from the cache
                kb, vb = K.ksa_paged_read(cache, step.cu_rows, step.start, room)
                want_k, off = turn(k[rows].double(), rule, pos)
                held_as = (lambda x: e2m1(x)[0]) if kind == "fp4" else (lambda x: stands_for(x.to(torch.bfloat16), kind == "fp8"))
                group = 32 if kind == "fp4" else d
                near = (kb[rows].double() - held_as(want_k.to(torch.bfloat16).double())).abs()
                step_of = want_k.abs().unflatten(-1, (-1, group)).amax(-1).repeat_interleave(group, -1)
                # (a value next to a border may go to the other side: a whole step of the format at most, with all of its group's where the exponent changes)
                assert bool((near <= off + step_of * (0.5 if kind == "fp4" else 0.125 if kind == "fp8" else 0.0)).all()) and float((near > off).double().mean()) < 0.02
                assert torch.equal(vb[rows].double(), held_as(v[rows].double()))
                seqs[b][0].append(kb[rows].double()), seqs[b][1].append(vb[rows].double())
                ks, vs = torch.cat(seqs[b][0]), torch.cat(seqs[b][1])
                qs, q_off = turn(q[rows].double(), rule, pos)
                assert bool(((q_out[rows].double() - qs).abs() <= q_off).all())
                want, want_lse, o_off, lse_off = attend(q_out[rows].double(), ks, vs, list(range(first, end)), p)
                assert bool(((o[rows].double() - want).abs() <= o_off + ks.shape[0] * 2.0 ** -119 * float(vs.abs().max())).all()), (i, b)
                assert bool(((lse[rows].double() - want_lse).abs() <= lse_off).all()), (i, b)
            at += end - first
            lengths[b] += t[b]
        assert bool((o[at:] == 7).all())                                   # rows behind the last sequence
    assert int((refs > 0).sum()) < n_pages and frequencies(rule)[1] > 1


def test_python_refuses_what_does_not_fit():
    books = Books(2, 100, 16, 2, 1, 16, 30)
    i32 = books.dev([0, 0])
    good = (books.cache, books.refs_dev, i32, i32, 5)
    step = K.ksa_paged_advance(*good)
    for at, bad in ((1, books.refs_dev[:-1]), (1, books.refs_dev.long()), (2, i32[:1]), (2, i32.float()), (3, i32.cpu()), (3, torch.stack([i32, i32], 1)[:, 0]), (4, -1)):
        args = list(good)
        args[at] = bad
        with pytest.raises(ValueError):
            K.ksa_paged_advance(*args)
    with pytest.raises(ValueError):
        K.ksa_paged_advance(*good[:4], 6, step=step)
    with pytest.raises(ValueError):
        K.ksa_paged_advance(*good, step=step._replace(slots=step.slots.int()))
    with pytest.raises(ValueError):
        K.ksa_paged_advance(*good, workspace=torch.empty(100, device="cuda"))
    with pytest.raises(K.KsaError):
        K.ksa_paged_advance(*good, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert bits(torch.zeros(1, dtype=torch.bfloat16)).item() == 0


def test_two_graphs_share_a_workspace():
    """Two batches' steps captured with one workspace, replayed in turn: each as alone."""
    say("advance two graphs")
    a, b = Books(5, 300, 16, 2, 1, 16, 60), Books(9, 500, 64, 8, 1, 32, 200)
    ws = torch.empty(max(K.paged_advance_workspace_bytes(x.cache) for x in (a, b)), dtype=torch.uint8, device="cuda")
    made = []
    for books, total in ((a, 100), (b, 300)):
        n = len(books.text)
        held, new = books.dev([0] * n), books.dev([0] * n)
        step = K.ksa_paged_advance(books.cache, books.refs_dev, held, new, total, workspace=ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            K.ksa_paged_advance(books.cache, books.refs_dev, held, new, total, step=step, workspace=ws)
        made.append((books, total, held, new, step, graph, [0] * n))
    g = random.Random(8)
    for _ in range(6):
        wants = []
        for books, total, held, new, step, graph, lengths in made:
            t = [min(g.choice([0, 1, g.randint(1, 60)]), books.shape[4] - h) for h in lengths]
            held.copy_(books.dev(lengths)), new.copy_(books.dev(t))
            wants.append(advance(*books.shape, books.text, books.sums, books.refs, lengths, t))
            lengths[:] = [h + x for h, x in zip(lengths, t)]
        for books, total, held, new, step, graph, lengths in made:
            graph.replay()
        torch.cuda.synchronize()
        for (books, total, held, new, step, graph, lengths), want in zip(made, wants):
            books.check(step, want, total)


@pytest.mark.parametrize("batch", [3, 5, 4099])
def test_more_rows_than_32_bits_in_a_step_whose_maps_are_short(batch):
    say(f"advance rows beyond 32 bits, {batch}")
    n, c, m, page, total, some = 2 ** 29, 16, 4, 8, 40, 6
    p = K.make_params(batch, n, c, m, 2, 1, 1, 64)
    L = n + n // c * m                                                      # of a sequence: 3 and more of them pass 2^31 - 256
    pool = torch.zeros(40, 1, page, 64, dtype=torch.bfloat16, device="cuda")
    text, sums = (torch.full((batch, cols), -1, dtype=torch.int32, device="cuda") for cols in (4, 2))
    refs = torch.zeros(40, dtype=torch.int32, device="cuda")
    cache = K.PagedCache(p, pool, pool, text, sums)
    held, new = (torch.full((batch,), x, dtype=torch.int32, device="cuda") for x in (0, n))
    step = K.ksa_paged_advance(cache, refs, held, new, total)
    assert step.cu_rows.tolist() == [min(b * L, 2 ** 31 - 1) for b in range(batch + 1)] and step.start.tolist() == [0] * batch
    assert step.lacking.tolist() == [max(batch * 6 - 40, 0)]
    got = torch.cat([text, sums], 1)[:some].tolist()
    assert got == [[6 * b + x if 6 * b + x < 40 else -1 for x in range(6)] for b in range(min(batch, some))]
    want = []
    for row in range(total):                                                # all of the first sequence
        j, r = divmod(row, c + m)
        idx = j * c + r if r < c else j * m + r - c
        col, at = idx // page, idx % page
        want.append((((col if r < c else 4 + col) * page + at) if col < (4 if r < c else 2) else -1, j * c + min(r, c - 1), idx if r < c else c - 1 - r))
    assert list(zip(step.slots.tolist(), step.positions.tolist(), step.tokens.tolist())) == want


@pytest.mark.parametrize("last", [16 * 6710886 + 7, 16 * 6710886 + 8, 2 ** 29])
def test_the_last_sequence_alone_is_beyond_32_bits(last):
    """Three sequences' rows fit 32 bits; with the fourth's there are 2^31 - 1, one more, or many more."""
    say(f"advance last sequence beyond 32 bits, {last}")
    n, c, m, page, total, batch = 2 ** 29, 16, 4, 8, 24, 4
    p = K.make_params(batch, n, c, m, 2, 1, 1, 64)
    L, last_rows = n + n // c * m, last + last // c * m
    assert 3 * L < 2 ** 31 - 256 and 3 * L + last_rows - (2 ** 31 - 1) in (0, 1, 4 * L - (2 ** 31 - 1))
    pool = torch.zeros(40, 1, page, 64, dtype=torch.bfloat16, device="cuda")
    text, sums = (torch.full((batch, cols), -1, dtype=torch.int32, device="cuda") for cols in (4, 2))
    refs = torch.zeros(40, dtype=torch.int32, device="cuda")
    cache = K.PagedCache(p, pool, pool, text, sums)
    held, new = torch.zeros(batch, dtype=torch.int32, device="cuda"), torch.tensor([n, n, n, last], dtype=torch.int32, device="cuda")
    step = K.ksa_paged_advance(cache, refs, held, new, total)
    assert step.cu_rows.tolist() == [0, L, 2 * L, 3 * L, min(3 * L + last_rows, 2 ** 31 - 1)] and step.start.tolist() == [0] * batch
    assert step.lacking.tolist() == [0] and refs.tolist() == [1] * 24 + [0] * 16
    assert torch.cat([text, sums], 1).tolist() == [[6 * b + x for x in range(6)] for b in range(batch)]
    want = []
    for row in range(total):                                                # all of the first sequence
        j, r = divmod(row, c + m)
        idx = j * c + r if r < c else j * m + r - c
        col, at = idx // page, idx % page
        want.append((((col if r < c else 4 + col) * page + at) if col < (4 if r < c else 2) else -1, j * c + min(r, c - 1), idx if r < c else c - 1 - r))
    assert list(zip(step.slots.tolist(), step.positions.tolist(), step.tokens.tolist())) == want
