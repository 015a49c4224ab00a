"""How ksa_paged_fwd deals a call to workgroups (plan_paged in ksa_paged_api.cpp; no GPU needed)."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_24432_amd", "csrc")
INVALID, TOO_SMALL = -1, -3


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """Of a list of (batch, heads, KV heads, d, tokens, c, m, C, new rows, most of a sequence, spans, bytes of workspace or -1)."""
    exe = str(tmp_path_factory.mktemp("plan") / "paged_plan")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    os.path.join(ROOT, "tests", "plan", "paged_plan.cpp"), os.path.join(CSRC, "ksa_paged_api.cpp"), os.path.join(CSRC, "ksa_layout.cpp"),
                    "-o", exe], check=True)

    def run(calls):
        out = subprocess.run([exe], input="\n".join(" ".join(map(str, c)) for c in calls), capture_output=True, text=True)
        assert out.returncode == 0, out.stderr[-2000:]
        return [dict(zip(("status", "few", "n_splits", "pairs", "groups", "slots", "bytes"), map(int, line.split()))) for line in out.stdout.splitlines()]
    return run


def random_calls(count, seed):
    rng = random.Random(seed)
    for _ in range(count):
        c, m, C = rng.choice([(64, 8, 1), (8, 1, 128), (16, 2, 64), (48, 6, 2), (1, 0, 1023), (64, 0, 4096)])
        kv_heads = rng.choice([1, 2, 3, 4, 8, 16])
        batch, most = rng.choice([1, 1, 2, 3, 8, 16, 64, 150]), rng.choice([1, 1, 4, 8, 33, 300, 2048])
        yield (batch, kv_heads * rng.choice([1, 2, 4, 8]), kv_heads, rng.choice([64, 128]), int(10 ** rng.uniform(2.5, 5.5)), c, m, C,
               rng.randint(1, batch * most), most, 0, -1)


def test_a_smaller_workspace_means_fewer_spans(plans):
    """A call that leaves the spans to the library takes any workspace: one sized for another call's rows, the least, none at all."""
    rng = random.Random(1)
    calls = list(random_calls(3000, 1))
    asked = plans(calls)
    assert all(x["status"] == 0 for x in asked) and sum(x["n_splits"] > 1 for x in asked) > 500
    for given in (lambda n: 0, lambda n: n // 2, lambda n: n - 1, lambda n: rng.randint(0, n), lambda n: n, lambda n: 2 * n + 100):
        sizes = [given(x["bytes"]) for x in asked]
        for c, want, size, got in zip(calls, asked, sizes, plans([(*c[:-1], max(n, 0)) for c, n in zip(calls, sizes)])):
            per_span = c[8] * c[1] * (c[3] + 4) * 4
            assert got["status"] == 0, (c, size, got)
            assert got["n_splits"] == 1 or got["n_splits"] * per_span <= size
            if size >= want["bytes"]:
                assert got == want
            elif got["few"]:
                assert got["n_splits"] == max(1, size // per_span)     # as many as it holds


def test_one_workspace_for_all_batches_of_a_serving_loop(plans):
    """64K tokens, 8 sequences: 8192 rows need no workspace, 512 and 64 would have some."""
    many, some, few = plans([(8, 32, 8, 128, 65536, 64, 8, 1, n, 2048, 0, -1) for n in (8192, 512, 64)])
    assert many["bytes"] == 0 < few["bytes"] < some["bytes"]
    for n in (512, 64):
        for size in (0, few["bytes"]):
            got, = plans([(8, 32, 8, 128, 65536, 64, 8, 1, n, 2048, 0, size)])
            assert got["status"] == 0


def test_a_number_of_spans_that_was_asked_for_needs_its_workspace(plans):
    for n, bytes_of in ((2, 64 * 32 * 2 * 132 * 4), (1024, 64 * 32 * 1024 * 132 * 4)):
        call = (64, 32, 8, 128, 4096, 64, 8, 1, 64, 1, n)
        exact, less, none = plans([(*call, bytes_of), (*call, bytes_of - 1), (*call, 0)])
        assert (exact["status"], less["status"], none["status"]) == (0, TOO_SMALL, INVALID) and exact["n_splits"] == n


def test_chunks_longer_than_any_text(plans):
    """c + m beyond 32 bits: as with chunks that are a little longer than the text (the host code runs under UBSan here)."""
    most = 2 ** 31 - 1
    for n, rows in ((100, 50), (100, 1), (5000, 300)):
        for d in (64, 128):
            calls = [(1, 4, 2, d, n, c, m, 1, rows, rows, 0, -1) for c, m in ((10 ** 9, 10 ** 9), (most, most), (10 ** 9, 10 ** 9 // 2), (most - 1, most // 2))]
            got = plans(calls)
            assert got[0] == got[1] and got[2] == got[3] and got[0]["status"] == got[2]["status"] == 0


def test_the_gpu_tests_reach_every_kernel(plans):
    """Which kernel a call takes is a matter of measured constants: with the present ones the cases of the GPU tests reach all of them, at both head
    sizes, with one span and with several, and so do the tests of the exponents.  (Tiles of 256 pairs are reached by the first four of LARGE and by none
    of MANY.)"""
    from tests.test_gpu_paged import FEW, LARGE, MANY
    from tests.test_gpu_paged_exponents import TILES
    calls = []
    for Hq, Hkv, d, c, m, C, _, first, count in FEW:
        calls += [(len(first), Hq, Hkv, d, 4096, c, m, C, sum(count), max(count), n, -1) for n in (1, 3, 0)]
    for Hq, Hkv, d, c, m, C, _, first, count in MANY:
        calls += [(len(first), Hq, Hkv, d, 4096, c, m, C, sum(count), sum(count), n, -1) for n in (1, 3, 0)]
    for Hq, Hkv, d, c, m, C, _, n_text, first, count in LARGE:
        calls += [(len(first), Hq, Hkv, d, n_text, c, m, C, sum(count), max(count), n, -1) for n in (1, 2, 0)]
    kinds = [(c[3], "few" if x["few"] else (x["pairs"], x["groups"]), x["n_splits"] > 1) for c, x in zip(calls, plans(calls))]
    every = {(d, kind, several) for d in (64, 128) for kind in ("few", (128, 1), (128, 2), (256, 1)) for several in (False, True)}
    assert set(kinds) == every, every - set(kinds)
    of_256 = {c[:3] for c, (_, kind, _) in zip(calls, kinds) if kind == (256, 1)}
    assert of_256 == {(len(x[8]), *x[:2]) for x in LARGE[:4]}
    calls = [(1, Hq, Hkv, d, n, 16, 2, 2, rows, rows, n_splits, -1) for Hq, Hkv, d, n, rows, n_splits in TILES]
    assert {(c[3], "few" if x["few"] else (x["pairs"], x["groups"])) for c, x in zip(calls, plans(calls))} == {x[:2] for x in every}
