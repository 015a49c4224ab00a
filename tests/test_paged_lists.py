"""Keys that the paged attention lists for a group of rows of which none sees them (no GPU needed): what may lie there is anything."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_listed_keys_that_no_row_sees(tmp_path):
    exe = str(tmp_path / "paged_lists")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-Wall", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I",
                    os.path.join(ROOT, "paper_2604_24432_amd", "csrc"), os.path.join(ROOT, "tests", "plan", "paged_lists.cpp"), "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr[-2000:]
    assert int(res.stdout) == 6      # c 6, m 3, C 2: two chunks' summaries
