"""How a decode call over a 4-bit cache is planned (``csrc/apb_plan.h``, plain
C++): every key is in one split, every row in one workgroup, the launch fits, and the
forms that the GPU tests' shapes are written for are the ones they run."""
import os
import random
import subprocess

import pytest

import test_gpu_decode4 as gpu

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2502_12085_amd", "csrc")
MAIN = r"""
#include <stdio.h>
#include "apb_plan.h"
int main() {
  long long a[5];
  while (scanf("%lld %lld %lld %lld %lld", a, a + 1, a + 2, a + 3, a + 4) == 5) {
    const apb::Decode4Plan p = apb::plan_decode4(a[0], a[1], (int)a[2], a[3], a[4]);
    printf("%d %d %d %d %d %llu\n", p.n_split, p.blocks_per_split, p.rows, p.waves, p.row_blocks,
           (unsigned long long)p.workspace_bytes);
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan4")
    (d / "plan.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, "-o", str(d / "plan"),
                    str(d / "plan.cpp")], check=True)

    def ask(problems):
        text = "\n".join(" ".join(str(int(x)) for x in p) for p in problems)
        out = subprocess.run([str(d / "plan")], input=text, capture_output=True, text=True,
                             check=True).stdout.split("\n")
        return [tuple(int(x) for x in line.split()) for line in out if line]

    return ask


def _check(problem, plan):
    n_q, n_kv, d, keys, n_new = problem
    n_split, bps, rows, waves, row_blocks, ws = plan
    r, nblk = n_q // n_kv * n_new, -(-keys // 32)
    assert rows == (16 if r <= 16 else 32) and waves in (4, 8)
    assert (row_blocks - 1) * rows < r <= row_blocks * rows
    assert n_split >= 1 and bps >= 1
    assert n_split * bps >= nblk and (n_split - 1) * bps < max(nblk, 1)   # no empty split
    assert n_split == 1 or n_split * row_blocks * n_kv <= 6 * 256         # rounds of the GPU's CUs
    assert n_split * row_blocks * n_kv * 64 * waves < 1 << 32             # threads of a launch
    assert 32 * n_split * bps < (1 << 31) - (1 << 20)                     # key numbers in int32
    assert ws == (n_split * n_q * n_new * (d + 2) * 4 if n_split > 1 else 16)


def test_every_key_and_row_once(plans):
    rng = random.Random(5)
    problems = [(1, 1, 64, 0, 1), (8, 2, 64, 0, 3), (1, 1, 128, 1 << 30, 1),
                (65536, 65536, 128, 1 << 30, 1), (65536, 65536, 64, 33, 255),
                ((1 << 24) - 1, 1, 64, 5, 1), (1, 1, 64, 1 << 30, (1 << 24) - 1), (512, 512, 128, 4097, 2),
                (4096, 64, 64, 100000, 100)]
    for _ in range(3000):
        n_kv = rng.choice((1, 2, 3, 8, 40, 300))
        n_new = int(2 ** rng.uniform(0, 10))
        keys = int(2 ** rng.uniform(0, 21))
        problems.append((n_kv * rng.randint(1, 9), n_kv, rng.choice((64, 128)), keys, n_new))
    got = plans(problems)
    assert len(got) == len(problems)
    for problem, plan in zip(problems, got):
        _check(problem, plan)


def test_the_gpu_tests_run_every_form(plans):
    shapes = [m.args[1] for f in (gpu.test_matches_oracle, gpu.test_long_caches, gpu.test_forms)
              for m in f.pytestmark if m.name == "parametrize"]
    problems = [(n_q, n_kv, d, keys, n_new) for s in shapes
                for n_q, n_kv, d, _, keys, n_new, _ in s]
    forms = {(p[2], g[2], g[3], g[0] > 1) for p, g in zip(problems, plans(problems))}
    want = {(d, rows, waves, split) for d in (64, 128) for split in (False, True)
            for rows in (16, 32) for waves in (4, 8)}
    assert forms >= want, sorted(want - forms)
    # and the merge with one, two and all thread groups a row, with a part of a workgroup
    merges = set()
    for p, g in zip(problems, plans(problems)):
        rows = p[0] * p[4]
        if g[0] > 1:
            groups = 0 if rows < 256 or g[0] > 16 else 1 if g[0] <= 8 else 2
            merges.add((p[2], groups, bool(groups) and rows % (1024 // p[2] // groups) != 0))
    assert merges >= {(d, n, odd) for d in (64, 128) for n in (1, 2) for odd in (True,)}, merges
    assert merges >= {(64, 0, False), (128, 0, False)}
