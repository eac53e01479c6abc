"""The INT8 product's choice of kernel (csrc/i8_plan.h), compiled for the host: over drawn sizes its shares
of k cover k with none empty and its workspace stays within the documented bound, and the sizes at
which the GPU tests hold the product to its definition take every path that the choice takes."""
import os
import shutil
import subprocess
from collections import Counter

import numpy as np
import pytest

import test_gpu_gemm_i8_scaled as G

HERE = os.path.dirname(os.path.abspath(__file__))
CUS = 256
KERNELS = ["16 rows streamed", "32 rows streamed", "64 rows streamed", "128 x 64", "128 x 128", "128 x 256", "256 x 128", "256 x 64",
           "192 x 128", "192 x 192", "256 x 256"]


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("plan") / "i8_plan_driver")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-I", os.path.join(os.path.dirname(HERE), "paper_2609_34185_amd", "csrc"),
                           os.path.join(HERE, "i8_plan_driver.cpp"), "-o", exe])

    def of(sizes, cus=CUS):
        out = subprocess.run([exe, str(cus)], input="\n".join("%d %d %d" % tuple(s) for s in sizes), text=True, capture_output=True, check=True)
        rows = [tuple(map(int, line.split())) for line in out.stdout.splitlines()]
        assert len(rows) == len(sizes)
        return rows
    return of


def drawn(count, seed):
    """Sizes spread over their logarithms: 1 to 9000 rows, 1 to 18000 columns, k from 16 to 17600."""
    s = np.exp(np.random.default_rng(seed).uniform(0, np.log((9000, 18000, 1100.49)), (count, 3))).round().astype(int).clip(1)
    return (s * (1, 1, 16)).tolist()


def path(plan):
    """What code a size reaches: the kernel, whether sums are joined, pieces, and whether one CU takes several workgroups."""
    kernel, parts, _, cut, over, _ = plan
    return KERNELS[kernel], "k shared out" if parts > 1 else "whole k", cut, "several rounds" if over else "one round"


def test_tested_sizes_take_every_path(plans):
    taken = Counter(map(path, plans(drawn(400000, 1))))
    tested = set(map(path, plans(G.SHAPES + G.PATHS + G.SHARED)))
    assert not {p: c for p, c in taken.items() if p not in tested}


def test_sizes_named_for_shares_of_k_share_it(plans):
    for plan in plans(G.SHARED):
        assert plan[1] > 1 and plan[5] > 0


@pytest.mark.parametrize("cus", [256, 304, 32, 1])
def test_shares_of_k_and_workspaces(plans, cus):
    sizes = drawn(20000, 2) + [[m, n, k] for m in (1, 17, 600, 1 << 24) for n in (1, 5120, 1 << 24) for k in (16, 131056)]
    for (m, n, k), (kernel, parts, steps, cut, _, room) in zip(sizes, plans(sizes, cus)):
        kb = -(-k // 128)
        assert (parts - 1) * steps < kb <= parts * steps
        assert room == (4 * parts * m * (n + 3 & ~3) if parts > 1 else 0) and room <= cus << 20
        assert parts == 1 or cut == 1
