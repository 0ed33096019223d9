"""Host only: the tiles that weight gradients from the cache take, and the parts that their sums are shared out in."""
import os
import random
import subprocess

import pytest
import torch

from paper_2305_18513_amd import binding as sf
from paper_2305_18513_amd import build
from tests.test_gpu_weight_grad import WIDE


@pytest.fixture(scope="module", autouse=True)
def built():
    if not sf.is_built():
        build.build_library(verbose=False)
    sf.lib()


def test_the_parts_memory_is_bounded():
    """By what the input as numbers would take, or 256 MiB, whatever the sizes."""
    rng = random.Random(1)
    cases = [(torch.bfloat16, 64, *sizes) for sizes in ((16384, 5120, 5120), (65536, 11008, 4096), (36390, 6579, 1920))]
    for _ in range(3000):
        M, N, K = (int(2 ** rng.uniform(0, top)) for top in (18, 16, 11))
        block = rng.choice([32, 64, 128, 256])
        cases.append((rng.choice([torch.float32, torch.bfloat16]), block, M, N, K * block))
    for dtype, block, M, N, K in cases:
        need = sf.weight_grad_dequant_workspace(dtype, block, M, N, K)
        assert need <= max(M * K * (2 if dtype == torch.bfloat16 else 4), 1 << 28), (dtype, block, M, N, K)
        assert need % (N * K * 4) == 0


def test_sizes_of_the_wide_tiles(tmp_path):
    """The sizes that test_gpu_weight_grad.py means to run on tiles 256 wide take them, and rows that begin anywhere never do."""
    source, program = tmp_path / "plan.cpp", tmp_path / "plan"
    source.write_text("""
#include <cstdio>
#include "weight_plan.hpp"
int main()
{
    for (long M, N, K; scanf("%ld %ld %ld", &M, &N, &K) == 3;) printf("%d\\n", slimfit::WeightPlan(SLIMFIT_BF16, 32, M, N, K).tile_n);
}
""")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-I", build.INCLUDE, "-I", build.CSRC, str(source), "-o", str(program)], check=True)
    rng = random.Random(2)
    sizes = WIDE + [(int(2 ** rng.uniform(0, 17)), 8 * int(2 ** rng.uniform(0, 13)) + rng.randint(1, 7), 32 * int(2 ** rng.uniform(0, 9))) for _ in range(5000)]
    out = subprocess.run([str(program)], input="\n".join("%d %d %d" % s for s in sizes), capture_output=True, text=True, check=True).stdout.split()
    assert out == ["256"] * len(WIDE) + ["128"] * 5000
