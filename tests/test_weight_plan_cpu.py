"""Host only: how many parts the sums of weight gradients from the cache are shared out in, by the workspace that they ask for."""
import random

import pytest
import torch

from paper_2305_18513_amd import binding as sf


@pytest.fixture(scope="module", autouse=True)
def built():
    if not sf.is_built():
        from paper_2305_18513_amd import build
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
