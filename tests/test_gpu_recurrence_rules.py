"""The recurrence on both sides of the rules that choose its kernels; definition and bounds as in test_gpu_recurrence."""
import pytest
import torch

import test_gpu_recurrence as recurrence

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


@pytest.mark.parametrize("case", [
    # B, T, block, H, D, dtype, state given: fp32 heads of 64 with 48, 50, 74 and 76 tiles
    (1, 1536, 64, 2, 64, FP, True), (2, 1500, 120, 2, 64, FP, True), (1, 2360, 64, 2, 64, FP, False), (1, 2432, 64, 2, 64, FP, True),
])
def test_few_tiles(case):
    recurrence.check(case)
