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


@pytest.mark.parametrize("case", [
    # the scan's directions at once (13 heads of 128, 55 of 64) or, with more states or blocks, one after the other, a thread with four elements
    (1, 800, 200, 13, 128, BF, True), (1, 800, 200, 14, 128, BF, True), (1, 300, 100, 40, 128, FP, True), (2, 500, 131, 8, 128, BF, False),
    (1, 640, 16, 56, 64, BF, True), (1, 300, 70, 55, 64, FP, True), (1, 400, 150, 57, 64, FP, False), (3, 900, 7, 5, 128, BF, True), (1, 1541, 1, 6, 128, FP, True),
])
def test_scan_directions(case):
    recurrence.check(case)
    B, T, block, H, D, _, _ = case
    if B * H * D * D <= 148 * 3 // 2 * 1024 and B * H * -(-T // block) <= 592:
        return
    from paper_2605_16579_b200 import arl2

    recurrence.check(case, flags=arl2.ARL2_FLAG_FORCE_SIMT)
