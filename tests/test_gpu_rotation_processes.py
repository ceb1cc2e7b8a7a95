"""The rotation's gradients of weights do not depend on what a process called before."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CHILD = """
import hashlib, sys
sys.path[:0] = [sys.argv[1], sys.argv[1] + "/tests"]
import torch
import test_gpu_rotation as rotation
for D in map(int, sys.argv[2:]):
    H, T = 1664 // D, 5000
    case = (1, T, H, H, D, torch.float32, "token", (12, 10, 10), (9, 11))
    _, r, _, _ = rotation.op(case)
    q, k, (qw, kw), start, randn = rotation.inputs(case, 1)
    grads = r.backward(randn(*q.shape), randn(*k.shape), q, k, start=start, q_weight=qw, k_weight=kw)
    print(D, *(hashlib.sha256(g.cpu().numpy().tobytes()).hexdigest() for g in grads))
"""


def test_head_sizes_in_either_order():
    """fp32, rows of 1664 channels: of 26 heads of 64 an SM holds more CTAs than of 13 heads of 128, whose tables are larger."""
    lines = [sorted(subprocess.run([sys.executable, "-c", CHILD, ROOT, *order], check=True, capture_output=True, text=True, timeout=300).stdout.splitlines())
             for order in (("64", "128"), ("128", "64"))]
    assert len(lines[0]) == 2 and lines[0] == lines[1]
