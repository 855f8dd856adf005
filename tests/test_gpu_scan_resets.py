"""The scan of one sequence (strd_ssd_prefill) where tokens reset a head: what comes behind one in the same few tokens keeps its weights, which are not
differences of numbers as large as the reset's exponent.  Bounds: test_gpu_onward.py, whose count of roundings to bf16 (of a weight or the state, of a weighted
input, and two of an output whose parts are completed later) holds here too."""
import numpy as np
import pytest
import torch

import paper_2603_00198_amd as strd
import test_gpu_onward as base
from oracle import onward as plain
from paper_2603_00198_amd.synth import np64

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

# One workgroup walking the sequence, segments with four, two and one head of a group, and the general kernels
SHAPES = [(700, 128, 64, 8, 128, BF16), (8320, 128, 64, 8, 128, BF16), (4200, 16, 64, 8, 64, BF16), (4200, 12, 64, 4, 64, BF16), (2500, 32, 64, 4, 64, BF16),
          (700, 8, 64, 2, 64, F32), (4200, 8, 64, 2, 64, F32), (700, 6, 40, 2, 24, BF16)]


@pytest.mark.parametrize("T,H,P,G,n,dtype", SHAPES)
@pytest.mark.parametrize("size", [300.0, 1e4, 1e6, 1e9])
def test_scan_goes_on_behind_tokens_that_reset_a_head(size, T, H, P, G, n, dtype):
    base._say("scan of one sequence, resets", size, T, H, P, G, n, dtype)
    x, dt, A, B, C, D = base._scan_case(T, H, P, G, n, dtype, seed=6)
    dt *= 0.02
    reset = torch.rand((T, H), generator=torch.Generator().manual_seed(1)) < 1 / 30
    dt[reset] = (-size / A).expand(T, H)[reset]
    x[reset] = 0
    y, _ = strd.ssd_prefill(*(base._dev(t) for t in (x, dt, A, B, C)), D=base._dev(D))
    some = sorted({0, 1, H // 2, H - 1})
    gs, chans = [h * G // H for h in some], list(range(0, P, 7))
    want, _, my, mS = plain.scan(*(np64(t) for t in (x[:, some][:, :, chans], dt[:, some], A[some], B[:, gs], C[:, gs], D[some])), np.zeros((len(some), len(chans), n)))
    # (a reset leaves a few dozen tokens to add up, whatever T)
    by, _ = base._scan_bounds(want, my, mS, min(T, 700), n, dtype)
    base._within(y[:, some][:, :, chans], want, by, "y")
