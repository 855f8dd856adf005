"""Calls behind a prompt that the general tests do not make, against the plain fp64 forms of oracle/onward.py (bounds there and in
test_gpu_onward.py; half a step of bf16 is 2^-8, of fp32 2^-24, relative)."""
import numpy as np
import pytest
import torch

import paper_2603_00198_amd as strd
import test_gpu_onward as base
from oracle import onward as plain
from paper_2603_00198_amd.synth import np64

pytestmark = pytest.mark.gpu
DEV, BF16, F32 = "cuda", torch.bfloat16, torch.float32
U32, HALF = base.U32, base.HALF


# ------------------------------------------------------------------ drafted trees: scores far from zero
# One, two, four and eight computing waves of the matrix cores' kernel, then the general one.
TREES = [(BF16, 64, 2, 1, 11), (BF16, 128, 8, 2, 16), (BF16, 96, 4, 1, 32), (BF16, 64, 8, 1, 40), (BF16, 128, 12, 2, 33), (F32, 64, 4, 2, 11), (BF16, 40, 4, 2, 33)]


@pytest.mark.parametrize("dtype,d,Hq,Hkv,m", TREES)
@pytest.mark.parametrize("cap,slope", [(0.0, None), (0.0, 0.5), (1e9, None), (1e9, 0.5)])
@pytest.mark.parametrize("size", [1000.0, -1000.0, -1e6])
def test_tree_nodes_that_see_nothing_beside_scores_far_from_zero(size, cap, slope, dtype, d, Hq, Hkv, m):
    """Without a cache every other node sees nothing and gets zeros, whatever scores the rows beside it have: equal ones, 8e6 to 8e12 from zero, which
    weigh the same."""
    base._say("tree nothing seen", size, cap, slope, dtype, d, Hq, Hkv, m)
    q, k = torch.full((m, Hq, d), abs(size), dtype=dtype, device=DEV), torch.full((m, Hkv, d), size, dtype=dtype, device=DEV)
    v = base._rand(torch.Generator().manual_seed(m), m, Hkv, d, dtype=dtype)
    mask = torch.tensor([0 if i % 2 == 0 else 1 << i | 1 << (i - 1) for i in range(m)], dtype=torch.int64, device=DEV)
    sl = None if slope is None else torch.full((Hq,), slope, device=DEV)
    ps = None if slope is None else torch.full((m,), 7, dtype=torch.int32, device=DEV)
    none = torch.empty((0, Hkv, d), dtype=dtype, device=DEV)
    o = strd.attn_tree_step(q, none, none, k, base._dev(v), mask, cap=cap, slopes=sl, pos=ps)
    assert (o[::2] == 0).all()
    vv = np64(v)
    want = np.repeat((vv[0:m - 1:2] + vv[1:m:2]) / 2, Hq // Hkv, axis=1)
    mag = np.repeat((np.abs(vv[0:m - 1:2]) + np.abs(vv[1:m:2])) / 2, Hq // Hkv, axis=1)
    # weights of 1 each: a sum of two, and a division
    base._within(o[1::2], want, 4 * U32 * mag + HALF[dtype] * np.abs(want), "o")
