"""The kernels that the serving calls choose among, each at sizes that reach it, against the plain fp64 forms of oracle/serving.py
(bounds: test_gpu_serving.py)."""
import numpy as np
import pytest
import torch

import paper_2603_00198_amd as strd
import test_gpu_serving as base
from oracle import serving as plain
from paper_2603_00198_amd.synth import np64

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

# Packed attention: what reaches each kernel (rows of the sequences, heads, prefix).  "tiles" is the one for any shape.
PREFILL = {
    "64 four waves": (BF16, 64, [(130, 20, 0), (60, 9, 0)], 4, 2, None),
    "64 two groups": (BF16, 64, [(400, 30, 0), (60, 9, 0)], 4, 2, None),
    "64 four waves, many": (BF16, 64, [(400, 30, 0), (60, 9, 0)], 180, 4, None),
    "128 four waves": (BF16, 128, [(130, 20, 0), (60, 9, 0)], 4, 2, None),
    "128 two groups": (BF16, 128, [(400, 30, 0), (60, 9, 0)], 4, 2, None),
    "128 four waves, many": (BF16, 128, [(400, 30, 0), (60, 9, 0)], 120, 2, False),
    "128 eight waves": (BF16, 128, [(1050, 50, 0), (20, 3, 0)], 80, 8, False),
    "128 eight waves, prefix": (BF16, 128, [(580, 30, 0), (20, 3, 0)], 64, 8, True),
    "tiles fp32": (F32, 64, [(130, 20, 0), (60, 9, 0)], 4, 2, None),
    "tiles": (BF16, 96, [(130, 20, 0), (60, 9, 0)], 4, 2, None),
}


def _prefill_kernels():
    return [pytest.param(name, p, id="%s-%s" % (name, "prefix" if p else "causal"))
            for name, k in PREFILL.items() for p in (False, True) if k[5] in (None, p)]


def _sees(seqs, prefix):
    rows = sum(s[0] + s[1] for s in seqs)
    sees, r = np.zeros((rows, rows), bool), 0
    for n, m, _ in seqs:
        i = np.arange(n + m)
        sees[r:r + n + m, r:r + n + m] = (i[None] <= i[:, None]) | (prefix & (i[None] < n) & (i[:, None] < n))
        r += n + m
    return sees


# ------------------------------------------------------------------ scores far from zero ---
@pytest.mark.parametrize("kernel,prefix", _prefill_kernels())
@pytest.mark.parametrize("cap", [0.0, 1e9])
@pytest.mark.parametrize("size", [3008.0, -3008.0, -1e6])
def test_prefill_varlen_scores_far_from_zero(kernel, prefix, cap, size):
    """Equal queries and equal keys: every score is the same number, some 1e8 to 1e13 from zero.  Without a bias, or with one of 0, every row that is
    seen counts the same; with a steep one a row's own is all that is left."""
    dtype, d, seqs, Hq, Hkv, _ = PREFILL[kernel]
    base._say("far scores", kernel, prefix, cap, size)
    rows, rep = sum(s[0] + s[1] for s in seqs), Hq // Hkv
    v = base._rand(torch.Generator().manual_seed(1), rows, Hkv, d, dtype=dtype)
    q, k = torch.full((rows, Hq, d), abs(size), dtype=dtype), torch.full((rows, Hkv, d), size, dtype=dtype)
    sees = _sees(seqs, prefix)
    p = sees / sees.sum(1, keepdims=True)
    want = np.einsum("tj,jhd->thd", p, np64(v)).repeat(rep, 1)
    mag = np.einsum("tj,jhd->thd", p, np.abs(np64(v))).repeat(rep, 1)
    bound = base._out_bound(want, 0.0, mag, dtype, rows)
    for sl in (None, 0.0, 1e30):
        o = strd.attn_prefill_varlen(base._dev(q), base._dev(k), base._dev(v), seqs, prefix=prefix, cap=cap,
                                     slopes=None if sl is None else torch.full((Hq,), sl, device="cuda"))
        if sl:
            assert torch.equal(o.cpu(), v.repeat_interleave(rep, 1)), sl
        else:
            base._within(o, want, bound, "o, slopes %r" % sl)


@pytest.mark.parametrize("kernel,prefix", _prefill_kernels())
@pytest.mark.parametrize("cap", [0.0, 1e9])
@pytest.mark.parametrize("slopes", [False, True])
def test_prefill_varlen_rows_beside_one_with_scores_far_from_zero(kernel, prefix, cap, slopes):
    """Its neighbours keep their bits."""
    dtype, d, seqs, Hq, Hkv, _ = PREFILL[kernel]
    base._say("beside far scores", kernel, prefix, cap, slopes)
    q, k, v, sl, _ = base._prefill(seqs, Hq, Hkv, d, dtype, cap, slopes, False, prefix, seed=5)
    first = strd.attn_prefill_varlen(base._dev(q), base._dev(k), base._dev(v), seqs, prefix=prefix, cap=cap, slopes=base._dev(sl))
    for at in (0, 37, 131):
        q[at] *= 1e9
    o = strd.attn_prefill_varlen(base._dev(q), base._dev(k), base._dev(v), seqs, prefix=prefix, cap=cap, slopes=base._dev(sl))
    others = torch.ones(q.shape[0], dtype=torch.bool)
    others[[0, 37, 131]] = False
    assert torch.equal(o[others], first[others])
    assert torch.isfinite(o.float()).all()
