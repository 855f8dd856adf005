"""The first launch of the packed scans', trees' and long convolutions' kernels in a process against the second, bit for bit (why: test_gpu_cold_start.py).
Needs a GPU."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = r"""
import sys, torch
sys.path.insert(0, sys.argv[1])
import paper_2603_00198_amd as strd
case = sys.argv[2]
DEV = "cuda"
g = torch.Generator().manual_seed(7)
def rnd(*shape, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(*shape, generator=g) * scale).to(dtype).to(DEV)
# launches of other kernels first: what the caches and the LDS hold when the case starts is not its own
strd.rmsnorm(rnd(3000, 1024), rnd(1024))
strd.select_topk(torch.rand(20000, generator=g).to(DEV), 5000)
torch.cuda.synchronize()

def scan(seqs, H, P, G, n, dtype=torch.bfloat16):
    T = sum(s[0] + s[1] for s in seqs)
    x, B, C = rnd(T, H, P, dtype=dtype), rnd(T, G, n, dtype=dtype), rnd(T, G, n, dtype=dtype)
    dt = torch.nn.functional.softplus(torch.randn(T, H, generator=g)).to(DEV)
    A = -torch.exp(2 * torch.rand(H, generator=g))
    A[::4] *= 0.003
    A, D, state, out = A.to(DEV), rnd(H, dtype=torch.float32), rnd(len(seqs), H, P, n, dtype=torch.float32), torch.zeros(len(seqs), H, P, n, device=DEV)
    def call():
        out.zero_()
        return strd.ssd_prefill_varlen(x, dt, A, B, C, seqs, D, state, out), out
    return call

def tree(T, m, Hq, Hkv, d, dtype=torch.bfloat16):
    q, k, v, kn, vn = rnd(m, Hq, d, dtype=dtype), rnd(T, Hkv, d, dtype=dtype), rnd(T, Hkv, d, dtype=dtype), rnd(m, Hkv, d, dtype=dtype), rnd(m, Hkv, d, dtype=dtype)
    mask, slopes = strd.tree_mask(range(-1, m - 1)), torch.rand(Hq, generator=g).to(DEV)
    return lambda: (strd.attn_tree_step(q, k, v, kn, vn, mask), strd.attn_tree_step(q, k, v, kn, vn, mask, cap=20.0, slopes=slopes))

call = {
    "scan_segments": lambda: scan([(901, 48, 0), (377, 21, 0), (1207, 33, 0)], 128, 64, 8, 128),
    "scan_segments_64": lambda: scan([(901, 48, 0), (377, 21, 0), (1207, 33, 0)], 64, 64, 4, 64),
    "scan_segments_in_parts": lambda: scan([(12000, 0, 0), (5000, 0, 0)], 128, 64, 8, 64),
    "scan_chunks": lambda: scan([(600, 48, 0), (377, 21, 0)], 16, 64, 2, 128),
    "scan_chunks_fp32": lambda: scan([(3000, 48, 0), (377, 21, 0)], 8, 64, 8, 64, torch.float32),
    "tree_eight_waves": lambda: tree(20003, 33, 32, 8, 128),
    "tree_four_waves": lambda: tree(20003, 20, 32, 8, 128),
    "tree_two_waves_short": lambda: tree(843, 16, 32, 8, 128),
    "tree_96": lambda: tree(9999, 40, 16, 4, 96),
    "tree_general": lambda: tree(3001, 20, 8, 2, 64, torch.float32),
}[case]()
first = [t.clone() for t in call()]
torch.cuda.synchronize()
for rep in range(2):
    again = call()
    torch.cuda.synchronize()
    for i, (u, v_) in enumerate(zip(first, again)):
        bad = int((u != v_).sum())
        if bad:
            raise SystemExit("%s: output %d of the first launch differs from launch %d in %d of %d elements"
                             % (case, i, rep + 2, bad, u.numel()))
print("ok", case, flush=True)
"""

CASES = ["scan_segments", "scan_segments_64", "scan_segments_in_parts", "scan_chunks", "scan_chunks_fp32", "tree_eight_waves", "tree_four_waves",
         "tree_two_waves_short", "tree_96", "tree_general"]


@pytest.mark.parametrize("case", CASES)
def test_first_launch_in_a_process_equals_the_second(case):
    print("[case] cold start: " + case, flush=True)
    r = subprocess.run([sys.executable, "-c", SCRIPT, ROOT, case], capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and ("ok " + case) in r.stdout, (r.stdout[-2000:], r.stderr[-2000:])
