"""Calls behind a prompt whose tensors have more than 2^31 elements: their last rows and slots, against the same call on those alone."""
import numpy as np
import pytest
import torch

import paper_2603_00198_amd as strd
import test_gpu_onward as base
import test_gpu_onward_edges as edges
from paper_2603_00198_amd.synth import np64

pytestmark = pytest.mark.gpu
DEV, BF16, F32, PAST = "cuda", torch.bfloat16, torch.float32, 1 << 31


@pytest.fixture(autouse=True)
def _memory_goes_back():
    yield
    torch.cuda.empty_cache()


def _gen(seed=1):
    return torch.Generator(device=DEV).manual_seed(seed)


def test_slots_of_large_pools():
    """States and windows of the last slots: single tokens, and packed sequences in both scans, in place."""
    base._say("large pools")
    H, P, G, n, far = 128, 64, 8, 128, [2099, 2050, 3]
    pool = torch.zeros((2100, H, P, n), device=DEV)
    assert pool.numel() > PAST
    few = torch.randn((3, H, P, n), generator=_gen(), device=DEV)
    pool[far] = few
    seqs = [(150, 3, 0), (600, 0, 0), (0, 0, 0)]
    for dtype in (BF16, F32):
        x, dt, A, B, C, D = (base._dev(t) for t in base._scan_case(753, H, P, G, n, dtype))
        at = torch.tensor(far, dtype=torch.int32, device=DEV)
        y = strd.ssd_decode_steps(x[:3], dt[:3], A, B[:3], C[:3], D, pool, slots=at)
        assert torch.equal(y, strd.ssd_decode_steps(x[:3], dt[:3], A, B[:3], C[:3], D, few)) and torch.equal(pool[far], few)
        y = strd.ssd_prefill_varlen(x, dt, A, B, C, seqs, D, state=pool, slots=far)
        assert torch.equal(y, strd.ssd_prefill_varlen(x, dt, A, B, C, seqs, D, state=few)) and torch.equal(pool[far], few)
    rest = torch.ones(2100, dtype=torch.bool, device=DEV)
    rest[far] = False
    assert not any(bool(part.any()) for part in pool[rest].split(100))
    del pool
    Cx, Cb, W, far = 8192, 1024, 4, [70099, 69950, 3]
    pool = torch.zeros((70100, W - 1, Cx + 2 * Cb), dtype=BF16, device=DEV)
    assert pool.numel() > PAST
    few = torch.randn((3, W - 1, Cx + 2 * Cb), generator=_gen(), device=DEV).to(BF16)
    pool[far] = few
    u, w = (torch.randn(s, generator=_gen(2), device=DEV).to(BF16) for s in ((20, Cx + 2 * Cb), (Cx + 2 * Cb, W)))
    a = strd.conv1d_silu_step(u[:3], w, None, Cx, Cb, pool, slots=torch.tensor(far, dtype=torch.int32, device=DEV))
    b = strd.conv1d_silu_step(u[:3], w, None, Cx, Cb, few)
    assert all(torch.equal(s, t) for s, t in zip(a[:3], b[:3])) and torch.equal(pool[far], few)
    a = strd.conv1d_silu_varlen(u, w, None, Cx, Cb, [(2, 0, 0), (17, 1, 0), (0, 0, 0)], window=pool, slots=far)
    b = strd.conv1d_silu_varlen(u, w, None, Cx, Cb, [(2, 0, 0), (17, 1, 0), (0, 0, 0)], window=few)
    assert all(torch.equal(s, t) for s, t in zip(a, b)) and torch.equal(pool[far], few)


@pytest.mark.parametrize("dtype,Cx,Cb,rows", [(BF16, 8192, 1024, 210000), (BF16, 8193, 1024, 210000)])
def test_convolution_of_many_rows(dtype, Cx, Cb, rows):
    base._say("many rows, convolution", Cx)
    u = torch.zeros((rows, Cx + 2 * Cb), dtype=dtype, device=DEV)
    assert (rows - 100) * Cx > 0.79 * PAST and (rows - 100) * (Cx + 2 * Cb) > PAST
    u[-100:] = torch.randn((100, Cx + 2 * Cb), generator=_gen(), device=DEV).to(dtype)
    w, b = (torch.randn(s, generator=_gen(2), device=DEV).to(dtype) for s in ((Cx + 2 * Cb, 4), (Cx + 2 * Cb,)))
    got = strd.conv1d_silu_varlen(u, w, b, Cx, Cb, [(rows - 90, 0, 0), (90, 0, 0)])
    alone = strd.conv1d_silu_varlen(u[-110:], w, b, Cx, Cb, [(20, 0, 0), (90, 0, 0)])
    assert all(torch.equal(s[-107:], t[-107:]) for s, t in zip(got, alone))


@pytest.mark.parametrize("H,P,G,n", [(128, 64, 8, 64), (128, 64, 8, 16)])
def test_scan_of_many_rows(H, P, G, n):
    """The last of three sequences, on the matrix cores and in chunks."""
    base._say("many rows, scan", n)
    lens = [150000, 114000, 700]
    rows = sum(lens)
    x = torch.randn((rows, H, P), generator=_gen(), device=DEV, dtype=BF16)
    assert (rows - lens[2]) * H * P > PAST
    B, C = (torch.randn((rows, G, n), generator=_gen(k), device=DEV, dtype=BF16) for k in (2, 3))
    dt = torch.rand((rows, H), generator=_gen(4), device=DEV)
    A, D = -0.02 - torch.rand(H, generator=_gen(5), device=DEV), torch.randn(H, generator=_gen(6), device=DEV)
    state, seqs = torch.zeros((3, H, P, n), device=DEV), [(t, 0, 0) for t in lens]
    y = strd.ssd_prefill_varlen(x, dt, A, B, C, seqs, D, state_out=state)
    for s, r0, r1 in ((1, 150000, 150300), (2, 264000, 264700)):   # a sequence's beginning, a whole one
        at, t = slice(r0, r1), r1 - r0
        edges._check_fine([(t, 0, 0)], x[at], dt[at], A, B[at], C[at], D, None, [s], None, y[at], state if s == 2 else None, 2, [0, 5, H - 1], [0, 17, P - 1])


@pytest.mark.parametrize("dtype,d,interleaved", [(BF16, 128, False), (BF16, 120, True)])
def test_rotary_positions_of_many_rows(dtype, d, interleaved):
    base._say("many rows, rotary positions", d)
    rows = PAST // (40 * d) + 2000
    qkv = torch.zeros((rows, 40, d), dtype=dtype, device=DEV)
    tail = torch.randn((1500, 40, d), generator=_gen(), device=DEV).to(dtype)
    qkv[-1500:] = tail
    q, k = qkv[:, :32], qkv[:, 32:]
    pos, freq = torch.arange(rows, dtype=torch.int32, device=DEV), strd.rope_frequencies(d)
    strd.rope(q, k, pos, freq, interleaved, 1.0, q, k)
    a, b = strd.rope(tail[:, :32], tail[:, 32:], pos[-1500:], freq, interleaved)
    assert torch.equal(q[-1500:], a) and torch.equal(k[-1500:], b) and not qkv[:-1500].any()


@pytest.mark.parametrize("dtype,m,Hq,Hkv,d", [(BF16, 40, 32, 8, 128), (BF16, 5, 8, 8, 96), (F32, 9, 8, 4, 128)])
def test_tree_over_a_cache_of_many_rows(dtype, m, Hq, Hkv, d):
    """Keys of zeros and values of zeros but for the last hundred rows: the others are a number of weights of 1."""
    base._say("many rows, tree", dtype, d)
    T = PAST // (Hkv * d) + 5000
    q, k, v, mask = base._tree_case(100, m, Hq, Hkv, d, dtype, seed=2, size=4.0)
    k *= 2
    kc, vc = torch.zeros((T, Hkv, d), dtype=dtype, device=DEV), torch.zeros((T, Hkv, d), dtype=dtype, device=DEV)
    kc[-100:], vc[-100:] = base._dev(k[:100]), base._dev(v[:100])
    o = strd.attn_tree_step(base._dev(q), kc, vc, base._dev(k[100:]), base._dev(v[100:]), base._dev(mask))
    rep, sees = Hq // Hkv, np.concatenate([np.ones((m, 100), bool), np.array([[int(x) >> j & 1 for j in range(m)] for x in mask], bool)], 1)
    Q, K, V = np64(q), np64(k), np64(v)
    for h in range(Hq):
        x = d ** -0.5 * Q[:, h] @ K[:, h // rep].T
        # rounded products and sums of a score, and its exponent's argument
        delta = d ** -0.5 * (d + 2) * base.U32 * np.abs(Q[:, h]) @ np.abs(K[:, h // rep]).T + 8 * base.U32 * np.abs(x)
        top = np.maximum(np.where(sees, x, 0).max(1, keepdims=True), 0)
        e = np.where(sees, np.exp(x - top), 0)
        p = e / (e.sum(1, keepdims=True) + (T - 100) * np.exp(-top))
        want, mag = p @ V[:, h // rep], p @ np.abs(V[:, h // rep])
        # the T weights of 1 add up in splits of a few thousand; a lane's and a row's sums of 32 at a time: 2^17 roundings of them at most
        off = (p * delta) @ np.abs(V[:, h // rep]) + (p * delta).sum(1, keepdims=True) * mag + 2.0 ** 17 * base.U32 * mag
        base._within(o[:, h], want, base._tree_bound(want, off, mag, dtype, 0), "o of head %d" % h)
