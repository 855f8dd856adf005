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


@pytest.mark.parametrize("dtype,d,Hq,Hkv,m", [(BF16, 64, 4, 1, 8), (BF16, 128, 8, 2, 16), (BF16, 96, 4, 1, 32), (BF16, 64, 8, 1, 40), (BF16, 128, 8, 1, 40), (F32, 64, 4, 2, 11)])
@pytest.mark.parametrize("cap", [0.0, 20.0, 1e9])
@pytest.mark.parametrize("T", [100, 3000])
def test_tree_equal_scores_far_from_zero(T, cap, dtype, d, Hq, Hkv, m):
    """Rows of the cache at one position that is 2^24 - 1 from the nodes', of one key: whatever the slope, from none to 64, and whatever block or split they are
    in, they weigh the same, a sum of T of them and a division away from their mean.  Every other node sees itself, at its own position: where there is a slope
    that is all it sees."""
    base._say("tree equal scores", T, cap, dtype, d, Hq, Hkv, m)
    g = torch.Generator().manual_seed(T + m)
    far = 2.0 if cap < 1e9 else 3e3   # (with the high cap scores of 1e6 and more)
    q = base._rand(g, m, Hq, d, dtype=dtype, size=far)
    k = base._rand(g, 1, Hkv, d, dtype=dtype, size=far).expand(T + m, Hkv, d).contiguous()
    v = base._rand(g, T + m, Hkv, d, dtype=dtype)
    sl = torch.tensor([0.0, 1.0, 8.0, 64.0], dtype=F32).repeat(Hq // 4)
    ps = torch.cat([torch.zeros(T), torch.full((m,), 2.0 ** 24 - 1)]).to(torch.int32)
    mask = torch.tensor([1 << i if i % 2 else 0 for i in range(m)], dtype=torch.int64)
    o = strd.attn_tree_step(*(base._dev(t) for t in (q, k[:T], v[:T], k[T:], v[T:], mask)), cap=cap, slopes=base._dev(sl), pos=base._dev(ps))
    vv, rep = np64(v), Hq // Hkv
    want, mag = np.zeros((m, Hq, d)), np.zeros((m, Hq, d))
    for i in range(m):
        for h in range(Hq):
            seen = vv[:T, h // rep]
            if i % 2:
                seen = vv[T + i:T + i + 1, h // rep] if sl[h] else np.concatenate([seen, vv[T + i:T + i + 1, h // rep]])
            want[i, h], mag[i, h] = seen.mean(0), np.abs(seen).mean(0)
    # (a weight is rounded to bf16 before the product; it is a power of two or 1 here, or all of a row's are the same number)
    base._within(o, want, (T + m) * U32 * mag + (2 * 2.0 ** -8 * mag if dtype == BF16 else 0) + HALF[dtype] * np.abs(want) + 1e-30, "o")


# ------------------------------------------------------------------ single tokens of a filter of one tap
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("listed", [False, True])
def test_conv_step_of_one_tap_needs_no_window(listed, dtype):
    """Nothing is carried, so there is no pool whose size a slot could be past; a batch may still be padded."""
    base._say("conv step one tap", listed, dtype)
    g = torch.Generator().manual_seed(3)
    batch, Cx, Cb, H = 5, 32, 8, 3
    row, w, b, bias = (base._rand(g, *s, dtype=t) for s, t in (((batch, 48 + H), dtype), ((48, 1), dtype), ((48,), dtype), ((H,), F32)))
    slots = torch.tensor([900, -1, 0, 900, 7], dtype=torch.int32) if listed else None
    args = [base._dev(t) for t in (row, w, b)]
    live = [0, 2, 4] if listed else list(range(batch))
    for pool in (None, torch.zeros(1000, 0, 48, dtype=dtype, device=DEV)):
        x, B, C, dt = strd.conv1d_silu_step(*args, Cx, Cb, pool, slots=base._dev(slots), H=H, dt_bias=base._dev(bias))
        got, want, mag = torch.cat([x, B, C], 1), np64(w)[:, 0] * np64(row)[:, :48] + np64(b), np.abs(np64(w)[:, 0] * np64(row)[:, :48]) + np.abs(np64(b))
        o = plain.silu(want)
        base._within(got[live], o[live], base._conv_bound(o, want, mag, 1, dtype)[live], "o")
        raw = np64(row)[:, 48:] + np64(bias)
        steps = np.logaddexp(0.0, raw)
        size = np.abs(np64(row)[:, 48:]) + np.abs(np64(bias))
        base._within(dt[live], steps[live], (steps * (3 * size + 16) * 2 * U32)[live], "dt")
        rest = [i for i in range(batch) if i not in live]
        assert (got[rest] == 0).all() and (dt[rest] == 0).all()


# ------------------------------------------------------------------ packed scans: tokens that reset a head
def _fine_scan(x, dt, A, B, C, D, S):
    """One sequence in 64 bits (x [T, H, P], B, C [T, H, n]) -> y, S and bounds of fp32 arithmetic without a factor of all T: a partial sum is rounded where
    it is made and decays with what it holds.  With term_j what token j leaves in the state now and l_j the exponent (base 2) of its decay,
        n = sum_j (tokens since j + 1) |term_j|,   l = sum_j |l_j| |term_j|,   m = sum_j |term_j|.
    Returns y and S, their fp32 error bounds, and the sums of absolute values under both."""
    T, H, P = x.shape
    S, m = S.copy(), np.abs(S)
    n, l = m.copy(), np.zeros_like(m)
    y, ey, my = np.zeros(x.shape), np.zeros(x.shape), np.zeros(x.shape)
    width = B.shape[2]
    for t in range(T):
        d = dt[t] * A
        a = np.exp(d)[:, None, None]
        add = (dt[t][:, None] * x[t])[:, :, None] * B[t][:, None, :]
        # (what is left of l is a power of two far from 1: nothing beyond 2^-200)
        l = a * (l + np.minimum(np.abs(d) / np.log(2), 200.0)[:, None, None] * m)
        S, m = a * S + add, a * m + np.abs(add)
        n = a * n + m
        c = C[t][:, :, None]
        y[t] = (S @ c)[..., 0] + (0 if D is None else D[:, None] * x[t])
        skip = 0 if D is None else np.abs(D[:, None] * x[t])
        my[t] = (m @ np.abs(c))[..., 0] + skip
        # additions and products of the state; up to 32 roundings of an exponent, in sums and products; 64 + n of the product with c and of factors
        ey[t] = (((2 * n + 32 * l) @ np.abs(c))[..., 0] + (128 + width) * my[t]) * 2 * U32
    return y, S, ey, (2 * n + 32 * l + (128 + width) * m) * 2 * U32, my, m


def _heads(H, G, some):
    return [h * G // H for h in some]


def _check_fine(seqs, x, dt, A, B, C, D, pool, slots, fresh, got, after, roundings, some=None, chans=None, pieces=True):
    """Heads `some` and their channels `chans` (None: all) of a packed scan: states as fp32 sums (`pieces`: whose terms go in as two bf16 numbers at
    least, which leave out 2^-16 of one), outputs with `roundings` to bf16 of what they sum, and their own."""
    H, G = x.shape[1], B.shape[1]
    some, chans = list(range(H)) if some is None else some, list(range(x.shape[2])) if chans is None else chans
    gs = _heads(H, G, some)
    X, DT, AA, BB, CC = np64(x[:, some][:, :, chans]), np64(dt[:, some]), np64(A[some]), np64(B[:, gs]), np64(C[:, gs])
    DD, r, half = None if D is None else np64(D[some]), 0, HALF[got.dtype]
    for i, s in enumerate(seqs):
        at = slice(r, r + s[0] + s[1])
        r = at.stop
        S0 = np64(pool[slots[i], some][:, chans]) if pool is not None and not (fresh is not None and fresh[i]) else np.zeros((len(some), len(chans), B.shape[2]))
        y, S, ey, eS, my, m = _fine_scan(X[at], DT[at], AA, BB[at], CC[at], DD, S0)
        inner = ey + roundings * 2.0 ** -8 * (1 + 2.0 ** -7) * my
        base._within(got[at][:, some][:, :, chans], y, inner + half * (np.abs(y) + inner) + 1e-37, "y of sequence %d" % i)
        if after is not None:
            base._within(after[slots[i], some][:, chans], S, eS + (2.0 ** -16 * m if pieces else 0) + 1e-37, "state of sequence %d" % i)


RESETS = [(BF16, 64, 4, 64, 64), (BF16, 32, 2, 128, 64), (BF16, 8, 2, 128, 64), (F32, 8, 2, 64, 64), (BF16, 6, 6, 24, 40)]


@pytest.mark.parametrize("dtype,H,G,n,P", RESETS)
@pytest.mark.parametrize("size", [300.0, 1e4, 1e6, 1e9])
def test_scan_varlen_goes_on_behind_tokens_that_reset_a_head(size, dtype, H, G, n, P):
    """A token in thirty decays its head by e^-size and brings nothing itself: what comes behind it in the same few tokens keeps its weights, which are not
    differences of numbers that large."""
    base._say("scan resets", size, dtype, H, G, n, P)
    seqs = [(700, 5, 0), (290, 10, 0)] + [(i % 7, i % 3 + 1, 0) for i in range(16)]
    rows = sum(s[0] + s[1] for s in seqs)
    x, dt, A, B, C, D = base._scan_case(rows, H, P, G, n, dtype, seed=6)
    dt *= 0.02
    reset = torch.rand((rows, H), generator=torch.Generator().manual_seed(1)) < 1 / 30
    dt[reset] = (-size / A).expand(rows, H)[reset]
    x[reset] = 0
    pool = base._rand(torch.Generator().manual_seed(2), len(seqs), H, P, n)
    state = base._dev(pool)
    y = strd.ssd_prefill_varlen(*(base._dev(t) for t in (x, dt, A, B, C)), seqs, base._dev(D), state=state)
    _check_fine(seqs, x, dt, A, B, C, D, pool, list(range(len(seqs))), None, y, state, 0 if dtype == F32 else 2, some=list(range(0, H, max(1, H // 8))),
                pieces=dtype == BF16)


@pytest.mark.parametrize("H,G,n", [(64, 4, 64), (32, 2, 128)])
def test_scan_varlen_a_reset_does_not_cost_the_steps_that_remember_a_rounding(H, G, n):
    """A reset, one token that writes and many that read it, again and again, with next to nothing forgotten in between: an output is one term, which passes two
    roundings to bf16, of its weight or of the state and its own, however strong the resets are on average.  Terms are a little above 1, where half a step is
    largest, so that three roundings show."""
    base._say("scan resets between steps that remember", H, G, n)
    P, T = 64, 1920
    g = torch.Generator().manual_seed(5)
    x, dt = torch.zeros(T, H, P, dtype=BF16), torch.full((T, H), 1e-3)
    x[1::96] = (1.0 + torch.randint(8, 13, (T // 96, H, P), generator=g) / 128).to(BF16)
    dt[1::96] = 1.0 + 0.05 * torch.rand((T // 96, H), generator=g)
    dt[0::96] = 1e4
    A = -0.6 - 0.1 * torch.rand(H, generator=g)
    B, C = torch.zeros(T, G, n, dtype=BF16), torch.zeros(T, G, n, dtype=BF16)
    B[..., 3] = C[..., 3] = 1
    seqs = [(T, 0, 0)]
    y = strd.ssd_prefill_varlen(*(base._dev(t) for t in (x, dt, A, B, C)), seqs)
    _check_fine(seqs, x, dt, A, B, C, None, None, [0], None, y, None, 1)


# ------------------------------------------------------------------ packed scans: values that are not finite, and where they show
@pytest.mark.parametrize("dtype,H,P,G,n", [(BF16, 64, 64, 4, 64), (BF16, 32, 64, 2, 128), (BF16, 8, 64, 2, 128), (F32, 4, 32, 2, 16), (BF16, 8, 64, 8, 64), (F32, 4, 20, 2, 160)])
@pytest.mark.parametrize("what", ["B", "C", "dt", "state"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_scan_varlen_where_values_that_are_not_finite_show(what, value, dtype, H, P, G, n):
    """One in B: all channels of its group's heads, one in dt: of its head, one in a state: its channel, from its token on and up to 63 tokens before (a state:
    everywhere), and their final states; one in C: its group's heads at its token.  Everything else has the bits that it has without -- but for earlier outputs of a head whose dt is not finite:
    how many pieces a state between segments is made of follows from the decays behind it, so those are off by a rounding at most."""
    base._say("scan not finite", what, value, dtype, H, P, G, n)
    seqs, at = [(700, 0, 0), (40, 0, 0), (900, 5, 0)], 650
    x, dt, A, B, C, D = base._scan_case(1645, H, P, G, n, dtype, slow=True)
    pool = base._rand(torch.Generator().manual_seed(1), 3, H, P, n)
    want_S = base._dev(pool)
    want = strd.ssd_prefill_varlen(*(base._dev(t) for t in (x, dt, A, B, C)), seqs, base._dev(D), state=want_S)
    g, h, p, c = 1, H - 1, 3, 5
    mine = torch.zeros(H, P, dtype=torch.bool)     # heads and channels that it reaches
    if what in ("B", "C"):
        (B if what == "B" else C)[at, g, c] = value
        mine[g * H // G:(g + 1) * H // G] = True
    elif what == "dt":
        dt[at, h] = value
        mine[h] = True
    else:
        pool[0, h, p, c], at = value, 0
        mine[h, p] = True
    state = base._dev(pool)
    y = strd.ssd_prefill_varlen(*(base._dev(t) for t in (x, dt, A, B, C)), seqs, base._dev(D), state=state)
    fine, yes = torch.isfinite(y).cpu(), mine[None].expand(700, H, P)
    last = at + 1 if what == "C" else 700
    assert not fine[at:last][yes[at:last]].any()
    touched = torch.zeros(y.shape, dtype=torch.bool)
    touched[at if what == "C" else max(0, at - 63):last] = mine
    same = (y == want).cpu()
    if what == "dt":
        # two pieces of bf16 or three are 2^-16 of a term apart, which is rounded as part of a state and of the output either way
        my = _fine_scan(*(np64(t) for t in (x[:at, h:], dt[:at, h:], A[h:], B[:at, -1:], C[:at, -1:], D[h:], pool[0, h:])))[4][:at - 63, 0]
        was = np64(want[:at - 63, h])
        assert (np.abs(np64(y[:at - 63, h]) - was) <= 2 * HALF[dtype] * np.abs(was) + (2.0 ** -16 + 2 * HALF[dtype]) * my).all()
        touched[:at, h] = True
    assert same[~touched].all()
    fine_S, same_S, reached = torch.isfinite(state).cpu(), (state == want_S).cpu(), torch.zeros(state.shape, dtype=torch.bool)
    if what != "C":
        reached[0] = mine[..., None]
        assert not fine_S[0].all(-1)[mine].any()
    assert same_S[~reached].all()
