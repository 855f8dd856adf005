"""What serves the rows that a reduced prefill keeps, against plain fp64 forms (oracle/serving.py): packed attention with capped
and biased scores, the 4-bit cache, decode steps that gather weights, eviction, and a run of them together.

Bounds (half a step of bf16 is 2^-8, of fp32 2^-24, relative): the error of an output is the scores' share, which the plain form
gives, plus roundings: of a sum of T products in fp32 (T 2^-24 of sum p |v|), with bf16 tensors of the probabilities and of their
sum (2 * 2^-8 of sum p |v|) and of the output (2^-8)."""
import numpy as np
import pytest
import torch

import paper_2603_00198_amd as strd
from oracle import serving as plain
from paper_2603_00198_amd.synth import np64

pytestmark = pytest.mark.gpu
DEV, BF16, F32 = "cuda", torch.bfloat16, torch.float32


def _say(*a):
    print("[case]", *a, flush=True)


def _slopes(Hq):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)])


def _rand(g, *shape, dtype=F32, size=1.0):
    return (size * torch.randn(shape, generator=g)).to(dtype)


def _within(got, want, bound, what):
    got = np64(got)
    assert np.array_equal(np.isfinite(got), np.isfinite(want)), what + ": finite in other places"
    fine = np.isfinite(want)
    off = np.abs(got - want)[fine] - bound[fine]
    assert (off <= 0).all(), "%s: off by %.3e more than the bound %.3e allows" % (what, off.max(), bound[fine][off.argmax()])


def _out_bound(o, es, mag, dtype, T):
    b = es + T * plain.U32 * mag + 1e-30
    return b + 2.0 ** -24 * np.abs(o) if dtype == F32 else b + 2 * 2.0 ** -8 * mag + 2.0 ** -8 * np.abs(o)


# ------------------------------------------------------------------ attn_prefill_varlen ----
SEQS = {
    "one_row": [(0, 1, 0)],
    "one": [(100, 12, 100)],
    "packed": [(33, 5, 0), (0, 0, 0), (1, 1, 1), (64, 0, 3), (0, 17, 0), (150, 31, 20)],
    "tiles": [(128, 128, 0), (16, 16, 0), (32, 0, 0)],
    "longer": [(700, 41, 0), (300, 3, 0)],
}


def _prefill(seqs, Hq, Hkv, d, dtype, cap, slopes, pos, prefix, seed=0, size=1.5):
    g = torch.Generator().manual_seed(seed + 7)
    rows = sum(s[0] + s[1] for s in seqs)
    q, k, v = _rand(g, rows, Hq, d, dtype=dtype, size=size), _rand(g, rows, Hkv, d, dtype=dtype), _rand(g, rows, Hkv, d, dtype=dtype)
    sl = _slopes(Hq) if slopes else None
    ps = torch.randperm(5 * rows, generator=g)[:rows].to(torch.int32) if pos else None
    return q, k, v, sl, ps


def _dev(t):
    return None if t is None else t.to(DEV)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cap,slopes,pos,prefix", [(0.0, False, False, False), (20.0, False, False, True), (0.0, True, False, True),
                                                   (5.0, True, True, False), (0.0, True, True, True)])
@pytest.mark.parametrize("name,Hq,Hkv,d", [("one_row", 4, 2, 64), ("one", 8, 2, 128), ("packed", 4, 4, 64), ("packed", 7, 1, 128),
                                           ("packed", 6, 2, 96), ("tiles", 4, 1, 128), ("tiles", 3, 1, 33), ("packed", 2, 2, 200),
                                           ("longer", 16, 2, 64)])
def test_prefill_varlen(name, Hq, Hkv, d, cap, slopes, pos, prefix, dtype):
    _say("prefill", name, Hq, Hkv, d, cap, slopes, pos, prefix, dtype)
    seqs = SEQS[name]
    q, k, v, sl, ps = _prefill(seqs, Hq, Hkv, d, dtype, cap, slopes, pos, prefix)
    o = strd.attn_prefill_varlen(_dev(q), _dev(k), _dev(v), seqs, prefix=prefix, cap=cap, slopes=_dev(sl), pos=_dev(ps))
    want, es, mag = plain.attn_varlen(np64(q), np64(k), np64(v), seqs, prefix, cap, None if sl is None else np64(sl),
                                      None if ps is None else ps.numpy())
    _within(o, want, _out_bound(want, es, mag, dtype, max(s[0] + s[1] for s in seqs)), "o")


@pytest.mark.parametrize("dtype,d", [(F32, 64), (BF16, 64), (BF16, 128), (BF16, 96)])
def test_prefill_varlen_spread_scores(dtype, d):
    """Scores far apart, whose reference moves from tile to tile, and a bias that reaches far below it."""
    _say("spread", dtype, d)
    seqs = [(400, 30, 0), (90, 0, 0)]
    q, k, v, _, _ = _prefill(seqs, 4, 2, d, dtype, 0.0, False, False, True, seed=3, size=8.0)
    k *= torch.linspace(0.2, 2.0, k.shape[0])[:, None, None].to(dtype)
    sl = torch.tensor([0.0, 30.0, -0.05, 2.0])
    o = strd.attn_prefill_varlen(_dev(q), _dev(k), _dev(v), seqs, prefix=True, slopes=_dev(sl))
    want, es, mag = plain.attn_varlen(np64(q), np64(k), np64(v), seqs, True, 0.0, np64(sl), None)
    _within(o, want, _out_bound(want, es, mag, dtype, 430), "o")


@pytest.mark.parametrize("dtype,d", [(F32, 64), (BF16, 64), (BF16, 128), (BF16, 96)])
@pytest.mark.parametrize("cap", [1e5, 1e7, 1e10, 3e38])
def test_prefill_varlen_caps_far_above_the_scores(cap, dtype, d):
    """Such a cap leaves scores of up to 30 as they are: 30^3 / (3 cap^2) is below a step.  Its form may add ten roundings of a score, which a
    second share of the score's own bound ((d + 2) roundings of the sum of |q| |k|) covers."""
    _say("far cap", cap, dtype, d)
    seqs = [(200, 30, 0), (90, 0, 0)]
    q, k, v, _, _ = _prefill(seqs, 4, 2, d, dtype, 0.0, False, False, True, seed=4, size=4.0)
    o = strd.attn_prefill_varlen(_dev(q), _dev(k), _dev(v), seqs, prefix=True, cap=cap)
    want, es, mag = plain.attn_varlen(np64(q), np64(k), np64(v), seqs, True, 0.0, None, None)
    _within(o, want, _out_bound(want, 2 * es, mag, dtype, 230), "o")


@pytest.mark.parametrize("dtype,d", [(F32, 64), (BF16, 64), (BF16, 128), (BF16, 96)])
@pytest.mark.parametrize("cap,slopes", [(0.0, False), (20.0, False), (20.0, True)])
def test_prefill_varlen_rows_keep_their_bits_whatever_comes_behind_them(cap, slopes, dtype, d):
    _say("bits", cap, slopes, dtype, d)
    for seqs, Hq, Hkv in (([(300, 30, 0), (90, 0, 0)], 4, 2), ([(600, 0, 0), (90, 0, 0)], 40, 2), ([(1100, 0, 0), (20, 0, 0)], 80, 8)):
        q, k, v, sl, _ = _prefill(seqs, Hq, Hkv, d, dtype, cap, slopes, False, False, seed=6)
        first = strd.attn_prefill_varlen(_dev(q), _dev(k), _dev(v), seqs, cap=cap, slopes=_dev(sl))
        for at in (135, 200):
            for x in (q, k, v):
                x[at:seqs[0][0]] *= 37.0
            o = strd.attn_prefill_varlen(_dev(q), _dev(k), _dev(v), seqs, cap=cap, slopes=_dev(sl))
            assert torch.equal(o[:135], first[:135]) and torch.equal(o[seqs[0][0] + seqs[0][1]:], first[seqs[0][0] + seqs[0][1]:])


@pytest.mark.parametrize("dtype,d", [(F32, 64), (BF16, 64), (BF16, 128), (BF16, 96)])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_prefill_varlen_steep_biases(cap, dtype, d):
    """Every key but a row's own far below it, in blocks that are taken before the row's own as well."""
    _say("steep", cap, dtype, d)
    for seqs, Hq, Hkv in (([(700, 30, 0), (90, 0, 0)], 4, 2), ([(600, 0, 0)], 40, 2), ([(20, 5, 0), (230, 0, 0)], 5, 1)) + (
            (([(1100, 0, 0)], 80, 8),) if d == 128 else ()):
        q, k, v, _, _ = _prefill(seqs, Hq, Hkv, d, dtype, cap, False, False, True, seed=8)
        sl = torch.tensor([1e3, 1e10, 3e38, 0.0, 1e6])[torch.arange(Hq) % 5]
        o = strd.attn_prefill_varlen(_dev(q), _dev(k), _dev(v), seqs, prefix=True, cap=cap, slopes=_dev(sl))
        steep = torch.arange(Hq)[sl > 0]   # exp(-1000) and less is 0: a row's own value is all that is left, with a weight of 1
        assert torch.equal(o[:, steep.to(DEV)], _dev(v[:, steep // (Hq // Hkv)]))
        if Hq > 3:
            want, es, mag = plain.attn_varlen(np64(q[:, 3:4]), np64(k[:, [3 // (Hq // Hkv)]]), np64(v[:, [3 // (Hq // Hkv)]]), seqs, True, cap, None, None)
            _within(o[:, 3:4], want, _out_bound(want, es, mag, dtype, max(s[0] + s[1] for s in seqs)), "o")


@pytest.mark.parametrize("cap", [1e-38, 1e-3])
@pytest.mark.parametrize("dtype,d", [(F32, 64), (BF16, 128)])
def test_prefill_varlen_caps_far_below_the_scores(cap, dtype, d):
    """What is left of the scores is within cap of 0: every key a row sees counts the same to within 2 cap (and its roundings)."""
    _say("near cap", cap, dtype, d)
    seqs = [(100, 30, 0)]
    q, k, v, _, _ = _prefill(seqs, 4, 2, d, dtype, 0.0, False, False, False, seed=4)
    o = strd.attn_prefill_varlen(_dev(q), _dev(k), _dev(v), seqs, cap=cap)
    want, es, mag = plain.attn_varlen(np64(q), np64(k), np64(v), seqs, False, cap, None, None)
    _within(o, want, _out_bound(want, es, mag, dtype, 130), "o")


@pytest.mark.parametrize("dtype,d,Hkv", [(F32, 64, 2), (BF16, 128, 2), (BF16, 64, 4), (BF16, 72, 1)])
def test_prefill_varlen_takes_column_ranges_of_a_projection(dtype, d, Hkv):
    _say("pitched", dtype, d, Hkv)
    seqs, Hq = [(61, 9, 0), (20, 3, 0)], 4
    rows = sum(s[0] + s[1] for s in seqs)
    g = torch.Generator().manual_seed(5)
    wide = _rand(g, rows, (Hq + 2 * Hkv) * d + 8, dtype=dtype).to(DEV)
    q = wide[:, :Hq * d].unflatten(1, (Hq, d))
    k = wide[:, Hq * d:(Hq + Hkv) * d].unflatten(1, (Hkv, d))
    v = wide[:, (Hq + Hkv) * d:(Hq + 2 * Hkv) * d].unflatten(1, (Hkv, d))
    assert not q.is_contiguous()
    out = torch.full((rows, Hq, d), 7.0, dtype=dtype, device=DEV)
    o = strd.attn_prefill_varlen(q, k, v, seqs, cap=10.0, out=out)
    assert o.data_ptr() == out.data_ptr()
    same = strd.attn_prefill_varlen(q.contiguous(), k.contiguous(), v.contiguous(), seqs, cap=10.0)
    assert torch.equal(o, same)
    # two bytes off a 16-byte boundary: the same values by whatever kernel takes them
    odd = torch.empty(rows * (Hq + 2 * Hkv) * d + 1, dtype=dtype, device=DEV)[1:].view(rows, -1)
    odd.copy_(wide[:, :odd.shape[1]])
    o2 = strd.attn_prefill_varlen(odd[:, :Hq * d].unflatten(1, (Hq, d)), odd[:, Hq * d:(Hq + Hkv) * d].unflatten(1, (Hkv, d)),
                                  odd[:, (Hq + Hkv) * d:].unflatten(1, (Hkv, d)), seqs, cap=10.0)
    want, es, mag = plain.attn_varlen(np64(q), np64(k), np64(v), seqs, False, 10.0, None, None)
    for got in (o, o2):
        _within(got, want, _out_bound(want, es, mag, dtype, 70), "o")


def test_prefill_varlen_leaves_rows_behind_the_last_sequence():
    _say("rows behind")
    g = torch.Generator().manual_seed(1)
    for dtype, d in ((F32, 64), (BF16, 128)):
        q, k, v = (_rand(g, 90, 2, d, dtype=dtype).to(DEV) for _ in range(3))
        for t in (q, k, v):
            t[70:] = float("nan")
        o = torch.full((90, 2, d), 3.0, dtype=dtype, device=DEV)
        strd.attn_prefill_varlen(q[:70], k[:70], v[:70], [(50, 3, 0), (17, 0, 0)], prefix=True, out=o[:70])
        assert torch.isfinite(o).all() and (o[70:] == 3.0).all()


@pytest.mark.parametrize("dtype,d", [(F32, 64), (F32, 33), (BF16, 64), (BF16, 128), (BF16, 96)])
@pytest.mark.parametrize("prefix", [False, True])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_prefill_varlen_hidden_rows_that_are_not_finite_do_not_reach_others(dtype, d, prefix, bad):
    """Keys and values that are not finite, in every place of a tile: rows that do not see them come out as without them."""
    _say("not finite", dtype, d, prefix, bad)
    seqs = [(37, 20, 0), (40, 9, 0)]
    rows = sum(s[0] + s[1] for s in seqs)
    q, k, v, _, _ = _prefill(seqs, 4, 2, d, dtype, 0.0, False, False, prefix, seed=2)
    sees = np.zeros((rows, rows), bool)
    r = 0
    for n, m, _ in seqs:
        i = np.arange(n + m)
        sees[r:r + n + m, r:r + n + m] = (i[None] <= i[:, None]) | (prefix & (i[None] < n) & (i[:, None] < n))
        r += n + m
    base = strd.attn_prefill_varlen(_dev(q), _dev(k), _dev(v), seqs, prefix=prefix).cpu()
    for at in (0, 15, 36, 37, 45, 56, 57, 96, 97, 105):
        for which in "kv":
            kk, vv = k.clone(), v.clone()
            (kk if which == "k" else vv)[at, :, ::3] = bad
            o = strd.attn_prefill_varlen(_dev(q), _dev(kk), _dev(vv), seqs, prefix=prefix).cpu()
            hidden = torch.from_numpy(~sees[:, at])
            assert torch.equal(o[hidden], base[hidden]), (at, which)
            seen = ~hidden
            if which == "v":   # the channels of a row that sees it, and no others (a probability of 0 times infinity is NaN)
                assert not torch.isfinite(o[seen][:, :, ::3].float()).any()
                assert torch.equal(o[seen][:, :, 1::3], base[seen][:, :, 1::3])


def test_prefill_varlen_equals_the_causal_call():
    _say("against attn_prefill")
    g = torch.Generator().manual_seed(9)
    for dtype in (F32, BF16):
        q, k, v = _rand(g, 300, 8, 64, dtype=dtype).to(DEV), _rand(g, 300, 2, 64, dtype=dtype).to(DEV), _rand(g, 300, 2, 64, dtype=dtype).to(DEV)
        a = strd.attn_prefill_varlen(q, k, v, [(200, 100, 0)]).float()
        b = strd.attn_prefill(q, k, v).float()
        # both are within the bound of the same numbers: 2 (3 * 2^-8 of the largest |v|, 4), resp. a few hundred steps of fp32
        assert (a - b).abs().max().item() <= (2 * 3 * 2.0 ** -8 * 4.5 if dtype == BF16 else 600 * 2.0 ** -24 * 4.5)


# ------------------------------------------------------------------ the 4-bit cache --------
def _cache(rows, Hkv, d, fill=None):
    c = strd.Kv4Cache.empty(rows, Hkv, d, device=DEV)
    if fill is not None:
        for t in c:
            t.view(torch.uint8).fill_(fill)
    return c


def _equal(got, want):
    a, b = got.float().cpu().numpy(), np.asarray(want, np.float32)
    assert a.shape == b.shape and np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(a[~np.isnan(b)], b[~np.isnan(b)])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,row0,R,Hkv,d", [(1, 0, 1, 1, 32), (40, 7, 29, 3, 64), (20, 19, 1, 8, 128), (9, 0, 9, 2, 96), (5, 2, 0, 2, 64),
                                               (300, 1, 290, 2, 256)])
def test_kv4_store_and_load(rows, row0, R, Hkv, d, dtype):
    _say("kv4", rows, row0, R, Hkv, d, dtype)
    g = torch.Generator().manual_seed(rows + d)
    k = _rand(g, R, Hkv, d, dtype=dtype) + 0.7
    v = _rand(g, R, Hkv, d, dtype=dtype, size=30.0)
    c = _cache(rows, Hkv, d, 0x5A)
    strd.kv4_store(_dev(k), _dev(v), c, row0)
    at = slice(row0, row0 + R)
    out = strd.kv4_load(c, row0, R, dtype=F32)
    out16 = strd.kv4_load(c, row0, R, dtype=BF16)
    for i, x in enumerate((k, v)):
        codes, meta = plain.kv4_quantize(x.float().numpy())
        assert np.array_equal(c[2 * i][at].cpu().numpy(), codes)
        _equal(c[2 * i + 1][at], meta)
        val, _ = plain.kv4_values(codes, meta)
        _equal(out[i], val)
        _equal(out16[i], plain.bf16(val))
        if R:   # what the header promises
            s, z = np.repeat(meta[..., 0], 32, -1), np.repeat(meta[..., 1], 32, -1)
            assert (np.abs(val - x.float().numpy()) <= s * (0.5 + 1 / 16) + np.abs(z) * 2.0 ** -8).all()
    rest = torch.ones(rows, dtype=torch.bool)
    rest[at] = False
    for t in c:
        assert (t[rest.to(DEV)].view(torch.uint8) == 0x5A).all()


def test_kv4_groups_at_the_ends_of_the_range():
    """Equal values, steps that round to 0, zeros, the largest numbers, ties of the quotient, values that are not finite."""
    _say("kv4 ends")
    x = torch.zeros(12, 1, 64)
    x[0] = 3.1415927
    x[1] = torch.linspace(0, 1e-31, 64)
    x[2] = torch.linspace(-3e38, 3e38, 64)
    x[3] = torch.linspace(-1.6e38, 1.6e38, 64)
    x[4] = torch.arange(64) * 0.25          # quotients of a half
    x[5] = (torch.arange(64) % 31) * 0.5
    x[6, 0, 5] = float("nan")
    x[7, 0, 40] = float("inf")
    x[8, 0, 0], x[8, 0, 63] = -float("inf"), float("inf")
    x[9] = 3.4e38
    x[10] = 1e5 + torch.arange(64) / 64
    x[11] = -torch.arange(64) * 1e-38
    for dtype in (F32, BF16):
        y = x.to(dtype)
        c = _cache(12, 1, 64)
        strd.kv4_store(_dev(y), _dev(-y), c, 0)
        got = strd.kv4_load(c, 0, 12, dtype=F32)
        for i, z in enumerate((y, -y)):
            codes, meta = plain.kv4_quantize(z.float().numpy())
            _equal(c[2 * i + 1], meta)
            _equal(got[i], plain.kv4_values(codes, meta)[0])


def test_kv4_store_takes_column_ranges():
    _say("kv4 pitched")
    for dtype in (F32, BF16):
        for shift in (0, 3):   # 3: rows that cannot be read as vectors
            g = torch.Generator().manual_seed(shift)
            wide = _rand(g, 21, 2 * 2 * 64 + 16 + shift, dtype=dtype).to(DEV)
            k, v = wide[:, shift:shift + 128].unflatten(1, (2, 64)), wide[:, shift + 128:shift + 256].unflatten(1, (2, 64))
            a, b = _cache(21, 2, 64), _cache(21, 2, 64)
            strd.kv4_store(k, v, a, 0)
            strd.kv4_store(k.contiguous(), v.contiguous(), b, 0)
            assert all(torch.equal(x, y) for x, y in zip(a, b))


# ------------------------------------------------------------------ decode steps -----------
def _decode_case(T, Hq, Hkv, d, dtype, kv4, slopes, pos, seed=0, size=1.5):
    g = torch.Generator().manual_seed(T + 31 * d + seed)
    q = _rand(g, Hq, d, dtype=dtype, size=size)
    k, v = _rand(g, T, Hkv, d, dtype=dtype) + 0.3, _rand(g, T, Hkv, d, dtype=dtype)
    sl = _slopes(Hq) if slopes else None
    ps = torch.randperm(3 * T, generator=g)[:T].sort().values.to(torch.int32) if pos else None
    w = torch.rand(T, generator=g)
    return q, k, v, sl, ps, w


def _decode_check(q, k, v, sl, ps, w, cap, kv4, spare=0, w_out=None):
    T, Hkv, d = k.shape
    sln, psn = None if sl is None else np64(sl), None if ps is None else ps.numpy()
    if kv4:
        c = _cache(T + spare, Hkv, d, 0xFF)   # rows behind T hold NaN
        strd.kv4_store(_dev(k), _dev(v), c, 0)
        kk = plain.kv4_values(*plain.kv4_quantize(k.float().numpy()))[0].astype(np.float64)
        vv, part = (a.astype(np.float64) for a in plain.kv4_values(*plain.kv4_quantize(v.float().numpy())))
        o, got = strd.attn_decode_step_kv4(_dev(q), c, T, cap=cap, slopes=_dev(sl), pos=_dev(ps), weights=_dev(w), weights_out=w_out)
        want, ww, es, mag, ew = plain.decode(np64(q), kk, vv, cap, sln, psn, None if w is None else np64(w), vmag=np.abs(part) + np.abs(vv))
    else:
        o, got = strd.attn_decode_step_weights(_dev(q), _dev(k), _dev(v), cap=cap, slopes=_dev(sl), pos=_dev(ps), weights=_dev(w), weights_out=w_out)
        want, ww, es, mag, ew = plain.decode(np64(q), np64(k), np64(v), cap, sln, psn, None if w is None else np64(w))
    # (a sum of T products goes through chains of a few hundred at most)
    _within(o, want, _out_bound(want, es, mag, q.dtype, min(T, 512)), "o")
    _within(got, ww, ew + min(T, 512) * plain.U32 * np.abs(ww) + 1e-30, "weights")
    return o, got


@pytest.mark.parametrize("kv4", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,Hq,Hkv,d,cap,slopes,pos", [
    (1, 4, 2, 64, 0.0, False, False), (2, 8, 2, 128, 30.0, True, False), (31, 4, 4, 128, 0.0, False, False), (33, 7, 1, 64, 5.0, False, False),
    (100, 6, 2, 96, 10.0, True, True), (843, 32, 8, 128, 0.0, True, True), (1000, 16, 1, 64, 50.0, False, False), (777, 10, 2, 128, 0.0, True, False),
    (2500, 16, 2, 128, 20.0, True, True), (300, 40, 1, 128, 0.0, False, False), (500, 2, 2, 256, 8.0, True, True), (70, 3, 3, 32, 0.0, False, False)])
def test_decode_steps(T, Hq, Hkv, d, cap, slopes, pos, dtype, kv4):
    _say("decode", T, Hq, Hkv, d, cap, slopes, pos, dtype, kv4)
    _decode_check(*_decode_case(T, Hq, Hkv, d, dtype, kv4, slopes, pos), cap, kv4, spare=5)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,Hq,Hkv,d", [(20011, 8, 2, 128), (33000, 4, 2, 64)])
def test_decode_steps_long(T, Hq, Hkv, d, dtype):
    for kv4 in (True, False):
        _say("decode long", T, Hq, Hkv, d, dtype, kv4)
        _decode_check(*_decode_case(T, Hq, Hkv, d, dtype, kv4, True, True), 30.0, kv4)


@pytest.mark.parametrize("kv4", [True, False])
@pytest.mark.parametrize("d,dtype", [(64, BF16), (128, BF16), (128, F32)])
def test_decode_spread_scores(d, dtype, kv4):
    """References that rise late and far, and one row that takes it all."""
    _say("decode spread", d, dtype, kv4)
    q, k, v, sl, ps, w = _decode_case(1500, 8, 2, d, dtype, kv4, False, False, seed=4, size=6.0)
    k *= torch.linspace(0.1, 2.0, 1500)[:, None, None].to(dtype)
    k[1203] = (3 * q.view(2, 4, d)[:, 1]).to(dtype)
    _decode_check(q, k, v, sl, ps, w, 0.0, kv4)


@pytest.mark.parametrize("T,Hq,Hkv,d", [(843, 32, 8, 128), (2000, 8, 2, 64), (33, 4, 4, 128)])
@pytest.mark.parametrize("kv4", [True, False])
def test_decode_takes_a_query_that_wide_reads_do_not_fit(T, Hq, Hkv, d, kv4):
    """It runs on the other kernel, whose shares of the cache are others, in the same workspace (and not behind it)."""
    _say("odd query", T, Hq, Hkv, d, kv4)
    q, k, v, sl, ps, w = _decode_case(T, Hq, Hkv, d, BF16, kv4, True, True)
    wide = torch.zeros(Hq * d + 8, dtype=BF16, device=DEV)
    odd = wide[1:1 + Hq * d].view(Hq, d)
    odd.copy_(q)
    c = _cache(T, Hkv, d)
    strd.kv4_store(_dev(k), _dev(v), c, 0)
    need = (strd.binding.lib().strd_attn_decode_step_kv4_workspace if kv4 else strd.binding.lib().strd_attn_decode_step_weights_workspace)(T, Hq, Hkv, d, 1, 1)
    room = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
    more = dict(cap=20.0, slopes=_dev(sl), pos=_dev(ps), weights=_dev(w), ws=room[:need])
    o, got = strd.attn_decode_step_kv4(odd, c, T, **more) if kv4 else strd.attn_decode_step_weights(odd, _dev(k), _dev(v), **more)
    kk, vv, part = np64(k), np64(v), np.zeros(1)
    if kv4:
        kk = plain.kv4_values(*plain.kv4_quantize(k.float().numpy()))[0].astype(np.float64)
        vv, part = (a.astype(np.float64) for a in plain.kv4_values(*plain.kv4_quantize(v.float().numpy())))
    want, ww, es, mag, ew = plain.decode(np64(q), kk, vv, 20.0, np64(sl), ps.numpy(), np64(w), vmag=np.abs(part) + np.abs(vv))
    _within(o, want, _out_bound(want, es, mag, BF16, min(T, 512)), "o")
    _within(got, ww, ew + min(T, 512) * plain.U32 * np.abs(ww) + 1e-30, "weights")
    assert (room[need:] == 0x5A).all()


@pytest.mark.parametrize("d,dtype", [(64, BF16), (128, BF16), (96, BF16), (128, F32)])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_decode_heads_keep_their_bits_whatever_the_others_do(cap, d, dtype):
    _say("decode bits", cap, d, dtype)
    q, k, v, _, _, _ = _decode_case(500, 8, 2, d, dtype, False, False, False)
    first, _ = strd.attn_decode_step_weights(_dev(q), _dev(k), _dev(v), cap=cap)
    q[1::2] *= 37.0
    o, _ = strd.attn_decode_step_weights(_dev(q), _dev(k), _dev(v), cap=cap)
    assert torch.equal(o[0::2], first[0::2])


@pytest.mark.parametrize("cap", [1e-38, 1e7, 3e38])
@pytest.mark.parametrize("d,dtype", [(64, BF16), (128, BF16), (96, BF16), (128, F32)])
def test_decode_caps_far_from_the_scores(cap, d, dtype):
    """Far above them it leaves them as they are (see the packed form's test), far below it leaves nothing of them."""
    _say("decode far cap", cap, d, dtype)
    q, k, v, _, _, w = _decode_case(333, 8, 2, d, dtype, False, False, False, size=4.0)
    o, got = strd.attn_decode_step_weights(_dev(q), _dev(k), _dev(v), cap=cap, weights=_dev(w))
    want, ww, es, mag, ew = plain.decode(np64(q), np64(k), np64(v), cap if cap < 1 else 0.0, None, None, np64(w))
    _within(o, want, _out_bound(want, 2 * es, mag, dtype, 333), "o")
    _within(got, ww, 2 * ew + 333 * plain.U32 * np.abs(ww) + 1e-30, "weights")


@pytest.mark.parametrize("kv4", [True, False])
@pytest.mark.parametrize("d,dtype", [(64, BF16), (128, BF16), (96, BF16), (128, F32)])
def test_decode_weights_in_place_none_in_and_none_out(d, dtype, kv4):
    _say("decode weights", d, dtype, kv4)
    q, k, v, sl, ps, w = _decode_case(333, 8, 2, d, dtype, kv4, True, True)
    o, first = _decode_check(q, k, v, sl, ps, w, 20.0, kv4)
    own = _dev(w)
    c = _cache(333, 2, d)
    strd.kv4_store(_dev(k), _dev(v), c, 0)
    more = dict(cap=20.0, slopes=_dev(sl), pos=_dev(ps))
    call = (lambda **kw: strd.attn_decode_step_kv4(_dev(q), c, 333, **more, **kw)) if kv4 else \
        (lambda **kw: strd.attn_decode_step_weights(_dev(q), _dev(k), _dev(v), **more, **kw))
    o2, same = call(weights=own, weights_out=own)
    assert same.data_ptr() == own.data_ptr() and torch.equal(own, first) and torch.equal(o, o2)
    o3, none = call(want_weights=False)
    assert none is None and torch.equal(o, o3)
    o4, fresh = call()
    assert torch.equal(o, o4)
    # each step's weights add up to 1: 333 sums and two exponentials of some steps each
    assert abs(fresh.double().sum().item() - 1) <= 600 * 2.0 ** -24 + 64 * 2.0 ** -22
    assert ((first - _dev(w)) - fresh).abs().max().item() <= 2.0 ** -23 * 2


@pytest.mark.parametrize("kv4", [True, False])
def test_decode_rows_that_are_not_finite(kv4):
    """A row with NaN keys makes its head's results NaN, a NaN value its channels (4 bits: its group of channels)."""
    _say("decode not finite", kv4)
    for d, dtype in ((128, BF16), (64, BF16), (96, F32)):
        q, k, v, _, _, _ = _decode_case(150, 4, 2, d, dtype, kv4, False, False)
        v[149, 1, 5] = float("nan")
        c = _cache(150, 2, d)
        strd.kv4_store(_dev(k), _dev(v), c, 0)
        o, w = strd.attn_decode_step_kv4(_dev(q), c, 150) if kv4 else strd.attn_decode_step_weights(_dev(q), _dev(k), _dev(v))
        bad = torch.zeros(4, d, dtype=torch.bool)
        bad[2:, :32] = True if kv4 else bad[2:, :32]
        bad[2:, 5] = True
        assert torch.equal(torch.isnan(o).cpu(), bad) and torch.isfinite(w).all()
        k[20, 0] = float("nan")
        strd.kv4_store(_dev(k), _dev(v), c, 0)
        o, w = strd.attn_decode_step_kv4(_dev(q), c, 150) if kv4 else strd.attn_decode_step_weights(_dev(q), _dev(k), _dev(v))
        assert torch.isnan(o[:2]).all() and torch.isnan(w).all()


# ------------------------------------------------------------------ eviction ---------------
@pytest.mark.parametrize("T,K,first,last", [(1, 1, 0, 0), (7, 7, 2, 3), (50, 5, 2, 3), (50, 20, 0, 0), (64, 63, 4, 0), (1075, 512, 4, 64),
                                            (4096, 1000, 0, 1), (5000, 1700, 1500, 100), (8363, 2176, 4, 128), (20000, 3000, 4, 2000),
                                            (33000, 9000, 4, 128), (70001, 17000, 4500, 513), (40000, 39999, 1, 1)])
@pytest.mark.parametrize("kind", ["spread", "ties", "odd"])
def test_evict(T, K, first, last, kind):
    _say("evict", T, K, first, last, kind)
    g = torch.Generator().manual_seed(T + K)
    w = torch.exp(2 * torch.randn(T, generator=g)) / T
    if kind == "ties":
        w = torch.randint(0, 3, (T,), generator=g).float()
    if kind == "odd":
        w[torch.rand(T, generator=g) < 0.3] = 0.0
        w[T // 2] = float("inf")
        w[0] = -1.0
    pos = torch.randperm(4 * T, generator=g)[:T].to(torch.int32)
    rows = [torch.randint(-128, 127, (T, 3, 16), generator=g, dtype=torch.int8), torch.randn(T, 5, generator=g), torch.randn(T, 2, 64, generator=g).to(BF16)]
    idx, kw, out, kp = strd.cache_evict(_dev(w), K, first, last, [_dev(t) for t in rows], pos=_dev(pos))
    want = torch.from_numpy(plain.evict(w.numpy(), K, first, last))
    assert torch.equal(idx.cpu().long(), want)
    assert torch.equal(kw.cpu(), w[want]) and torch.equal(kp.cpu(), pos[want])
    for a, b in zip(out, rows):
        assert torch.equal(a.cpu(), b[want])


def test_evict_into_given_tensors_and_without_any():
    _say("evict outs")
    w = torch.rand(300, device=DEV)
    x = torch.randn(300, 4, device=DEV)
    y = torch.empty(40, 4, device=DEV)
    idx, kw, out, kp = strd.cache_evict(w, 40, 4, 8, [x], outs=[y])
    assert out[0].data_ptr() == y.data_ptr() and torch.equal(y, x[idx.long()]) and kp is None
    idx2, kw2, none, _ = strd.cache_evict(w, 40, 4, 8, [])
    assert torch.equal(idx, idx2) and torch.equal(kw, kw2) and none == []


# ------------------------------------------------------------------ together ---------------
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 96)])
def test_prefill_store_decode_evict_together(dtype, d):
    """A reduced prompt goes through packed attention, into the 4-bit cache, tokens are generated with a cap and a bias by the old
    positions, the cache is cut down by the weights that the steps gathered, and generation goes on."""
    _say("together", dtype, d)
    Hq, Hkv, N, M, K, new, cap = 8, 2, 400, 24, 180, 6, 30.0
    g = torch.Generator().manual_seed(d)
    rows, room = N + M + 2 * new, K + M + new
    q, k, v = _rand(g, rows, Hq, d, dtype=dtype, size=1.5), _rand(g, rows, Hkv, d, dtype=dtype) + 0.2, _rand(g, rows, Hkv, d, dtype=dtype)
    sl, qd, kd, vd = _slopes(Hq), _dev(q), _dev(k), _dev(v)
    # reduced prefill: score, select, compact, attend at the old positions
    s = strd.score_attn(qd[N:N + M], kd[:N])
    idx = strd.select_topk(s, K)
    (qc, kc, vc), pos = strd.compact_batch([qd[:N + M], kd[:N + M], vd[:N + M]], idx, N, M, want_pos=True)
    o = strd.attn_prefill_varlen(qc, kc, vc, [(K, M, K)], prefix=True, cap=cap, slopes=_dev(sl), pos=pos)
    p64 = pos.cpu().numpy()
    want, es, mag = plain.attn_varlen(np64(qc), np64(kc), np64(vc), [(K, M, K)], True, cap, np64(sl), p64)
    _within(o, want, _out_bound(want, es, mag, dtype, K + M), "prefill")
    # into the cache, with room for new rows
    cache, T = strd.Kv4Cache.empty(room, Hkv, d, device=DEV), K + M
    strd.kv4_store(kc, vc, cache, 0)
    held = [plain.kv4_quantize(x.float().cpu().numpy()) for x in (kc, vc)]
    positions = torch.zeros(room, dtype=torch.int32, device=DEV)
    positions[:T] = pos
    weights = torch.zeros(room, device=DEV)
    w64, wb, at = np.zeros(T), np.zeros(T), N + M
    for part in range(2):
        for _ in range(new):
            strd.kv4_store(kd[at:at + 1], vd[at:at + 1], cache, T)
            positions[T:T + 1] = at
            held = [tuple(np.concatenate([a, b]) for a, b in zip(h, plain.kv4_quantize(x[at:at + 1].float().numpy()))) for h, x in zip(held, (k, v))]
            p64, w64, wb = np.append(p64, at), np.append(w64, 0.0), np.append(wb, 0.0)
            T, at = T + 1, at + 1
            o, _ = strd.attn_decode_step_kv4(qd[at - 1], cache, T, cap=cap, slopes=_dev(sl), pos=positions, weights=weights, weights_out=weights)
            kk, (vv, sn) = plain.kv4_values(*held[0])[0], plain.kv4_values(*held[1])
            want, w64, es, mag, ew = plain.decode(np64(q[at - 1]), kk.astype(float), vv.astype(float), cap, np64(sl), p64, w64, vmag=np.abs(sn) + np.abs(vv))
            _within(o, want, _out_bound(want, es, mag, dtype, T), "step")
            wb = wb + ew + T * plain.U32 * w64
        _within(weights[:T], w64, wb + 1e-30, "weights")
        if part == 0:
            keep = 100
            kept, weights_k, cut, pos_k = strd.cache_evict(weights[:T], keep, 4, 20, [t[:T] for t in cache], pos=positions[:T])
            i = kept.cpu().numpy()
            assert np.array_equal(i, plain.evict(weights[:T].cpu().numpy(), keep, 4, 20))
            for a, b in zip(cache, cut):
                a[:keep] = b
            weights[:keep], positions[:keep], T = weights_k, pos_k, keep
            weights[keep:] = 0
            held = [tuple(a[i] for a in h) for h in held]
            p64, w64, wb = p64[i], w64[i], wb[i]


@pytest.mark.parametrize("seed", range(40))
def test_random_shapes_prefill(seed):
    rng = np.random.default_rng(seed)
    Hkv = int(rng.integers(1, 5))
    Hq, d = Hkv * int(rng.integers(1, 9)), int(rng.choice([64, 128, 64, 128, 96, 40, 160]))
    dtype = F32 if rng.random() < 0.25 else BF16
    seqs, left = [], int(2 ** rng.uniform(1, 10.5))
    while left > 0 and len(seqs) < 16:
        t = left if rng.random() < 0.3 or len(seqs) == 15 else int(rng.integers(0, left + 1))
        m = int(rng.integers(0, t + 1)) if rng.random() < 0.3 else int(rng.integers(0, t // 8 + 1))
        seqs.append((t - m, m, 0))
        left -= t
    cap, prefix = float(rng.choice([0.0, 0.0, 1.0, 5.0, 30.0])), bool(rng.random() < 0.5)
    slopes, pos, pad = bool(rng.random() < 0.5), bool(rng.random() < 0.5), int(rng.choice([0, 0, 8, 3]))
    _say("random prefill", seed, seqs, Hq, Hkv, d, dtype, cap, prefix, slopes, pos, pad)
    q, k, v, sl, ps = _prefill(seqs, Hq, Hkv, d, dtype, cap, slopes, pos, prefix, seed=seed)
    rows = q.shape[0]
    wide = torch.cat([x.flatten(1) for x in (q, k, v)] + [torch.zeros(rows, pad, dtype=dtype)], 1).to(DEV)
    parts = [x.unflatten(1, (h, d)) for x, h in zip(wide[:, :(Hq + 2 * Hkv) * d].split([Hq * d, Hkv * d, Hkv * d], 1), (Hq, Hkv, Hkv))]
    o = strd.attn_prefill_varlen(*parts, seqs, prefix=prefix, cap=cap, slopes=_dev(sl), pos=_dev(ps))
    want, es, mag = plain.attn_varlen(np64(q), np64(k), np64(v), seqs, prefix, cap, None if sl is None else np64(sl), None if ps is None else ps.numpy())
    _within(o, want, _out_bound(want, es, mag, dtype, max(s[0] + s[1] for s in seqs)), "o")


@pytest.mark.parametrize("seed", range(40))
def test_random_shapes_decode(seed):
    rng = np.random.default_rng(100 + seed)
    Hkv, kv4 = int(rng.integers(1, 10)), bool(rng.random() < 0.6)
    Hq, d = Hkv * int(rng.integers(1, 13)), int(rng.choice([64, 128, 64, 128, 96, 32, 256] if kv4 else [64, 128, 64, 128, 96, 40, 200]))
    dtype, T = F32 if rng.random() < 0.25 else BF16, int(2 ** rng.uniform(0, 13))
    cap, slopes, pos = float(rng.choice([0.0, 0.0, 1.0, 5.0, 30.0])), bool(rng.random() < 0.5), bool(rng.random() < 0.5)
    _say("random decode", seed, T, Hq, Hkv, d, dtype, kv4, cap, slopes, pos)
    _decode_check(*_decode_case(T, Hq, Hkv, d, dtype, kv4, slopes, pos, seed=seed), cap, kv4, spare=int(rng.integers(0, 3)))


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes_evict(seed):
    rng = np.random.default_rng(200 + seed)
    T = int(2 ** rng.uniform(0, 17.5))
    K = int(rng.integers(1, T + 1))
    first = int(rng.integers(0, K + 1)) if rng.random() < 0.3 else min(K, int(rng.integers(0, 200)))
    last = int(rng.integers(0, K - first + 1)) if rng.random() < 0.3 else min(K - first, int(rng.integers(0, 200)))
    _say("random evict", seed, T, K, first, last)
    w = torch.from_numpy(rng.random(T).astype(np.float32))
    if seed % 3 == 0:
        w = (w * 50).floor()
    rows, pos = torch.arange(3 * T, dtype=torch.int32).view(T, 3), torch.arange(T, dtype=torch.int32) * 2
    idx, kw, (out,), kp = strd.cache_evict(_dev(w), K, first, last, [_dev(rows)], pos=_dev(pos))
    want = torch.from_numpy(plain.evict(w.numpy(), K, first, last))
    assert torch.equal(idx.cpu().long(), want) and torch.equal(kw.cpu(), w[want]) and torch.equal(kp.cpu(), pos[want])
    assert torch.equal(out.cpu(), rows[want])


def _calls():
    g = torch.Generator().manual_seed(11)
    q, k, v = _rand(g, 200, 8, 64, dtype=BF16).to(DEV), _rand(g, 200, 2, 64, dtype=BF16).to(DEV), _rand(g, 200, 2, 64, dtype=BF16).to(DEV)
    sl, pos, w = _slopes(8).to(DEV), torch.arange(0, 400, 2, dtype=torch.int32, device=DEV), torch.rand(200, device=DEV)
    cache = _cache(200, 2, 64, 0)
    strd.kv4_store(k, v, cache, 0)
    wo = torch.empty(200, device=DEV)

    def every():
        strd.kv4_store(k, v, cache, 0)
        a = strd.attn_prefill_varlen(q, k, v, [(100, 20, 0), (70, 10, 0)], prefix=True, cap=9.0, slopes=sl, pos=pos)
        b, c = strd.attn_decode_step_kv4(q[7], cache, 200, cap=9.0, slopes=sl, pos=pos, weights=w, weights_out=wo)
        d, e = strd.attn_decode_step_weights(q[7], k, v, weights=w)
        idx, kw, rows, kp = strd.cache_evict(c, 50, 4, 10, list(cache), pos=pos)
        f, h = strd.kv4_load(strd.Kv4Cache(*rows), 0, 50)
        return [a, b, c, d, e, idx, kw, kp, f, h]
    return every


def test_captured_calls_replay_as_they_run():
    _say("graph")
    every = _calls()
    want = [t.clone() for t in every()]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        every()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = every()
    for _ in range(3):
        for t in outs:
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        again = every()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, want))


def test_calls_on_two_streams_at_once():
    _say("streams")
    one, two = _calls(), _calls()
    want_a, want_b = [t.clone() for t in one()], [t.clone() for t in two()]   # (their weights are drawn apart)
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(5):
        with torch.cuda.stream(sa):
            a = one()
        with torch.cuda.stream(sb):
            b = two()
        got += [(want_a, a), (want_b, b)]
    torch.cuda.synchronize()
    for want, outs in got:
        assert all(torch.equal(x, y) for x, y in zip(outs, want))
