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


# ------------------------------------------------------------------ decode steps: weights in full --
@pytest.mark.parametrize("kv4", [True, False])
@pytest.mark.parametrize("T,Hq,Hkv,d,dtype", [(100, 8, 2, 128, BF16), (100, 8, 2, 64, BF16), (843, 16, 2, 128, BF16), (843, 32, 2, 64, BF16), (300, 8, 2, 96, BF16),
                                              (300, 8, 2, 128, F32)])
def test_decode_rows_of_equal_values_come_out_as_these(T, Hq, Hkv, d, dtype, kv4):
    """The weights add up to 1 whatever they are: here 7 of 8 are the same number below 1 before they are divided by their sum, which 8 bits would
    round by up to 2^-8.  Kept to 16 bits or more they are off by 2^-16, 8 steps of the 4-bit cache by 2^-13: values come out exactly, 0 below 2^-12."""
    base._say("equal values", T, Hq, Hkv, d, dtype, kv4)
    v = torch.arange(d).remainder(16).float().expand(T, Hkv, d).to(dtype).contiguous()   # (in 4 bits: step 1, middle 8)
    q, k = torch.zeros(Hq, d, dtype=dtype), torch.zeros(T, Hkv, d, dtype=dtype)
    k[::8, :, 0] = 1
    for i in range(24):
        q[:, 0] = (0.03 * (i + 1) + 0.01 * torch.arange(Hq)) * d ** 0.5
        if kv4:
            c = base._cache(T, Hkv, d)
            strd.kv4_store(base._dev(k), base._dev(v), c, 0)
            o, w = strd.attn_decode_step_kv4(base._dev(q), c, T)
        else:
            o, w = strd.attn_decode_step_weights(base._dev(q), base._dev(k), base._dev(v))
        o, want = o.float().cpu(), v[0, 0].float().expand(Hq, d)
        if dtype == BF16:
            assert torch.equal(o[want > 0], want[want > 0]), i
        assert (o - want).abs().max() <= 2.0 ** -12, i
        assert abs(w.double().sum().item() - 1) <= (T + 64) * 2.0 ** -24


@pytest.mark.parametrize("T,Hq,Hkv,d", [(100, 8, 2, 128), (843, 16, 2, 64), (100, 8, 2, 96)])
def test_decode_rows_with_infinite_values(T, Hq, Hkv, d):
    """Every row has a weight above 0: an infinite value is the result of its channel, of either sign."""
    base._say("infinite values", T, Hq, Hkv, d)
    q, k, v, _, _, _ = base._decode_case(T, Hq, Hkv, d, BF16, False, False, False)
    for at in (0, 17, T - 1):
        x = v.clone()
        x[at, :, 3], x[at, :, 40] = float("inf"), -float("inf")
        o, _ = strd.attn_decode_step_weights(base._dev(q), base._dev(k), base._dev(x))
        assert (o[:, 3] == float("inf")).all() and (o[:, 40] == -float("inf")).all(), at
        o[:, 3] = o[:, 40] = 0
        assert torch.isfinite(o.float()).all()


# ------------------------------------------------------------------ the loop in the README ---
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 96)])
def test_the_loop_in_the_readme_goes_on_behind_a_full_cache(dtype, d):
    """As it stands there, over two evictions; the last step against the plain form over the rows that the cache then holds."""
    import os
    base._say("readme", dtype, d)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    block = next(b for b in open(os.path.join(root, "README.md")).read().split("```") if "cache_evict(" in b and b.startswith("python"))
    g = torch.Generator().manual_seed(d)
    Hq, Hkv, K0, M0, K1, M1, rows, K, new = 8, 2, 150, 10, 70, 5, 230, 170, 165
    pos = torch.cat([torch.randperm(4 * n, generator=g)[:n].sort().values for n in (K0 + M0, K1 + M1)]).to(torch.int32)
    total = K0 + M0 + K1 + M1
    q, k, v = (base._rand(g, total, h, d, dtype=dtype).to("cuda") for h in (Hq, Hkv, Hkv))
    tokens = [(base._rand(g, Hq, d, dtype=dtype, size=1.5).to("cuda"), base._rand(g, 1, Hkv, d, dtype=dtype).to("cuda"),
               base._rand(g, 1, Hkv, d, dtype=dtype).to("cuda"), 1000 + i) for i in range(new)]
    names = dict(strd=strd, torch=torch, q=q, k=k, v=v, pos=pos.to("cuda"), slopes=base._slopes(Hq).to("cuda"), tokens=tokens, Hq=Hq, Hkv=Hkv, d=d, K0=K0,
                 M0=M0, K1=K1, M1=M1, rows=rows, K=K)
    exec(block[len("python"):], names)
    T, place = names["T"], names["place"].cpu().numpy()
    assert T == K + (K0 + M0 + new - rows) - (rows - K)      # 70 rows till it is full, 60 more, then what is left
    assert (np.diff(place[:T]) > 0).all() and place[T - 1] == 1000 + new - 1 and (place[:4] == pos[:4].numpy()).all()
    held = [t[:T].cpu() for t in names["cache"]]
    (kk, _), (vv, part) = (plain.kv4_values(codes.numpy(), meta.float().numpy()) for codes, meta in (held[:2], held[2:]))
    want, _, es, mag, _ = plain.decode(np64(tokens[-1][0]), kk.astype(float), vv.astype(float), 50.0, np64(base._slopes(Hq)), place[:T],
                                       vmag=np.abs(part) + np.abs(vv))
    base._within(names["o1"], want, base._out_bound(want, es, mag, dtype, T), "o1")
    assert (names["w"][:T] > 0).all() and (names["w"][T:] == 0).all()


# ------------------------------------------------------------------ every kernel against the plain forms --
def _heads(Hq, Hkv, some=5):
    """Some query heads and their kv heads, the first and the last among them."""
    h = np.unique(np.linspace(0, Hq - 1, min(some, Hq)).astype(int))
    return h, h // (Hq // Hkv)


def _plain_prefill(q, k, v, seqs, prefix, cap, sl, ps, heads, kv):
    """The plain form of some query heads, one kv head to each."""
    return plain.attn_varlen(np64(q[:, heads]), np64(k[:, kv]), np64(v[:, kv]), seqs, prefix, cap, None if sl is None else np64(sl[heads]),
                             None if ps is None else ps.numpy())


@pytest.mark.parametrize("kernel,prefix", _prefill_kernels())
@pytest.mark.parametrize("cap,slopes,pos", [(0.0, False, False), (20.0, False, False), (0.0, True, True), (2.0, True, False)])
def test_prefill_varlen_every_kernel(kernel, prefix, cap, slopes, pos):
    dtype, d, seqs, Hq, Hkv, _ = PREFILL[kernel]
    base._say("every prefill kernel", kernel, prefix, cap, slopes, pos)
    q, k, v, sl, ps = base._prefill(seqs, Hq, Hkv, d, dtype, cap, slopes, pos, prefix, seed=11)
    o = strd.attn_prefill_varlen(base._dev(q), base._dev(k), base._dev(v), seqs, prefix=prefix, cap=cap, slopes=base._dev(sl), pos=base._dev(ps))
    heads, kv = _heads(Hq, Hkv)
    want, es, mag = _plain_prefill(q, k, v, seqs, prefix, cap, sl, ps, heads, kv)
    base._within(o[:, heads], want, base._out_bound(want, es, mag, dtype, max(s[0] + s[1] for s in seqs)), "o")


@pytest.mark.parametrize("kernel,prefix", _prefill_kernels())
def test_prefill_varlen_every_kernel_spread_scores(kernel, prefix):
    """References that move from tile to tile; a bias that is steep, none, one that favours what is far."""
    dtype, d, seqs, Hq, Hkv, _ = PREFILL[kernel]
    base._say("spread, every kernel", kernel, prefix)
    q, k, v, _, _ = base._prefill(seqs, Hq, Hkv, d, dtype, 0.0, False, False, prefix, seed=12, size=8.0)
    k *= torch.linspace(0.2, 2.0, k.shape[0])[:, None, None].to(dtype)
    heads, kv = _heads(Hq, Hkv)
    for sl in (None, torch.tensor([30.0, 0.0, -0.02, 2.0, 1e7])[torch.arange(Hq) % 5]):
        o = strd.attn_prefill_varlen(base._dev(q), base._dev(k), base._dev(v), seqs, prefix=prefix, slopes=base._dev(sl))
        want, es, mag = _plain_prefill(q, k, v, seqs, prefix, 0.0, sl, None, heads, kv)
        base._within(o[:, heads], want, base._out_bound(want, es, mag, dtype, max(s[0] + s[1] for s in seqs)), "o")


@pytest.mark.parametrize("kernel,prefix", _prefill_kernels())
@pytest.mark.parametrize("cap,slopes", [(0.0, False), (20.0, True)])
def test_prefill_varlen_every_kernel_hides_what_is_not_finite(kernel, prefix, cap, slopes):
    """Keys and values that are not finite, near the ends of tiles, blocks and sequences: rows that do not see them keep their bits, and a value shows
    in its channel of the rows that see it, in no other."""
    dtype, d, seqs, Hq, Hkv, _ = PREFILL[kernel]
    base._say("not finite, every kernel", kernel, prefix, cap, slopes)
    q, k, v, sl, _ = base._prefill(seqs, Hq, Hkv, d, dtype, cap, slopes, False, prefix, seed=13)
    call = lambda kk, vv: strd.attn_prefill_varlen(base._dev(q), base._dev(kk), base._dev(vv), seqs, prefix=prefix, cap=cap, slopes=base._dev(sl)).cpu()
    first, sees, rows = call(k, v), _sees(seqs, prefix), q.shape[0]
    n, m = seqs[0][0], seqs[0][1]
    for at in sorted({0, 31, 63, 64, n - 1, n, n + m - 1, n + m, rows - 1} | ({127, 128, 255, 300} if n > 300 else set()) | ({511, 512, 1000} if n > 1000 else set())):
        for which, bad in (("k", float("nan")), ("k", float("inf")), ("v", float("nan")), ("v", -float("inf"))):
            kk, vv = k.clone(), v.clone()
            (kk if which == "k" else vv)[at, :, ::3] = bad
            o = call(kk, vv)
            hidden = torch.from_numpy(~sees[:, at])
            assert torch.equal(o[hidden], first[hidden]), (at, which, bad)
            if which == "v":
                assert not torch.isfinite(o[~hidden][:, :, ::3].float()).any(), (at, which, bad)
                assert torch.equal(o[~hidden][:, :, 1::3], first[~hidden][:, :, 1::3]), (at, which, bad)


# Caches long enough for workgroups that fill a CU (16 MB of keys and values: 13.4 million elements of a side in 4 bits, 4.2 million in bf16), not
# multiples of a trip: 4, 2 and 1 kv heads of a workgroup, one and two sets of query heads.
LONG = [(13141, 32, 8, 128, True), (13141, 64, 8, 128, True), (52453, 8, 2, 128, True), (52453, 12, 2, 128, True), (34977, 3, 3, 128, True), (34977, 21, 3, 128, True),
        (52453, 8, 4, 64, True), (52453, 40, 4, 64, True), (69931, 9, 3, 64, True), (4123, 32, 8, 128, False), (8231, 64, 4, 128, False), (10947, 6, 3, 128, False),
        (16423, 28, 4, 64, False), (65575, 16, 1, 64, False), (65575, 2, 1, 64, False)]


@pytest.mark.parametrize("T,Hq,Hkv,d,kv4", LONG)
def test_decode_steps_every_long_kernel(T, Hq, Hkv, d, kv4):
    """With a cap and a bias and with neither.  (More than 65536 tokens: two blocks of weights to a workgroup.)"""
    base._say("long decode", T, Hq, Hkv, d, kv4)
    q, k, v, sl, ps, w = base._decode_case(T, Hq, Hkv, d, BF16, kv4, True, True)
    kk, vv, part = np64(k), np64(v), np.zeros(1)
    if kv4:
        cache = base._cache(T + 3, Hkv, d, 0xFF)   # rows behind T hold NaN
        strd.kv4_store(base._dev(k), base._dev(v), cache, 0)
        held = [t[:T].cpu() for t in cache]
        (kk, _), (vv, part) = (tuple(x.astype(np.float64) for x in plain.kv4_values(a.numpy(), b.float().numpy())) for a, b in (held[:2], held[2:]))
    for cap, bias in ((30.0, True), (0.0, False)):
        more = dict(cap=cap, slopes=base._dev(sl) if bias else None, pos=base._dev(ps), weights=base._dev(w))
        o, got = strd.attn_decode_step_kv4(base._dev(q), cache, T, **more) if kv4 else strd.attn_decode_step_weights(base._dev(q), base._dev(k), base._dev(v), **more)
        want, ww, es, mag, ew = plain.decode(np64(q), kk, vv, cap, np64(sl) if bias else None, ps.numpy(), np64(w), vmag=np.abs(part) + np.abs(vv))
        # (a sum of T products goes through chains of a few hundred: of a wave's trips, the waves, the splits)
        base._within(o, want, base._out_bound(want, es, mag, BF16, 1024), "o")
        base._within(got, ww, ew + 512 * plain.U32 * np.abs(ww) + 1e-30, "weights")


# ------------------------------------------------------------------ values near the end of fp32's range --
@pytest.mark.parametrize("kernel", ["64 two groups", "128 two groups", "128 eight waves, prefix", "tiles", "tiles fp32"])
def test_prefill_varlen_values_up_to_the_size_that_the_header_names(kernel):
    dtype, d, seqs, Hq, Hkv, prefix = PREFILL[kernel]
    base._say("large values", kernel)
    q, k, v, _, _ = base._prefill(seqs, Hq, Hkv, d, dtype, 0.0, False, False, bool(prefix), seed=14, size=4.0)
    v = (v / v.abs().max() * (2.0 ** 111 / (seqs[0][0] + seqs[0][1]))).to(dtype)
    o = strd.attn_prefill_varlen(base._dev(q), base._dev(k), base._dev(v), seqs, prefix=bool(prefix))
    heads, kv = _heads(Hq, Hkv)
    want, es, mag = _plain_prefill(q, k, v, seqs, bool(prefix), 0.0, None, None, heads, kv)
    base._within(o[:, heads], want, base._out_bound(want, es, mag, dtype, seqs[0][0] + seqs[0][1]), "o")


@pytest.mark.parametrize("kv4", [True, False])
@pytest.mark.parametrize("d,dtype", [(64, BF16), (128, BF16), (96, BF16), (128, F32)])
def test_decode_values_up_to_the_size_that_the_header_names(d, dtype, kv4):
    base._say("large values", d, dtype, kv4)
    q, k, v, _, _, w = base._decode_case(500, 8, 2, d, dtype, kv4, False, False, size=4.0)
    v = (v / v.abs().max() * (2.0 ** 111 / 500)).to(dtype)
    base._decode_check(q, k, v, None, None, w, 0.0, kv4)


# ------------------------------------------------------------------ biases that favour what is far --
@pytest.mark.parametrize("kernel,prefix", _prefill_kernels())
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_prefill_varlen_steep_biases_towards_far_rows(kernel, prefix, cap):
    """A slope below 0 raises scores with the distance: of 1e3 and more a row the farthest row that is seen takes all, with a weight of 1."""
    dtype, d, seqs, Hq, Hkv, _ = PREFILL[kernel]
    base._say("towards far rows", kernel, prefix, cap)
    q, k, v, _, _ = base._prefill(seqs, Hq, Hkv, d, dtype, cap, False, False, prefix, seed=15)
    sl = torch.tensor([-1e3, -1e6, -1e12, -1e26])[torch.arange(Hq) % 4]
    o = strd.attn_prefill_varlen(base._dev(q), base._dev(k), base._dev(v), seqs, prefix=prefix, cap=cap, slopes=base._dev(sl)).cpu()
    sees, rows = _sees(seqs, prefix), q.shape[0]
    far = np.where(sees, np.abs(np.arange(rows)[:, None] - np.arange(rows)[None]), -1)
    one = torch.from_numpy((far == far.max(1, keepdims=True)).sum(1) == 1)   # (in the middle of a prefix there are two)
    want = v[torch.from_numpy(far.argmax(1))].repeat_interleave(Hq // Hkv, 1)
    assert torch.equal(o[one], want[one])
    assert torch.isfinite(o.float()).all()


@pytest.mark.parametrize("kv4", [True, False])
@pytest.mark.parametrize("d,dtype", [(64, BF16), (128, BF16), (96, BF16), (128, F32)])
def test_decode_steep_biases_either_way(d, dtype, kv4):
    """The newest row takes all, or the oldest."""
    base._say("steep decode", d, dtype, kv4)
    T, Hq, Hkv = 1500, 8, 2
    q, k, v, _, _, _ = base._decode_case(T, Hq, Hkv, d, dtype, kv4, False, False)
    v = v.float().mul(4).round().clamp(-8, 7).to(dtype)
    v[:, :, ::32], v[:, :, 1::32] = -8, 7        # step 1 in 4 bits, middle 0: values are held as they are
    sl = torch.tensor([-1e3, 1e3, -1e12, 1e12, -1e26, 1e26, 1e6, -1e6])
    c = base._cache(T, Hkv, d)
    strd.kv4_store(base._dev(k), base._dev(v), c, 0)
    o, w = strd.attn_decode_step_kv4(base._dev(q), c, T, slopes=base._dev(sl)) if kv4 else \
        strd.attn_decode_step_weights(base._dev(q), base._dev(k), base._dev(v), slopes=base._dev(sl))
    want = torch.stack([v[0 if sl[h] < 0 else T - 1, h // 4] for h in range(Hq)])
    assert torch.equal(o.cpu(), want)
    assert w[0] == 0.5 and w[T - 1] == 0.5 and (w[1:T - 1] == 0).all()
