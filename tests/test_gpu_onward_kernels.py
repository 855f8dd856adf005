"""The kernels that the calls behind a prompt choose among for long sequences and large batches, each at sizes that reach it, against plain fp64 forms
(bounds: test_gpu_onward.py, test_gpu_onward_edges.py).  onward_plans.py says what reaches what."""
import ctypes

import numpy as np
import pytest
import torch

import onward_plans as plans
import paper_2603_00198_amd as strd
import test_gpu_onward as base
import test_gpu_onward_edges as edges
from oracle import serving
from paper_2603_00198_amd import binding
from paper_2603_00198_amd.synth import np64

pytestmark = pytest.mark.gpu
DEV, BF16, F32 = "cuda", torch.bfloat16, torch.float32


# ------------------------------------------------------------------ packed scans -----------
def _scan_bytes(lens, H, P, G, n, dtype):
    seqs = (binding._Seq * len(lens))(*[binding._Seq(t, 0, 0) for t in lens])
    return binding.lib().strd_ssd_prefill_varlen_workspace(ctypes.cast(seqs, ctypes.c_void_p), len(lens), H, P, G, n, 1 if dtype == BF16 else 0)


def _long_scan(lens, H, P, G, n, dtype, style):
    """Inputs made on the GPU.  style: how heads forget, within a step (32 tokens), over some, over hundreds, or four side by side each in its own way."""
    g = torch.Generator(device=DEV).manual_seed(len(lens) + n)
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV)
    T = sum(lens)
    x, B, C = rnd(T, H, P).to(dtype), rnd(T, G, n).to(dtype), rnd(T, G, n).to(dtype)
    dt = torch.nn.functional.softplus(rnd(T, H))
    A = -torch.exp(2.0 * torch.rand(H, generator=g, device=DEV))
    k = torch.arange(H, device=DEV) % 4
    A = A * {"forget": torch.ones_like(A), "some": torch.full_like(A, 0.1), "remember": torch.full_like(A, 0.003),
             "mixed": torch.where(k == 0, 0.003, torch.where(k == 1, 0.05, 1.0))}[style]
    return x, dt, A, B, C, rnd(H)


# lens, H, G, n, styles, and the parts of a full and of the last segment of each sequence
PARTS = {
    "two": ([9000, 300], 128, 8, 64, [2, 1], [2, 1]),
    "three": ([12000, 5000], 128, 8, 64, [3, 3], [2, 1]),
    "six": ([24000, 8256, 1024], 128, 8, 128, [6, 6, 2], [5, 6, 2]),
    "few heads": ([33280], 24, 3, 128, [2], [2]),
    "few heads, short end": ([30000], 32, 2, 64, [2], [1]),
}


@pytest.mark.parametrize("name,style", [(k, s) for k in PARTS for s in ("forget", "some", "remember", "mixed") if k in ("two", "three") or s == "mixed"])
def test_scan_of_segments_in_parts(name, style):
    """What parts of segments leave behind them, several of them alive or all but the last gone, and a last segment that has fewer."""
    lens, H, G, n, per, last = PARTS[name]
    base._say("scan parts", name, style)
    plan = plans.scan_plan(lens, H, n)
    assert not plans.chunks_wanted(lens, H, n) and plan["parts"] == per and plan["last_parts"] == last
    assert plan["bytes"] == _scan_bytes(lens, H, 64, G, n, BF16)
    x, dt, A, B, C, D = _long_scan(lens, H, 64, G, n, BF16, style)
    pool = torch.randn((len(lens) + 1, H, 64, n), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)
    slots, fresh, state = list(range(len(lens), 0, -1)), [i == 1 for i in range(len(lens))], pool.clone()
    y = strd.ssd_prefill_varlen(x, dt, A, B, C, [(t, 0, 0) for t in lens], D, state=state, slots=slots, fresh=fresh)
    assert torch.equal(state[0], pool[0]) and torch.isfinite(y).all() and torch.isfinite(state).all()
    some = sorted(set([0, 1, 2, 3, H - 1] + list(range(5, H, 17))))
    edges._check_fine([(t, 0, 0) for t in lens], x, dt, A, B, C, D, pool, slots, fresh, y, state, 1 if style in ("remember", "mixed") else 2, some,
                      [0, 3, 4, 21, 42, 63])


@pytest.mark.parametrize("lens,H,G,n", [([9000, 300], 128, 8, 64), ([20000, 700], 64, 4, 128)])
@pytest.mark.parametrize("style", ["forget", "mixed"])
def test_scan_of_segments_in_parts_keeps_what_is_not_finite(lens, H, G, n, style):
    """... in every later output of its channel and in its final state, also where what a part leaves behind it is not worked out; in no other."""
    base._say("scan parts not finite", lens, H, G, n, style)
    plan = plans.scan_plan(lens, H, n)
    assert plan["segments"][0] > 3 and plan["parts"][0] > 1
    x, dt, A, B, C, D = _long_scan(lens, H, 64, G, n, BF16, style)
    seqs, pool = [(t, 0, 0) for t in lens], torch.zeros((len(lens), H, 64, n), device=DEV)
    want_S, state = pool.clone(), pool.clone()
    want = strd.ssd_prefill_varlen(x, dt, A, B, C, seqs, D, state=want_S)
    odd = [(100, 5, 37, float("nan")), (lens[0] // 2, H - 2, 2, float("inf")), (lens[0] + 200, 6, 63, float("-inf"))]
    touched, reached = torch.zeros(want.shape, dtype=torch.bool, device=DEV), torch.zeros(pool.shape, dtype=torch.bool, device=DEV)
    for t, h, p, value in odd:
        x[t, h, p] = value
    y = strd.ssd_prefill_varlen(x, dt, A, B, C, seqs, D, state=state)
    for t, h, p, value in odd:
        s = int(t >= lens[0])
        end = lens[0] + s * lens[1]
        assert not torch.isfinite(y[t:end, h, p]).any() and not torch.isfinite(state[s, h, p]).any()
        touched[max(t - 63, s * lens[0]):end, h, p] = True
        reached[s, h, p] = True
    assert (y == want)[~touched].all() and (state == want_S)[~reached].all()


@pytest.mark.parametrize("seed", range(12))
def test_random_long_scan(seed):
    rng = np.random.default_rng(700 + seed)
    H, G, n = [(128, 8, 64), (64, 4, 128), (24, 3, 128), (96, 8, 64), (32, 8, 128), (16, 2, 64)][seed % 6]
    left, lens = int(2 ** rng.uniform(12, 14.5)), []
    while left > 0 and len(lens) < 9:
        lens.append(left if rng.random() < 0.4 or len(lens) == 8 else int(rng.integers(0, left + 1)))
        left -= lens[-1]
    style, fresh = str(rng.choice(["forget", "some", "remember", "mixed"])), [bool(rng.random() < 0.3) for _ in lens]
    plan = plans.scan_plan(lens, H, n)
    base._say("random long scan", seed, lens, H, G, n, style, plan["parts"], plan["segments"])
    assert not plans.chunks_wanted(lens, H, n) and plan["bytes"] == _scan_bytes(lens, H, 64, G, n, BF16)
    x, dt, A, B, C, D = _long_scan(lens, H, 64, G, n, BF16, style)
    pool = torch.randn((len(lens) + 2, H, 64, n), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)
    slots, out = rng.permutation(len(lens) + 2)[:len(lens)].tolist(), torch.full_like(pool, 7.0)
    y = strd.ssd_prefill_varlen(x, dt, A, B, C, [(t, 0, 0) for t in lens], D, state=pool, state_out=out, slots=slots, fresh=fresh)
    some = sorted(set(int(h) for h in rng.integers(0, H, 6)))
    edges._check_fine([(t, 0, 0) for t in lens], x, dt, A, B, C, D, pool, slots, fresh, y, out, 1 if style in ("remember", "mixed") else 2, some,
                      sorted(set(int(p) for p in rng.integers(0, 64, 6))))


@pytest.mark.parametrize("lens,H,G,n", [([949, 398, 704, 129, 1240, 73], 128, 8, 128), ([1200, 395, 40], 64, 4, 64), ([2000, 31], 32, 2, 128)])
@pytest.mark.parametrize("style", ["forget", "mixed"])
def test_scan_final_states_are_fp32_sums(lens, H, G, n, style):
    """On the matrix cores: bounds that a term of a state rounded to bf16, once, does not keep."""
    base._say("scan states", lens, H, G, n, style)
    assert not plans.chunks_wanted(lens, H, n) and plans.scan_plan(lens, H, n)["bytes"] == _scan_bytes(lens, H, 64, G, n, BF16)
    x, dt, A, B, C, D = _long_scan(lens, H, 64, G, n, BF16, style)
    state, seqs = torch.zeros((len(lens), H, 64, n), device=DEV), [(t, 0, 0) for t in lens]
    y = strd.ssd_prefill_varlen(x, dt, A, B, C, seqs, D, state_out=state)
    some, chans = sorted(set([0, 1, 2, 3, H - 1] + list(range(5, H, 17)))), list(range(0, 64, 5))
    edges._check_fine(seqs, x, dt, A, B, C, D, None, list(range(len(lens))), None, y, state, 1 if style == "mixed" else 2, some, chans)
    if style == "forget":   # the bound's own test: an oracle that rounds what a sequence's last token brings to bf16 is outside it
        x64, ends = x.double().cpu(), np.cumsum(lens) - 1
        last = dt[ends].double().cpu()[..., None]
        x64[ends] = (last * x64[ends]).to(BF16).double() / last
        with pytest.raises(AssertionError, match="state of"):
            edges._check_fine(seqs, x64, dt, A, B, C, D, None, list(range(len(lens))), None, y, state, 2, some, chans)


@pytest.mark.parametrize("lens,H,P,G,n", [([57], 64, 64, 4, 64), ([500, 40, 1], 16, 64, 2, 128), ([3000, 200], 8, 64, 8, 64), ([2500], 8, 32, 1, 16), ([900, 70], 6, 40, 2, 24)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("style", ["forget", "mixed"])
def test_scan_in_chunks_rounds_an_output_once(lens, H, P, G, n, dtype, style):
    """Small batches and other shapes: products and sums in fp32 whatever the inputs are, and one rounding to their type."""
    base._say("scan chunks", lens, H, P, G, n, dtype, style)
    assert P != 64 or H // G % 4 or plans.chunks_wanted(lens, H, n)
    x, dt, A, B, C, D = _long_scan(lens, H, P, G, n, dtype, style)
    state, seqs = torch.randn((len(lens), H, P, n), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV), [(t, 0, 0) for t in lens]
    pool = state.clone()
    y = strd.ssd_prefill_varlen(x, dt, A, B, C, seqs, D, state=state)
    edges._check_fine(seqs, x, dt, A, B, C, D, pool, list(range(len(lens))), None, y, state, 0, None, list(range(0, P, 5)), pieces=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("batch,H,n,in_place,listed", [(18, 128, 128, True, True), (18, 128, 128, False, True), (36, 128, 64, True, False)])
def test_scan_steps_past_the_caches(batch, H, n, in_place, listed, dtype):
    assert batch * H * 64 * n * 4 > 64 << 20
    base.test_scan_steps(batch, H, 64, 8, n, in_place, listed, dtype)


# ------------------------------------------------------------------ convolution ------------
@pytest.mark.parametrize("dtype,Cx,Cb,W,pad", [(BF16, 2048, 128, 4, 8), (BF16, 2048, 128, 2, 0), (F32, 1024, 64, 4, 4), (F32, 1024, 64, 3, 0), (BF16, 515, 65, 4, 1), (F32, 515, 65, 3, 2)])
@pytest.mark.parametrize("carry", ["all", "some", "in_place"])
def test_conv_varlen_of_many_rows(dtype, Cx, Cb, W, pad, carry, monkeypatch):
    """Eight tokens a thread, windows and ends of sequences among them."""
    seqs = [(3000, 101, 0), (2, 0, 0), (0, 0, 0), (1700, 9, 0), (0, 7, 0), (1207, 0, 0), (8, 0, 0)]
    vec = pad % 4 == 0 and Cx % 8 == 0
    assert plans.conv_tokens([s[0] + s[1] for s in seqs], Cx + 2 * Cb, (8 if dtype == BF16 else 4) if vec else 1) == 8
    monkeypatch.setitem(base.SEQS, "many", seqs)
    base.test_conv_varlen("many", Cx, Cb, W, pad, carry, dtype)


# ------------------------------------------------------------------ drafted trees ----------
# T, m, Hq, Hkv, d: computing waves, keys of a chunk, chunks of a split at least, waves of the join
LONG = {
    (20003, 40, 8, 1, 64): (8, 128, 2, 16),
    (20000, 33, 32, 8, 128): (8, 128, 5, 4),
    (20017, 40, 16, 4, 96): (8, 128, 3, 8),
    (20003, 20, 32, 8, 128): (4, 64, 5, 8),
    (9999, 20, 32, 8, 96): (4, 64, 3, 8),
    (20003, 12, 32, 8, 64): (2, 64, 5, 8),
    (30001, 8, 32, 8, 96): (1, 64, 7, 8),
    (30001, 3, 32, 8, 128): (1, 64, 7, 8),
    (10001, 3, 8, 2, 128): (1, 32, 2, 16),
    (10001, 9, 8, 2, 64): (2, 32, 2, 16),
    (8001, 20, 8, 2, 64): (4, 32, 2, 16),
}


def _tree_oracle(q, k, v, T, mask, cap, slopes, pos):
    m, Hq, d = q.shape
    rep = Hq // k.shape[1]
    sees = np.ones((m, T + m), bool)
    for i in range(m):
        sees[i, T:] = [int(mask[i]) >> j & 1 for j in range(m)]
    if pos is None:
        pos = np.concatenate([np.arange(T), [T + bin(int(x) & ~(1 << i)).count("1") for i, x in enumerate(mask)]])
    far = np.abs(pos.astype(float)[T:, None] - pos.astype(float)[None])
    o, es, mag = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape)
    for h in range(Hq):
        o[:, h], _, _, es[:, h], mag[:, h] = serving.attend(q[:, h], k[:, h // rep], v[:, h // rep], d ** -0.5, cap, None if slopes is None else slopes[h], far, sees)
    return o, es, mag


def _long_tree(T, m, Hq, Hkv, d, dtype, cap, slopes, pos):
    q, k, v, mask = base._tree_case(T, m, Hq, Hkv, d, dtype, seed=T)
    hidden = m // 2   # a node that nobody sees, itself included, holds what is not finite
    mask &= ~(1 << hidden)
    ps = torch.randperm(2 * (T + m), generator=torch.Generator().manual_seed(T))[:T + m].to(torch.int32) if pos else None
    sl = base._slopes(Hq) if slopes else None
    want, es, mag = _tree_oracle(np64(q), np64(k), np64(v), T, [int(x) & (2 ** 64 - 1) for x in mask], cap, None if sl is None else np64(sl), None if ps is None else ps.numpy())
    k[T + hidden], v[T + hidden, :, ::2], v[T + hidden, :, 1::2] = float("nan"), float("inf"), float("nan")
    o = strd.attn_tree_step(*(base._dev(t) for t in (q, k[:T], v[:T], k[T:], v[T:], mask)), cap=cap, slopes=base._dev(sl), pos=base._dev(ps))
    base._within(o, want, base._tree_bound(want, es, mag, dtype, T + m), "o")


@pytest.mark.parametrize("T,m,Hq,Hkv,d", list(LONG))
@pytest.mark.parametrize("cap,slopes,pos", [(0.0, False, False), (0.0, True, False), (30.0, False, False), (5.0, True, True)])
def test_tree_over_long_caches(T, m, Hq, Hkv, d, cap, slopes, pos):
    """Several chunks of keys in a split, so that its buffers come round, and many splits to join."""
    base._say("long tree", T, m, Hq, Hkv, d, cap, slopes, pos)
    plan = plans.tree_plan(T, m, Hq, Hkv, d)
    assert (plan["nw"], plan["keys"], plans.waves_of_the_join(plan["splits"])) == LONG[T, m, Hq, Hkv, d][:2] + LONG[T, m, Hq, Hkv, d][3:]
    assert plan["per"] * 32 > (LONG[T, m, Hq, Hkv, d][2] - 1) * plan["keys"]
    assert plan["bytes"] == binding.lib().strd_attn_tree_step_workspace(T, m, Hq, Hkv, d, 1)
    _long_tree(T, m, Hq, Hkv, d, BF16, cap, slopes, pos)


@pytest.mark.parametrize("dtype,T,m,Hq,Hkv,d,join", [(F32, 9001, 20, 8, 2, 64, 16), (F32, 3001, 33, 8, 2, 128, 8), (F32, 12001, 5, 4, 1, 96, 16), (BF16, 12001, 20, 4, 2, 40, 16),
                                                     (BF16, 5001, 7, 4, 2, 200, 8), (BF16, 9001, 7, 4, 2, 33, 4), (F32, 9001, 9, 6, 2, 250, 4)])
@pytest.mark.parametrize("cap,slopes,pos", [(0.0, False, False), (5.0, True, True)])
def test_tree_over_long_caches_of_other_shapes(dtype, T, m, Hq, Hkv, d, join, cap, slopes, pos):
    base._say("long tree, general", dtype, T, m, Hq, Hkv, d, cap, slopes, pos)
    plan = plans.tree_plan(T, m, Hq, Hkv, d)
    assert d % 4 or plans.waves_of_the_join(plan["general"]) == join
    assert plan["bytes"] == binding.lib().strd_attn_tree_step_workspace(T, m, Hq, Hkv, d, 1) or dtype == F32
    _long_tree(T, m, Hq, Hkv, d, dtype, cap, slopes, pos)


@pytest.mark.parametrize("seed", range(12))
def test_random_tree_over_a_long_cache(seed):
    rng = np.random.default_rng(900 + seed)
    Hkv = int(rng.choice([1, 2, 4, 8]))
    Hq, d, m = Hkv * int(rng.integers(1, 9)), int(rng.choice([64, 96, 128])), int(rng.integers(1, 65))
    T, dtype = int(2 ** rng.uniform(11, 15)), F32 if seed % 4 == 3 else BF16
    cap, slopes, pos = float(rng.choice([0.0, 1.0, 30.0, 50.0])), bool(rng.random() < 0.5), bool(rng.random() < 0.5)
    if dtype == F32:
        T //= 4
    base._say("random long tree", seed, T, m, Hq, Hkv, d, dtype, cap, slopes, pos, plans.tree_plan(T, m, Hq, Hkv, d))
    _long_tree(T, m, Hq, Hkv, d, dtype, cap, slopes, pos)
