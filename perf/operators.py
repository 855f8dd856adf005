"""What a program does with the rows that a reduced prefill keeps, as a list of cases with sizes.

*prefill*  causal attention over a packed batch of sequences, with a cap on the scores (tanh), a bias that falls with the
           distance of the tokens' positions, and vision rows that see all vision rows of their sequence (prefix).
*store*    key and value rows into the 4-bit cache and back out of it.
*decode*   the newest token's attention over a cache (4-bit or plain) with the same cap and bias, and the attention weight
           that every row has gathered so far.
*evict*    the cache cut down to K rows: the first ones, the last ones and the heaviest of the rest.

The 4-bit cache holds keys and values in groups of 32 channels of one (row, kv head): 32 codes n in 0..15, channel 2 i in the
low half of byte i, and two bf16 numbers, the step s and the value z of code 8; a code stands for z + s (n - 8).
Head layouts are those of the repository's workloads and tests.
"""
import math
import random

import numpy as np
import torch

own = False

GROUP = 32
TINY = 2.0 ** -100           # a step below this counts as 0
MOST_SCORES = 32 * 8320 * 8320   # scores of a prefill at most, masked ones counted
MOST_ROWS = 131072 + 512 + 43    # rows of a cache at most: the long video, its question and what was generated
MOST_STORED = 33280 * 8 * 128    # elements stored at most

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # three short clips with their questions in single precision: launches and host time count
        {"name": "prefill_clips_f32", "kind": "prefill", "dtype": "f32", "seqs": "512+32,64+3,1+1", "Hq": 4, "Hkv": 2, "d": 64,
         "cap": 30.0, "slopes": True, "prefix": True, "span": 1},
        # a server's batch of short clips of different lengths; the frames of a clip see each other
        {"name": "prefill_clips_6", "kind": "prefill", "dtype": "bf16", "seqs": "901+48,377+21,640+64,128+1,1207+33,55+18", "Hq": 28, "Hkv": 4,
         "d": 64, "cap": 0.0, "slopes": False, "prefix": True, "span": 1},
        # a quarter of 32 frames of 256 tokens, kept rows at their old positions
        {"name": "prefill_kept_2k", "kind": "prefill", "dtype": "bf16", "seqs": "2048+128", "Hq": 32, "Hkv": 8, "d": 128, "cap": 0.0,
         "slopes": True, "prefix": False, "span": 4},
        # 32 frames of 256 tokens, nothing dropped, capped scores
        {"name": "prefill_8k_capped", "kind": "prefill", "dtype": "bf16", "seqs": "8192+128", "Hq": 32, "Hkv": 8, "d": 128, "cap": 50.0,
         "slopes": False, "prefix": False, "span": 1},
        # the row of one generated token
        {"name": "store_token", "kind": "store", "dtype": "bf16", "rows": 1, "before": 843, "Hkv": 8, "d": 128},
        # the rows of a prefill of 128 frames of 256 tokens and its question, and back for the next part of the prompt
        {"name": "store_33k", "kind": "store", "dtype": "bf16", "rows": 33024, "before": 256, "Hkv": 8, "d": 128},
        # generation behind a short clip
        {"name": "decode_kv4_843", "kind": "decode", "cache": "kv4", "dtype": "bf16", "T": 843, "Hq": 32, "Hkv": 8, "d": 128, "cap": 0.0,
         "slopes": False, "span": 1},
        # generation behind a plain cache of a kept quarter, capped scores, 7 query heads to a key head
        {"name": "decode_plain_8k", "kind": "decode", "cache": "plain", "dtype": "bf16", "T": 8491, "Hq": 28, "Hkv": 4, "d": 64, "cap": 30.0,
         "slopes": False, "span": 4},
        # generation behind the whole long video
        {"name": "decode_kv4_131k", "kind": "decode", "cache": "kv4", "dtype": "bf16", "T": 131627, "Hq": 32, "Hkv": 8, "d": 128, "cap": 50.0,
         "slopes": True, "span": 1},
        # a small plain cache in single precision, half of it kept
        {"name": "evict_plain_f32", "kind": "evict", "cache": "plain", "dtype": "f32", "T": 1075, "K": 512, "first": 4, "last": 64, "Hkv": 2,
         "d": 64},
        # 32 frames of 256 tokens in 4 bits, a quarter kept
        {"name": "evict_kv4_8k", "kind": "evict", "cache": "kv4", "dtype": "bf16", "T": 8363, "K": 2176, "first": 4, "last": 128, "Hkv": 8,
         "d": 128},
        # the long video in 4 bits, a quarter kept
        {"name": "evict_kv4_131k", "kind": "evict", "cache": "kv4", "dtype": "bf16", "T": 131627, "K": 32896, "first": 4, "last": 512,
         "Hkv": 8, "d": 128},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("prefill", "store", "decode", "evict"))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    Hq, Hkv = rng.choice(((32, 8), (28, 4), (16, 2), (8, 8), (4, 2), (7, 1), (12, 4)))
    d = rng.choice((64, 128, 64, 128, 96))
    cap, slopes = rng.choice((0.0, 0.0, 30.0, 50.0)), rng.random() < 0.5
    if kind == "prefill":
        prefix = rng.random() < 0.5      # twice the visible pairs
        total = _log(rng, 16, min(8320 if dtype == "bf16" else 2361, math.isqrt(MOST_SCORES // Hq // (2 if prefix else 1))))
        parts, left = [], total
        while left > 0 and len(parts) < 16:
            n = left if rng.random() < 0.3 or len(parts) == 15 else rng.randint(1, left)
            m = rng.randint(0, max(0, n // 8))
            parts.append("%d+%d" % (n - m, m))
            left -= n
        return {"kind": kind, "dtype": dtype, "seqs": ",".join(parts), "Hq": Hq, "Hkv": Hkv, "d": d, "cap": cap, "slopes": slopes,
                "prefix": prefix, "span": rng.choice((1, 4))}
    if kind == "store":
        rows = _log(rng, 1, min(33024, MOST_STORED // (Hkv * d) // (2 if dtype == "f32" else 1)))
        return {"kind": kind, "dtype": dtype, "rows": rows, "before": rng.randint(0, 500), "Hkv": Hkv, "d": d}
    cache = "plain" if rng.random() < 0.3 else "kv4"
    most = MOST_ROWS * 8 * 128 // (Hkv * d) if cache == "kv4" else MOST_ROWS * 8 * 128 // (Hkv * d) // (7 if dtype == "f32" else 4)
    T = _log(rng, 1 if kind == "decode" else 8, min(MOST_ROWS, most))
    if kind == "decode":
        return {"kind": kind, "cache": cache, "dtype": dtype, "T": T, "Hq": Hq, "Hkv": Hkv, "d": d, "cap": cap, "slopes": slopes,
                "span": rng.choice((1, 4))}
    K = max(2, int(T * rng.uniform(0.15, 0.8)))
    K = min(K, 32896)
    first, last = rng.randint(0, min(4, K // 4)), rng.randint(0, min(512, K // 2))
    return {"kind": kind, "cache": cache, "dtype": dtype, "T": T, "K": K, "first": first, "last": last, "Hkv": Hkv, "d": d}


def _seqs(case):
    return [tuple(int(x) for x in part.split("+")) for part in case["seqs"].split(",")]


def _limits(case):
    """First visible row, and the row behind the last visible one, of every row."""
    start, stop, row = [], [], 0
    for n, m in _seqs(case):
        t = np.arange(n + m)
        start.append(np.full(n + m, row))
        stop.append(row + (np.where(t < n, n, t + 1) if case["prefix"] else t + 1))
        row += n + m
    return np.concatenate(start), np.concatenate(stop)


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "prefill":
        start, stop = _limits(case)
        return {"bytes": len(start) * case["d"] * (2 * case["Hq"] + 2 * case["Hkv"]) * es,
                "flops": 4.0 * case["d"] * case["Hq"] * float((stop - start).sum())}
    row = case["Hkv"] * case["d"]
    packed = 2 * row * (0.5 + 4 / GROUP)      # keys and values of a row in 4 bits
    if case["kind"] == "store":
        return {"bytes": case["rows"] * (2 * 2 * row * es + 2 * packed), "flops": case["rows"] * 2 * row * 8.0}
    kept = packed if case["cache"] == "kv4" else 2 * row * es
    if case["kind"] == "decode":
        return {"bytes": case["T"] * (kept + 8 + (4 if case["slopes"] else 0)) + 2 * case["Hq"] * case["d"] * es,
                "flops": 4.0 * case["T"] * case["Hq"] * case["d"]}
    values = 2 * row * es if case["cache"] == "kv4" else 0    # 4-bit rows come back as values, too
    return {"bytes": case["T"] * 4 + case["K"] * (2 * (kept + 8) + 4 + values), "flops": float(case["T"])}


# ---------------------------------------------------------------- inputs ------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) + 17)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _positions(g, T, span):
    """T ascending positions out of span * T: what a selection keeps."""
    if span == 1:
        return torch.arange(T, dtype=torch.int32, device="cuda")
    return torch.randperm(span * T, generator=g, device="cuda")[:T].sort().values.to(torch.int32)


def _slopes(Hq):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)], dtype=torch.float32, device="cuda")


def _rows(g, T, H, d, dt):
    """Keys or values of T rows: channels with means and sizes of their own, as projections have them."""
    size, mean = 0.5 + torch.rand((H, d), generator=g, device="cuda"), 0.5 * _randn(g, H, d)
    return (_randn(g, T, H, d) * size + mean).to(dt)


def _random_kv4(g, T, H, d):
    """A filled cache: uniform codes cover their range; steps and middles as rows of unit size give them."""
    codes = torch.randint(0, 256, (T, H, d // 2), generator=g, device="cuda", dtype=torch.uint8)
    step = 0.1 + 0.25 * torch.rand((T, H, d // GROUP), generator=g, device="cuda")
    return codes, torch.stack([step, 0.3 * _randn(g, T, H, d // GROUP)], dim=-1).to(torch.bfloat16)


def prepare(case, seed):
    g, dt, d = _gen(seed), DTYPES[case["dtype"]], case["d"]
    s = {"case": dict(case)}
    if case["kind"] == "prefill":
        Hq, Hkv = case["Hq"], case["Hkv"]
        start, stop = _limits(case)
        T = len(start)
        s["q"] = (1.5 * _randn(g, T, Hq, d)).to(dt)
        s["k"], s["v"] = _rows(g, T, Hkv, d, dt), _rows(g, T, Hkv, d, dt)
        s["slopes"] = _slopes(Hq) if case["slopes"] else None
        s["pos"] = torch.cat([_positions(g, n + m, case["span"]) for n, m in _seqs(case)]) if case["slopes"] else None
        s["seqs"] = [(n, m, n) for n, m in _seqs(case)]
        s["start"], s["stop"] = torch.from_numpy(start).cuda(), torch.from_numpy(stop).cuda()
    elif case["kind"] == "store":
        rows, H = case["rows"], case["Hkv"]
        s["k"], s["v"] = _rows(g, rows, H, d, dt), _rows(g, rows, H, d, dt)
        s["cache"] = tuple(x for _ in range(2) for x in _random_kv4(g, case["before"] + rows, H, d))
    elif case["kind"] == "decode":
        T, Hq, Hkv = case["T"], case["Hq"], case["Hkv"]
        s["q"] = (1.5 * _randn(g, Hq, d)).to(dt)
        if case["cache"] == "kv4":
            s["cache"] = tuple(x for _ in range(2) for x in _random_kv4(g, T, Hkv, d))
        else:
            s["cache"] = (_rows(g, T, Hkv, d, dt), _rows(g, T, Hkv, d, dt))
        s["slopes"] = _slopes(Hq) if case["slopes"] else None
        s["pos"] = _positions(g, T, case["span"]) if case["slopes"] else None
        s["weights"] = torch.rand(T, generator=g, device="cuda") * (64.0 / T)
        s["weights_out"] = torch.empty(T, device="cuda")
    else:
        T, K, Hkv = case["T"], case["K"], case["Hkv"]
        if case["cache"] == "kv4":
            s["cache"] = tuple(x for _ in range(2) for x in _random_kv4(g, T, Hkv, d))
        else:
            s["cache"] = (_rows(g, T, Hkv, d, dt), _rows(g, T, Hkv, d, dt))
        w = torch.exp(2.0 * _randn(g, T)) / T
        s["weights"] = torch.where(torch.rand(T, generator=g, device="cuda") < 0.03, 0.0, w)  # rows that no one looked at
        s["pos"] = _positions(g, T, 4)
    return s


# ---------------------------------------------------------------- plain forms -------------------------------
def _unpack(codes, meta):
    """fp32 [T, H, d] of 4-bit rows."""
    n = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).float()
    m = meta.float().repeat_interleave(GROUP, dim=-2)
    return m[..., 1] + m[..., 0] * (n - 8.0)


def _quantize(x):
    """The values that rows stand for in 4 bits, fp32."""
    g = x.float().unflatten(-1, (-1, GROUP))
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    s = ((hi - lo) / 15.0).to(torch.bfloat16).float()
    s = torch.where(s < TINY, 0.0, s)
    z = (lo + 8.0 * s).to(torch.bfloat16).float()
    n = torch.clamp(torch.round((g - z) / torch.where(s > 0, s, 1.0)) + 8.0, 0.0, 15.0)
    return (z + s * (n - 8.0)).flatten(-2)


def _capped(x, cap):
    return cap * torch.tanh(x / cap) if cap else x


def _plain_prefill(s):
    c, T = s["case"], s["q"].shape[0]
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    q = s["q"].float().view(T, Hkv, Hq // Hkv, d).permute(1, 2, 0, 3).reshape(Hkv, -1, d)
    k = s["k"].float().permute(1, 2, 0).contiguous()
    x = _capped(torch.matmul(q, k) * d ** -0.5, c["cap"]).view(Hq, T, T)
    if s["slopes"] is not None:
        p = s["pos"].float()
        x = x - s["slopes"].view(-1, 1, 1) * (p[:, None] - p[None, :]).abs()
    j = torch.arange(T, device=x.device)
    x = x.masked_fill((j < s["start"][:, None]) | (j >= s["stop"][:, None]), -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True))
    x = x / x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(Hkv, -1, T), s["v"].float().permute(1, 0, 2).contiguous())
    return o.view(Hq, T, d).permute(1, 0, 2).contiguous().to(s["q"].dtype)


def _plain_decode(s):
    c = s["case"]
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    ch = s["cache"]
    k, v = (_unpack(*ch[:2]), _unpack(*ch[2:])) if c["cache"] == "kv4" else (ch[0].float(), ch[1].float())
    q = s["q"].float().view(Hkv, Hq // Hkv, d)
    x = _capped(torch.matmul(q, k.permute(1, 2, 0).contiguous()) * d ** -0.5, c["cap"])
    if s["slopes"] is not None:
        p = s["pos"].float()
        x = x - s["slopes"].view(Hkv, -1, 1) * (p[-1] - p).abs()
    x = torch.exp(x - x.amax(-1, keepdim=True))
    x = x / x.sum(-1, keepdim=True)
    o = torch.matmul(x, v.permute(1, 0, 2).contiguous())
    return o.view(Hq, d).to(s["q"].dtype), s["weights"] + x.view(Hq, -1).mean(0)


def _plain_evict(s):
    c = s["case"]
    T, K, first, last = c["T"], c["K"], c["first"], c["last"]
    w = s["weights"]
    best = torch.sort(w[first:T - last], descending=True, stable=True).indices[:K - first - last] + first
    rows = torch.arange(T, device=w.device)
    idx = torch.cat([rows[:first], best.sort().values, rows[T - last:]])
    return [idx.to(torch.int32), w[idx], s["pos"][idx]] + [t[idx] for t in s["cache"]]


def run(state):
    c = state["case"]
    if own:
        return _run_own(state, c)
    if c["kind"] == "prefill":
        return _plain_prefill(state)
    if c["kind"] == "store":
        return [_quantize(state["k"]).to(state["k"].dtype), _quantize(state["v"]).to(state["v"].dtype)]
    return list(_plain_decode(state)) if c["kind"] == "decode" else _values(c, _plain_evict(state))


def _values(c, out):
    """What a cut-down cache stands for: 4-bit rows as values, plain rows as they are."""
    if c["cache"] == "kv4":
        return out[:3] + [_unpack(*out[3:5]).to(DTYPES[c["dtype"]]), _unpack(*out[5:7]).to(DTYPES[c["dtype"]])]
    return out


def _run_own(s, c):
    import paper_2603_00198_amd as strd
    if c["kind"] == "prefill":
        return strd.attn_prefill_varlen(s["q"], s["k"], s["v"], s["seqs"], prefix=c["prefix"], cap=c["cap"], slopes=s["slopes"], pos=s["pos"])
    if c["kind"] == "store":
        cache = strd.Kv4Cache(*s["cache"])
        strd.kv4_store(s["k"], s["v"], cache, c["before"])
        return list(strd.kv4_load(cache, c["before"], c["rows"], dtype=s["k"].dtype))
    if c["kind"] == "decode":
        more = dict(cap=c["cap"], slopes=s["slopes"], pos=s["pos"], weights=s["weights"], weights_out=s["weights_out"])
        if c["cache"] == "kv4":
            return list(strd.attn_decode_step_kv4(s["q"], strd.Kv4Cache(*s["cache"]), c["T"], **more))
        return list(strd.attn_decode_step_weights(s["q"], *s["cache"], **more))
    idx, w, rows, pos = strd.cache_evict(s["weights"], c["K"], c["first"], c["last"], s["cache"], pos=s["pos"])
    if c["cache"] == "kv4":
        rows = list(strd.kv4_load(strd.Kv4Cache(*rows), 0, c["K"], dtype=DTYPES[c["dtype"]]))
    return [idx, w, pos] + list(rows)


# ---------------------------------------------------------------- the definitions in 64 bits ----------------
def _exact_rows(codes, meta):
    low, high = (codes % 16).double(), torch.div(codes, 16, rounding_mode="floor").double()
    T, H, half = codes.shape
    n = torch.empty((T, H, 2 * half), dtype=torch.float64, device=codes.device)
    n[..., 0::2], n[..., 1::2] = low, high
    out = torch.empty_like(n)
    for g in range(meta.shape[2]):
        at = slice(GROUP * g, GROUP * (g + 1))
        out[..., at] = meta[:, :, g, 1:].double() + meta[:, :, g, :1].double() * (n[..., at] - 8)
    return out


def _exact_softmax(x):
    top = x.max(dim=-1, keepdim=True).values
    return torch.exp(x - top - torch.log(torch.exp(x - top).sum(dim=-1, keepdim=True)))


def _exact_scores(x, case, slope, far):
    if case["cap"]:
        e = torch.exp(-2.0 * x.abs() / case["cap"])
        x = torch.sign(x) * case["cap"] * (1.0 - e) / (1.0 + e)
    return x if slope is None else x - slope.double() * far


def exact(case, seed):
    s = prepare(case, seed)
    d = case["d"]
    if case["kind"] == "prefill":
        out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        row = 0
        for n, m in _seqs(case):   # one sequence and one head at a time
            T = n + m
            at = slice(row, row + T)
            t = torch.arange(T, device="cuda")
            hidden = t[None, :] > t[:, None]
            if case["prefix"]:
                hidden &= ~((t[None, :] < n) & (t[:, None] < n))
            far = (s["pos"][at].double()[:, None] - s["pos"][at].double()[None, :]).abs() if s["pos"] is not None else None
            for h in range(case["Hq"]):
                kv = h // (case["Hq"] // case["Hkv"])
                x = s["q"][at, h].double() @ s["k"][at, kv].double().t().contiguous() / math.sqrt(d)
                x = _exact_scores(x, case, s["slopes"][h] if s["slopes"] is not None else None, far)
                x[hidden] = -math.inf
                out[at, h] = _exact_softmax(x) @ s["v"][at, kv].double()
            row += T
        return out
    if case["kind"] == "store":
        both = []
        for x in (s["k"], s["v"]):   # the step and the middle are bf16 numbers by definition, the codes integers
            y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
            for g in range(d // GROUP):
                at = slice(GROUP * g, GROUP * (g + 1))
                v = x[..., at].double()
                low, high = v.min(dim=-1, keepdim=True).values, v.max(dim=-1, keepdim=True).values
                step = ((high - low) / 15).float().to(torch.bfloat16).double()
                mid = (low + 8 * step).float().to(torch.bfloat16).double()
                code = torch.round((v - mid) / step).clamp(-8, 7)
                y[..., at] = torch.where(step < TINY, mid, mid + step * code)
            both.append(y)
        return both
    if case["kind"] == "decode":
        if case["cache"] == "kv4":
            k, v = _exact_rows(*s["cache"][:2]), _exact_rows(*s["cache"][2:])
        else:
            k, v = s["cache"][0].double(), s["cache"][1].double()
        far = (s["pos"][-1].double() - s["pos"].double()).abs() if s["pos"] is not None else None
        o = torch.empty((case["Hq"], d), dtype=torch.float64, device="cuda")
        w = torch.zeros(case["T"], dtype=torch.float64, device="cuda")
        for h in range(case["Hq"]):
            kv = h // (case["Hq"] // case["Hkv"])
            x = (k[:, kv] * s["q"][h].double()).sum(-1) / math.sqrt(d)
            p = _exact_softmax(_exact_scores(x, case, s["slopes"][h] if s["slopes"] is not None else None, far))
            o[h] = (p[:, None] * v[:, kv]).sum(0)
            w += p
        return [o, s["weights"].double() + w / case["Hq"]]
    w = s["weights"].cpu().numpy()
    T, K, first, last = case["T"], case["K"], case["first"], case["last"]
    middle = sorted(range(first, T - last), key=lambda i: (-w[i], i))[:K - first - last]
    idx = torch.tensor(list(range(first)) + sorted(middle) + list(range(T - last, T)), device="cuda")
    out = [idx.to(torch.int32), s["weights"][idx].double(), s["pos"][idx]]
    if case["cache"] == "kv4":
        return out + [_exact_rows(s["cache"][0][idx], s["cache"][1][idx]), _exact_rows(s["cache"][2][idx], s["cache"][3][idx])]
    return out + [t[idx].double() for t in s["cache"]]
