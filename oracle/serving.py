"""Plain fp64 forms of what serves the rows that a reduced prefill keeps (include/strd.h): packed attention with capped and
biased scores, the 4-bit cache, the decode step that gathers weights, eviction.  numpy only; test infrastructure.

Attention comes with a bound of how far an implementation may be: `delta` bounds the error of a score (rounded products and
sums, the cap, the bias, the exponent's argument), which is the relative error of a probability before it is normalised."""
import numpy as np

U32 = 2.0 ** -24   # half a step of fp32, relative


def scores(q, k, scale, cap, slope, far):
    """x [R, T] of one head and delta [R, T]: q [R, d], k [T, d], far [R, T] distances or None."""
    d = q.shape[1]
    x = scale * (q @ k.T)
    delta = (d + 2) * U32 * scale * (np.abs(q) @ np.abs(k).T)
    if cap:
        x = cap * np.tanh(x / cap)
        delta = delta + 16 * U32 * cap   # an exponential form of tanh is off by some steps of 1, times the cap
    if slope is not None:
        x = x - slope * far
        delta = delta + 3 * U32 * np.abs(slope * far)
    return x, delta + 4 * U32 * (np.abs(x) + np.abs(x).max(initial=0.0))


def softmax(x, visible):
    x = np.where(visible, x, -np.inf)
    e = np.exp(x - x.max(axis=-1, keepdims=True))
    return e / e.sum(axis=-1, keepdims=True)


def attend(q, k, v, scale, cap, slope, far, visible, vmag=None):
    """o [R, d], p [R, T] and the parts of a bound: err_p [R, T] of p, the score's share of o's error, and sum p |v|."""
    x, delta = scores(q, k, scale, cap, slope, far)
    p = softmax(x, visible)
    err_p = p * (delta + (p * np.where(visible, delta, 0)).sum(-1, keepdims=True))
    vm = np.abs(v) if vmag is None else vmag
    return p @ v, p, err_p, err_p @ np.abs(v), p @ vm


def attn_varlen(q, k, v, seqs, prefix, cap, slopes, pos, scale=None):
    """o [rows, Hq, d], the scores' share of its error, sum p |v|.  seqs: (N, M, ...) per sequence."""
    rows, Hq, d = q.shape
    rep, scale = Hq // k.shape[1], d ** -0.5 if scale is None else scale
    o, es, mag = np.zeros((rows, Hq, d)), np.zeros((rows, Hq, d)), np.zeros((rows, Hq, d))
    r = 0
    for s in seqs:
        n, t = s[0], s[0] + s[1]
        at, i = slice(r, r + t), np.arange(t)
        if t:
            see = (i[None] <= i[:, None]) | (bool(prefix) & (i[None] < n) & (i[:, None] < n))
            ps = i.astype(float) if pos is None else pos[at].astype(float)
            far = np.abs(ps[:, None] - ps[None])
            for h in range(Hq):
                o[at, h], _, _, es[at, h], mag[at, h] = attend(q[at, h], k[at, h // rep], v[at, h // rep], scale, cap,
                                                               None if slopes is None else slopes[h], far, see)
        r += t
    return o, es, mag


def decode(q, k, v, cap, slopes, pos, w_in=None, scale=None, vmag=None):
    """o [Hq, d], w [T], the scores' share of o's error, sum p |v|, the bound of w's error."""
    Hq, d = q.shape
    T, rep, scale = k.shape[0], Hq // k.shape[1], d ** -0.5 if scale is None else scale
    ps = np.arange(T, dtype=float) if pos is None else pos[:T].astype(float)
    far, see = np.abs(ps[-1:, None] - ps[None]), np.ones((1, T), bool)
    o, es, mag, w, ew = np.zeros((Hq, d)), np.zeros((Hq, d)), np.zeros((Hq, d)), np.zeros(T), np.zeros(T)
    for h in range(Hq):
        g = h // rep
        o[h], p, ep, es[h], mag[h] = (a[0] for a in attend(q[h:h + 1], k[:, g], v[:, g], scale, cap, None if slopes is None else slopes[h],
                                                            far, see, None if vmag is None else vmag[:, g]))
        w, ew = w + p, ew + ep + (4 + Hq) * U32 * p
    w, ew = w / Hq, ew / Hq
    if w_in is not None:
        w, ew = w + w_in, ew + 2 * U32 * np.abs(w + w_in)
    return o, w, es, mag, ew


# ---- the 4-bit cache: the definition is in fp32 steps, so this is too -------------------------
def bf16(x):
    """fp32 numbers rounded to bf16 (nearest even), as fp32; NaN stays NaN."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(x), np.float32(np.nan), r)


def kv4_quantize(x):
    """codes uint8 [..., d/2], (s, z) fp32 [..., d/32, 2] of x [..., d]."""
    g = np.asarray(x, np.float32).reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    with np.errstate(all="ignore"):
        lo, hi = g.min(-1), g.max(-1)
        s = bf16((hi - lo) / np.float32(15))
        odd = ~np.isfinite(g).all(-1) | ~np.isfinite(s)
        s = np.where(s < np.float32(2.0 ** -100), np.float32(0), s)
        z = bf16(lo + np.float32(8) * s)
        odd |= ~np.isfinite(z)
        n = np.rint((g - z[..., None]) / np.where(s > 0, s, np.float32(1))[..., None])
        n = np.where(s[..., None] > 0, np.clip(n + 8, 0, 15), 8)
    n = np.where(odd[..., None], 0, n).astype(np.uint8)
    n = n.reshape(x.shape)
    meta = np.where(odd[..., None], np.float32(np.nan), np.stack([s, z], -1))
    return n[..., 0::2] | n[..., 1::2] << 4, meta.astype(np.float32)


def kv4_values(codes, meta):
    """fp32 values [..., d], and the part s (n - 8) of them."""
    n = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (2 * codes.shape[-1],)).astype(np.float32) - 8
    m = np.repeat(np.asarray(meta, np.float32), 32, axis=-2)
    part = m[..., 0] * n
    return m[..., 1] + part, part


def evict(w, K, first, last):
    """Kept rows, ascending; ties to the lowest row."""
    T = len(w)
    order = sorted(range(first, T - last), key=lambda i: (-w[i], i))
    return np.array(list(range(first)) + sorted(order[:K - first - last]) + list(range(T - last, T)), np.int64)
