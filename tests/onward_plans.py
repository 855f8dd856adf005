"""How the calls behind a prompt cut their work (ssd_packed_mfma.hip, attn_tree.hip, attn_tree_mfma.hip, conv_carry.hip), worked out again: tests that are
meant for one of their kernels ask here whether their sizes still reach it, and compare the workspace, whose size follows from the same numbers."""


def _up(v, to=256):
    return -(-v // to) * to


def ceil(a, b):
    return -(-a // b)


# ------------------------------------------------------------------ packed scans -----------
def chunks_wanted(lens, H, n):
    """Whether a batch that the matrix cores could take runs in fp32 chunks."""
    return sum(ceil(t, 64) for t in lens) * 64 * H * n <= 5 << 20


def scan_plan(lens, H, n):
    """Steps of a full segment and of its parts, segments and parts per sequence (a full segment's; the last one's own), bytes of the workspace."""
    wg, steps = H // 4, [ceil(t, 32) for t in lens]
    longest, best, take = max([1] + steps), 0.0, 0

    def look_at(length):
        nonlocal best, take
        length = min(max(length, 8), longest)
        fulls, multi, rest = 0, 0, []
        for k in steps:
            fulls += k // length
            if k % length:
                rest.append(k % length)
            if k > length:
                multi += ceil(k, length)
        rest.sort(reverse=True)
        worst = 0.0
        for x in range(8):
            total, first = float(fulls // 8 * (length + 3)), float(length + 3 if fulls >= 8 else 0)
            r = fulls // 8
            while r * 8 < fulls + len(rest):
                rank = r * 8 + (7 - x if r & 1 else x)
                r += 1
                if rank >= fulls + len(rest):
                    continue
                here = float((length if rank < fulls else rest[rank - fulls]) + 3)
                total, first = total + here, max(first, here)
            worst = max(worst, first, total * wg / 32)
        est = worst + (4 + multi * wg * (9.0 / 256) * n / 128 if multi else 0)
        if not take or est < best:
            best, take = est, length

    look_at(longest)
    for rounds in range(1, 5):
        places = rounds * 8 * max(1, 32 // wg)
        look_at(ceil(sum(steps), places))
        lo, hi = 1, longest
        while lo < hi:
            mid = (lo + hi) // 2
            if sum(ceil(k, mid) for k in steps) <= places:
                hi = mid
            else:
                lo = mid + 1
        look_at(lo)
    part = 24
    while part < 64 and sum(steps) // part > 80:
        part = min(2 * part, 64)
    part = ceil(take, ceil(take, part))
    seq_steps = [min(k, take) for k in steps]
    nseg = [ceil(k, take) if k else 0 for k in steps]
    segs, multi = sum(nseg), sum(s for s in nseg if s > 1)
    per = [ceil(k, part) for k in seq_steps]
    parts, state = sum(s * p for s, p in zip(nseg, per)), H * 64 * n * 4
    last = [ceil(k - (s - 1) * q, part) if s else 0 for k, s, q in zip(steps, nseg, seq_steps)]
    return {"take": take, "part": part, "segments": nseg, "parts": per, "last_parts": last,
            "bytes": (multi + parts) * state + _up(parts * wg * 4) + _up(segs * H * 4) + _up(segs * H * 8) + _up(sum(steps) * H * 4) + sum(steps) * H * 128}


# ------------------------------------------------------------------ drafted trees ----------
def tree_plan(T, m, Hq, Hkv, d):
    """Computing waves, keys of a chunk, blocks of 32 keys per split, splits on the matrix cores; splits of the general kernel; bytes of the workspace that
    has room for either."""
    R, blocks = m * (Hq // Hkv), ceil(T + m, 32)
    nw, per_cu = (8, 1) if R > 128 else (4, 2) if R > 64 else (2, 2) if R > 32 else (1, 2)
    want = max(1, 256 * per_cu // (ceil(R, 32 * nw) * Hkv))
    per = max(ceil(blocks, want), min(2, blocks))
    if ceil(blocks, per) * m * Hq * d * 4 > 8 << 20:
        per = max(per, 6)
    splits = ceil(blocks, per)
    wgs = Hkv * ceil(R, 16 * min(4, ceil(R, 16)))
    rows = max(32, ceil(ceil(max(T, 1), max(1, min(ceil(1024, wgs), T // 64))), 32) * 32)
    general = ceil(T, rows) + 1
    return {"nw": nw, "keys": 128 if nw == 8 else 32 if per <= 2 else 64, "per": per, "splits": splits, "general": general,
            "bytes": max(splits if d in (64, 96, 128) else 0, general) * m * Hq * (d + 2) * 4}


def waves_of_the_join(splits):
    return 16 if splits > 64 else 8 if splits > 32 else 4 if splits > 8 else 1


# ------------------------------------------------------------------ convolution ------------
def conv_tokens(lens, channels, per_thread):
    """Tokens of a thread, which has `per_thread` channels."""
    return 4 if sum(ceil(t, 8) for t in lens) * (channels // per_thread) < 200000 else 8
