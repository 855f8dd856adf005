// Packed attention with capped and biased scores and a prefix mask (strd.h) on bf16 matrix cores: the tiling of attn_mfma.hip -- a
// workgroup is one query head x 32 * NW rows of ONE sequence, S^T and then O^T tile by tile with v_mfma_f32_16x16x32_bf16, K and V
// through LDS -- with four things of its own.
//  * Blocks are dealt by level over the sequences (AttnTab), the longest first; rows have pitches.
//  * A row sees the keys before its limit: its own number + 1, or its sequence's vision rows.  Limits never fall from one row to
//    the next, so a wave meets at most two 32-key blocks that only some of its rows see.
//  * A score becomes cap * tanh(score / cap): up to cap / 4 by a polynomial in the square that takes three more instructions than a
//    score without, up to cap / 2 by one of four, and where a row sees more than that in a block, as c - 2 c / (2^(score * 2 log2 e / cap) + 1)
//    in units of log2 e, with two transcendental instructions of a quarter's rate beside the softmax's one.  What no row of a wave needs is not computed.
//    The bias takes the rows' positions from LDS, where they lie as fp32 numbers beside the keys.
//  * What a row does not see does not reach it.  A probability of 0 takes a value out of the second product only if it is finite: in
//    chunks with hidden keys the values are looked at when they have landed in LDS, and those that are not finite are taken out and
//    added at the end, row by row.  And a row's softmax reference moves by the row's own scores alone, never because of a neighbour in its wave: its
//    result has the same bits whatever the rows that it does not see hold.
// Bound by the matrix products and the vector instructions of a SIMD, which overlap only in part (attn_mfma.hip), and for short
// batches by the start and end of a workgroup.  us: 8320 tokens, 32 / 8 heads of 128: 498 (1.14 PFLOP/s), biased 535, cap 50 571 to 600, both 627;
// 2176 tokens, biased 64; six sequences of 3493 tokens, 28 / 4 heads of 64, prefix 41.  A cap of 15 at scores of deviation 1 629, one that
// every score is beyond 790; where some rows of a wave's blocks are beyond half of it and some not, both forms are computed: twice the time.
#include "attn_varlen.h"

namespace strd {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazy = 8.f;       // log2 of how far a probability may exceed 1 before the reference moves
constexpr float kFar = 1048576.f;  // a softmax reference further from zero than that, in units of log2 e, is taken off the scores themselves
constexpr float kLazySum = 256.f;  // the same, of what the probabilities of a lane's 8 keys add up to

// K rows are read 16 bytes per lane, lane = (row lane % 16, piece lane / 16), V with the transposing load,
// 8 consecutive rows per half wave: both run fastest at a row pitch of 8 words modulo 32 (two pad
// vectors, never copied): 180 and 118 bytes per clock and CU, against 117 and 108 with one pad vector.
// NC = number of waves that fill the tiles.
template <int D, int NC, int KC>
struct Tile {
    using A = AsyncTile<KC, D / 8, NC, 2, true>;
    static constexpr int kPitch = A::kPitch;
    struct alignas(16) Half {
        bf16_t e[A::kBytes / 2];
        __device__ __forceinline__ const bf16_t *at(int r, int c) const { return e + r * kPitch + c; }
    };
    Half k[2];
    Half v[2];
    // In the rows' padding, so that four workgroups of 40 KB fit the LDS (8320 tokens, 28 heads of 64: 286 us with three, 276): the keys'
    // positions, eight to a row of K (only where there is a bias), ...
    static_assert((kPitch - D) * sizeof(bf16_t) >= 32, "eight numbers");
    __device__ __forceinline__ float *pos(int b, int key) { return reinterpret_cast<float *>(k[b].e + (key >> 3) * kPitch + D) + (key & 7); }
    // ... and per wave that fills the tiles, whether it has taken values out (the first group's).
    __device__ __forceinline__ int *odd() { return reinterpret_cast<int *>(v[0].e + D); }
};

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ float quarters_max(float v) {  // over the four lanes 16 apart
    v = fmaxf(v, __shfl_xor(v, 16, kWave));
    return fmaxf(v, __shfl_xor(v, 32, kWave));
}

// Takes the elements that are not finite out of the slots of a tile that this lane has copied (and that have landed); whether
// there were any, in any lane of the wave.
template <class A>
__device__ __forceinline__ bool hide_odd(bf16_t *tile, int wave, int nw) {
    bool found = false;
#pragma unroll 1
    for (int i = 0; i < A::kIssues; ++i) {
        const int s = (i * nw + wave) * kWave + (int)(threadIdx.x & 63);
        if (!A::copied(s, A::kSlots)) continue;
        u32x4 *const at = reinterpret_cast<u32x4 *>(tile) + s;
        u32x4 x = *at;
        bool mine = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool lo = (x[e] & 0x7F80u) == 0x7F80u, hi = (x[e] & 0x7F800000u) == 0x7F800000u;
            mine |= lo || hi;
            x[e] = (lo ? 0u : x[e] & 0xFFFFu) | (hi ? 0u : x[e] & 0xFFFF0000u);
        }
        if (mine) *at = x;
        found |= mine;
    }
    return __any(found);
}

struct Params {
    const bf16_t *q, *k, *v;
    bf16_t *o;
    int Hq, Hkv, xcd_map;
    float scale2;              // scale * log2 e
    // with a cap: raw scores that are a quarter and half of it, 2 log2 e * scale / cap, cap * log2 e, -2 cap * log2 e
    float near, half, kappa, c2, c2_twice;
    float tanh_near[3], tanh_half[4];  // cap log2 e tanh(raw scale / cap) / raw in powers of raw^2, up to those
    AttnMod mod;
};

// G groups of NW computing waves, and NC copy waves that serve all groups; NC = 0: the computing waves request the copies of
// their group themselves.  Group g takes chunks g, g + G, ...
template <int D, int NW, int NC, int KC, int G, bool CAP, bool BIAS>
__global__ __launch_bounds__((G * NW + NC) * kWave) __attribute__((amdgpu_waves_per_eu(2, NC ? 3 : D == 64 ? 4 : 2))) void attn_varlen_mfma_kernel(Params pr) {
    constexpr int KS = D / 32, DT = D / 16, kBM = 32 * NW;
    constexpr bool kBySum = NW == 8;   // whether the probabilities' sum or the scores' maximum says when the reference moves (attn_mfma.hip)
    // (a cap leaves scores in units of log2 e, otherwise they are raw: what the product gives)
    using TileT = Tile<D, NC ? NC : NW, KC>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lb = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);  // wave index, in a scalar register
    const int grp = G == 1 ? 0 : wv / NW, w = G == 1 ? wv : wv % NW;
    const bool copies = NC > 0 && wv >= G * NW;              // a copy wave: it serves all groups
    TileT *const all = reinterpret_cast<TileT *>(smem_raw);
    TileT &lds = all[copies ? 0 : grp];
    // All query heads and blocks of a kv head on one XCD where the heads divide evenly (attn_mfma.hip).
    int h, unit, kvh;
    if (pr.xcd_map) {
        const int ps = (pr.xcd_map - 1) & 7, gs = (pr.xcd_map - 1) >> 3;
        const int xcd = blockIdx.x % kXcd, j = blockIdx.x / kXcd, r = j >> ps;
        kvh = xcd + kXcd * (j & ((1 << ps) - 1));
        h = (kvh << gs) + (r & ((1 << gs) - 1));
        unit = r >> gs;
    } else {
        h = blockIdx.x % pr.Hq;
        unit = blockIdx.x / pr.Hq;
        kvh = h / (pr.Hq / pr.Hkv);
    }
    int level, sq;
    pr.mod.tab.locate(unit, level, sq);
    const int T = pr.mod.tab.len[sq], vis = pr.mod.prefix ? pr.mod.tab.vis[sq] : 0;
    const size_t row0 = (size_t)pr.mod.tab.row0[sq];
    const bf16_t *const k = pr.k + row0 * pr.mod.ldk, *const v = pr.v + row0 * pr.mod.ldv;
    const int32_t *const pos = BIAS && pr.mod.pos ? pr.mod.pos + row0 : nullptr;
    const int t0 = level * kBM;
    auto limit = [&](int t) { return min(max(t + 1, t < vis ? vis : 0), T); };  // keys that row t sees
    // first row of the wave, in a scalar register so that tests on it are real branches (the wave
    // index comes from threadIdx, which the compiler cannot prove uniform)
    const int wq0 = __builtin_amdgcn_readfirstlane(t0 + 32 * w);
    auto row = [&](int qt) { return wq0 + 16 * qt + lr; };  // this lane's rows of the sequence (tiles 0 and 1)
    const int wlo = limit(wq0), whi = wq0 < T ? limit(wq0 + 31) < wlo ? wlo : limit(wq0 + 31) : 0;  // keys that every / any row of the wave sees
    const int nkeys = max(min(T, t0 + kBM), t0 < vis ? vis : 0);
    const int nchunk = (nkeys + KC - 1) / KC, nstep = (nchunk + G - 1) / G;

    // Chunks in the order they are taken.  With a bias the nearest keys come first, those of the workgroup's own rows and then back to the
    // first, then the ones ahead (a prefix): from far to near the softmax reference would move in every block.  8320 tokens, 32 heads of 128,
    // slopes up to 1: 519 us, 846 in the order of the keys.
    const int own = min(t0 + kBM, nkeys) - 1, nearest = own / KC;
    auto chunk_at = [&](int i) { return BIAS && i <= nearest ? nearest - i : i; };

    using AT = typename TileT::A;
    const int cw = NC ? wv - G * NW : w;
    const uint32_t k_row = (uint32_t)pr.mod.ldk * 2, v_row = (uint32_t)pr.mod.ldv * 2, kv_col = (uint32_t)kvh * D * 2;
    // Where this lane's copies of a chunk start, from its first row, which copy waves hold: a whole chunk takes no more than its base (keys
    // and values of one pitch).  Waves that compute as well have no registers for it.
    struct From {
        uint32_t at[AT::kIssues];
    };
    auto starts = [&](From &from) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < AT::kIssues; ++i) {
            int row, cv;
            AT::slot(cw, lane, i, row, cv);
            from.at[i] = (uint32_t)row * k_row + kv_col + (uint32_t)cv * 16;
        }
    };
    // requests a chunk into buffer b of a group's tiles; rows past T re-read row T - 1
    auto stage = [&](TileT &dst, int chunk, int b, const From &from) __attribute__((always_inline)) {
        const int at = cw * kWave + lane, key = min(chunk * KC + at, T - 1);
        int32_t key_pos = key;  // (asked for before the copies, which it would else wait for)
        if (BIAS && pos && at < KC) key_pos = pos[key];
        if (NC > 0 && (chunk + 1) * KC <= T && k_row == v_row) {  // uniform
            const char *const kc = reinterpret_cast<const char *>(k) + (size_t)chunk * KC * k_row;
            const char *const vc = reinterpret_cast<const char *>(v) + (size_t)chunk * KC * v_row;
#pragma unroll
            for (int i = 0; i < AT::kIssues; ++i) AT::issue(kc + from.at[i], &dst.k[b], cw, i);
#pragma unroll
            for (int i = 0; i < AT::kIssues; ++i) AT::issue(vc + from.at[i], &dst.v[b], cw, i);
        } else {
#pragma unroll
            for (int i = 0; i < AT::kIssues; ++i) {
                int row, cv;
                AT::slot(cw, lane, i, row, cv);
                const uint32_t at_row = (uint32_t)min(chunk * KC + row, T - 1), col = kv_col + (uint32_t)cv * 16;
                AT::issue(reinterpret_cast<const char *>(k) + (at_row * k_row + col), &dst.k[b], cw, i);
                AT::issue(reinterpret_cast<const char *>(v) + (at_row * v_row + col), &dst.v[b], cw, i);
            }
        }
        if constexpr (BIAS) {
            static_assert(KC <= (NC ? NC : NW) * kWave, "one position a lane");
            if (at < KC) *dst.pos(b, at) = (float)key_pos;
        }
    };
    // Chunks with keys that not every row of the workgroup sees: values that are not finite are taken out, by the wave that copied
    // them, before anyone reads them.
    const int wg_lo = limit(t0);
    bool odd = false;  // uniform
    auto hide = [&](TileT &dst, int chunk, int b) __attribute__((always_inline)) {
        if ((chunk + 1) * KC > wg_lo && chunk < nchunk) odd |= hide_odd<AT>(dst.v[b].e, cw, NC ? NC : NW);
        if (lane == 0) all[0].odd()[grp * NW * (NC == 0) + cw] = odd;
    };
    static_assert(G == 1 || NC > 0, "a flag per wave that fills tiles");
    if (copies) {
        From from;
        starts(from);
        // (the chunk after a group's last one: clamped rows, never read)
        auto stage_step = [&](int step) __attribute__((always_inline)) {
#pragma unroll
            for (int gr = 0; gr < G; ++gr) stage(all[gr], chunk_at(step * G + gr), step & 1, from);
            async_tile_wait();
#pragma unroll
            for (int gr = 0; gr < G; ++gr) hide(all[gr], chunk_at(step * G + gr), step & 1);
            lds_barrier();
        };
        stage_step(0);
        for (int step = 0; step < nstep; ++step) stage_step(step + 1);
        if (G > 1) {
            __syncthreads();  // the two barriers of the groups' meeting
            __syncthreads();
        }
        return;
    }

    // query fragments: B operand, column = query lr of the tile, k slots d = 32 ks + 8 lb ..
    bf16x8 bq[2][KS];
    {
        const bf16_t *const q = pr.q + row0 * pr.mod.ldq + (size_t)h * D + 8 * lb;
        const bf16_t *qp0 = q + (size_t)min(row(0), T - 1) * pr.mod.ldq, *qp1 = q + (size_t)min(row(1), T - 1) * pr.mod.ldq;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            bq[0][ks] = *reinterpret_cast<const bf16x8 *>(qp0 + 32 * ks);
            bq[1][ks] = *reinterpret_cast<const bf16x8 *>(qp1 + 32 * ks);
        }
    }
    float pos_q[2] = {0.f, 0.f}, slope = 0.f;
    if constexpr (BIAS) {
        slope = CAP ? pr.mod.slopes[h] * kLog2e : pr.mod.slopes[h] / pr.mod.scale;  // in the scores' units
        slope = fminf(fmaxf(slope, -1e30f), 1e30f);  // (infinity times a distance of 0 is NaN)
        slope = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, slope)));  // (a scalar register)
        pos_q[0] = (float)(pos ? pos[min(row(0), T - 1)] : row(0));
        pos_q[1] = (float)(pos ? pos[min(row(1), T - 1)] : row(1));
    }

    // O^T tiles: oacc[dt][qt][r] = channel 16 dt + 4 lb + r of query (qt, lr)
    f32x4 oacc[DT][2];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) oacc[dt][0] = oacc[dt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    // per query tile; l_run: this lane group's share of the row sum
    float m_run[2] = {-INFINITY, -INFINITY}, m_neg[2] = {0.f, 0.f}, l_run[2] = {0.f, 0.f};
    const float scale2 = CAP ? 1.f : pr.scale2, lazy_raw = kLazy / scale2;  // scores' units -> log2
    // A reference far from zero (large scores; keys ahead under a steep bias) has no place in the instruction that gives an exponent: what is rounded
    // off it there is half a step of its own size, from 2^26 on a power of two that a sum may not hold.  Such a row's scores are taken less the
    // reference first, in every block, and 0 is added.  What marks the row makes every block look at the references: with a cap m_neg is 0; without one
    // m_run is -inf, as before the first key, and m_neg the reference, else 0.  (A flag of the wave beside them: 2 to 4 % slower; so 1 % at most.)
    auto is_far = [&](float m) { return m > -INFINITY && fabsf(m * scale2) > kFar; };
    auto reference = [&](int qt) { return CAP || m_run[qt] > -INFINITY || m_neg[qt] == 0.f ? m_run[qt] : m_neg[qt]; };

    constexpr int kRowB = TileT::kPitch * 2;  // row pitch of the tiles in bytes
    From from;
    if (NC == 0) {
        stage(lds, chunk_at(grp), 0, from);
        async_tile_wait();
        hide(lds, chunk_at(grp), 0);
    }
    lds_barrier();  // the groups' first chunks have landed
    for (int step = 0; step < nstep; ++step) {
        const int cur = step & 1, chunk = chunk_at(step * G + grp), next = chunk_at((step + 1) * G + grp);
        if (NC == 0) stage(lds, next, cur ^ 1, from);  // the group's next chunk (past the last chunk: clamped rows, never read)
#pragma unroll
        for (int kn = 0; kn < KC / 32; ++kn) {
            const int kt = BIAS ? KC / 32 - 1 - kn : kn;  // (nearest first, as far as the chunks go back)
            const int kb = chunk * KC + 32 * kt;
            if (kb < whi) {  // uniform per wave
                // all key fragments of the 32 keys first (one LDS round trip, not one per product):
                // A operand, row = key lr of a 16-key tile, k slots d = 32 ks + 8 lb ..
                bf16x8 kf[2][KS];
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
                        kf[j][ks] = *reinterpret_cast<const bf16x8 *>(lds.k[cur].at(32 * kt + 16 * j + lr, 32 * ks + 8 * lb));
                __builtin_amdgcn_sched_barrier(0);
                // sacc[qt][j][r] = score of key kb + 16 j + 4 lb + r for query (qt, lr)
                f32x4 sacc[2][2];
#pragma unroll
                for (int qt = 0; qt < 2; ++qt) sacc[qt][0] = sacc[qt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
                // products first: the other wave of the SIMD is most likely in its softmax, and a
                // matrix instruction that waits behind its vector instructions leaves the matrix pipe idle
                __builtin_amdgcn_s_setprio(2);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int qt = 0; qt < 2; ++qt) sacc[qt][j] = mfma16(kf[j][ks], bq[qt][ks], sacc[qt][j]);
                }
                __builtin_amdgcn_s_setprio(0);
                // the transposed V fragments are requested now and arrive during the softmax: lane group lb
                // passes rows 4 lb + lr / 4 (then + 16) and columns 4 (lr % 4) of a 16-channel tile and
                // receives, for channel lr, the keys 4 lb .. 4 lb + 3 (then 16 + 4 lb ..): the slot order of P
                // (64 channels now -- with a cap or a bias once it is in, their registers are needed until then; the other 64 are requested after the
                // softmax, when the score registers are free)
                strd_s16x4 vr8[DT / 4][8];
                const bf16_t *vp = lds.v[cur].at(32 * kt + 4 * lb + (lr >> 2), 4 * (lr & 3));
                if constexpr (!CAP && !BIAS)
                    lds_issue_tr8<0, 16 * kRowB, 32, 16 * kRowB + 32, 64, 16 * kRowB + 64, 96, 16 * kRowB + 96>(vp, vr8[0]);
                const bool edge = kb + 32 > wlo;  // uniform: some (key, query) pair of the block is masked
                auto hide_scores = [&](float with) __attribute__((always_inline)) {
                    // (hides the row: keeps this a branch -- folded into selects it would run for every block -- and the limits out of registers)
                    int first = row(0);
                    asm volatile("" : "+v"(first));
                    const int lim[2] = {limit(first), limit(first + 16)};
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int key = kb + 16 * j + 4 * lb + r;
                            if (key >= lim[0]) sacc[0][j][r] = with;
                            if (key >= lim[1]) sacc[1][j][r] = with;
                        }
                };
                if constexpr (CAP) {
                    // (less the row's reference, added in the same instruction: the exponents as they are, unless the reference moves)
                    auto each = [&](auto form) __attribute__((always_inline)) {
#pragma unroll
                        for (int qt = 0; qt < 2; ++qt)
#pragma unroll
                            for (int j = 0; j < 2; ++j)
#pragma unroll
                                for (int r = 0; r < 4; ++r) sacc[qt][j][r] = form(qt, sacc[qt][j][r]);
                    };
                    auto near = [&](float w) { return fmaf(w, fmaf(w, pr.tanh_near[2], pr.tanh_near[1]), pr.tanh_near[0]); };
                    auto half = [&](int qt, float y) {
                        const float w = y * y, h = fmaf(w, fmaf(w, fmaf(w, pr.tanh_half[3], pr.tanh_half[2]), pr.tanh_half[1]), pr.tanh_half[0]);
                        return fmaf(y, fabsf(y) <= pr.near ? near(w) : h, m_neg[qt]);
                    };
                    auto any = [&](int qt, float y) { return fmaf(pr.c2_twice, __builtin_amdgcn_rcpf(ex2(y * pr.kappa) + 1.f), pr.c2 + m_neg[qt]); };
                    if (BIAS && edge) hide_scores(0.f);  // (here for registers' sake, else below)
                    float far = 0.f;
                    each([&](int, float y) { far = fmaxf(far, fabsf(y)); return y; });
                    if (__builtin_expect(!__any(far > pr.near), 1)) {
                        each([&](int qt, float y) { return fmaf(y, near(y * y), m_neg[qt]); });
                    } else if (!__any(far > pr.half)) {
                        each(half);
                    } else {
                        // What a row sees of the block decides for all of it, so that nothing else has a part in its bits; where every row takes the
                        // exponential form, nothing else is computed.
                        if (!BIAS && edge) hide_scores(0.f);
                        float top[2] = {0.f, 0.f};
                        each([&](int qt, float y) { top[qt] = fmaxf(top[qt], fabsf(y)); return y; });
                        top[0] = quarters_max(top[0]), top[1] = quarters_max(top[1]);
                        if (__any(fminf(top[0], top[1]) <= pr.half)) each([&](int qt, float y) { return top[qt] <= pr.half ? half(qt, y) : any(qt, y); });
                        else each(any);
                    }
                }
                if constexpr (BIAS) {
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const f32x4 pk = *reinterpret_cast<const f32x4 *>(lds.pos(cur, 32 * kt + 16 * j + 4 * lb));
#pragma unroll
                        for (int qt = 0; qt < 2; ++qt)
#pragma unroll
                            for (int r = 0; r < 4; ++r) sacc[qt][j][r] = fmaf(-slope, fabsf(pk[r] - pos_q[qt]), sacc[qt][j][r]);
                    }
                }
                if (edge) hide_scores(-INFINITY);
                if constexpr (CAP || BIAS)
                    lds_issue_tr8<0, 16 * kRowB, 32, 16 * kRowB + 32, 64, 16 * kRowB + 64, 96, 16 * kRowB + 96>(vp, vr8[0]);
                // The probabilities, against the reference as it is (of a row that has seen no key yet: 0), rounded to bf16 for the second product as in
                // attn_mfma.hip: in two parts they would take half of all products again, 235 us of 8320 tokens' 590 at the rate of a large one.  The row
                // sum is taken of them as they enter the product (numerator and denominator then carry the same rounding), two at a time.
                bf16x8 pf[2];
                float ps[2];
                auto probabilities = [&](const float (&less)[2]) __attribute__((always_inline)) {
#pragma unroll
                    for (int qt = 0; qt < 2; ++qt) {
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                pf[qt][4 * j + r] = (bf16_t)ex2(CAP ? sacc[qt][j][r] : fmaf(sacc[qt][j][r], scale2, less[qt]));
                        ps[qt] = kBySum ? 0.f : l_run[qt];
#pragma unroll
                        for (int e = 0; e < 8; e += 2)
                            ps[qt] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pf[qt][e], pf[qt][e + 1]}, bf16x2{(bf16_t)1.f, (bf16_t)1.f}, ps[qt], false);
                    }
                };
                float tm[2];  // max of this lane's 8 scores per query tile
                auto maxima = [&]() __attribute__((always_inline)) {
#pragma unroll
                    for (int qt = 0; qt < 2; ++qt) {
                        tm[qt] = sacc[qt][0][0];
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int r = 0; r < 4; ++r) tm[qt] = fmaxf(tm[qt], sacc[qt][j][r]);
                    }
                };
                // m_run is the reference the exponentials are taken against, common to the four lane groups of a query.  It
                // follows the running max lazily (attn_mfma.hip): it moves when some lane of the QUERY sees a score more than 2^kLazy above
                // it, or (kBySum) eight probabilities that add up to more than kLazySum, or the first key.
                auto limit_of = [&](int qt) { return CAP ? m_neg[qt] == 0.f ? -INFINITY : lazy_raw : m_run[qt] + lazy_raw; };  // (of a maximum)
                bool moves;
                if constexpr (kBySum) {
                    probabilities(m_neg);
                    moves = __any(fmaxf(ps[0], ps[1]) > kLazySum || (CAP ? m_neg[0] * m_neg[1] == 0.f : fminf(m_run[0], m_run[1]) == -INFINITY));
                    if (moves) maxima();
                } else {
                    maxima();
                    moves = __any(tm[0] > limit_of(0) || tm[1] > limit_of(1));
                }
                float less[2] = {m_neg[0], m_neg[1]};  // (without a cap: what is added to a score in the exponent)
                if (moves) {
#pragma unroll
                    for (int qt = 0; qt < 2; ++qt) {
                        const float t = quarters_max(tm[qt]), why = kBySum ? quarters_max(ps[qt]) : t, old = reference(qt);
                        const bool own = (CAP ? m_neg[qt] == 0.f : m_run[qt] == -INFINITY) || why > (kBySum ? kLazySum : limit_of(qt));
                        // (a row may not see any key of the groups behind the first, whose chunks start later)
                        const float nm = own ? fmaxf(old, CAP ? t - m_neg[qt] : t) : old;
                        const bool none = nm == -INFINITY, apart = is_far(nm);
                        const float corr = none ? 1.f : ex2((old - nm) * scale2);
                        l_run[qt] *= corr;
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) oacc[dt][qt] *= corr;
                        const float neg = none || apart ? 0.f : -nm * scale2, by = (CAP ? neg - m_neg[qt] : 0.f) - (apart ? nm : 0.f);
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int r = 0; r < 4; ++r) sacc[qt][j][r] += by;
                        m_run[qt] = !CAP && apart ? -INFINITY : nm;
                        m_neg[qt] = !CAP && apart ? nm : neg;
                        if constexpr (!CAP) less[qt] = neg;
                    }
                    if constexpr (kBySum) probabilities(less);
                }
                if constexpr (!kBySum) probabilities(less);
                l_run[0] = kBySum ? l_run[0] + ps[0] : ps[0];
                l_run[1] = kBySum ? l_run[1] + ps[1] : ps[1];
#pragma unroll
                for (int dp = 1; dp < DT / 4; ++dp)
                    lds_issue_tr8<0, 16 * kRowB, 32, 16 * kRowB + 32, 64, 16 * kRowB + 64, 96, 16 * kRowB + 96>(vp + 64 * dp, vr8[dp]);
                __builtin_amdgcn_s_setprio(2);
#pragma unroll
                for (int dp = 0; dp < DT / 4; ++dp) {
                    strd_s16x4(&r)[8] = vr8[dp];
                    if (dp + 1 < DT / 4)
                        lds_settle8_but<8 * (DT / 4 - 1)>(r);  // LDS reads return in order: the later batch may still travel
                    else
                        lds_settle8(r);
#pragma unroll
                    for (int dd = 0; dd < 4; ++dd) {
                        const bf16x8 vf = tr_pair(r[2 * dd], r[2 * dd + 1]);
                        oacc[4 * dp + dd][0] = mfma16(vf, pf[0], oacc[4 * dp + dd][0]);
                        oacc[4 * dp + dd][1] = mfma16(vf, pf[1], oacc[4 * dp + dd][1]);
                    }
                }
                __builtin_amdgcn_s_setprio(0);
            }
        }
        if (NC == 0) {
            async_tile_wait();
            hide(lds, next, cur ^ 1);
        }
        lds_barrier();  // the next chunk has landed, every wave is done with this one
    }

#pragma unroll
    for (int i = 0; i < (NC ? NC : NW); ++i) odd |= all[0].odd()[i] != 0;
    // this wave's row sums: the four lane groups of a query hold different keys
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
        l_run[qt] += __shfl_xor(l_run[qt], 16, kWave);
        l_run[qt] += __shfl_xor(l_run[qt], 32, kWave);
    }
    if constexpr (G > 1) {
        // the later groups leave their accumulators, maxima and sums in LDS (the chunks are done with), lane by
        // lane in the layout the first group's waves hold theirs
        static_assert(G == 2, "one partner per wave");
        constexpr int kPart = DT * 2 + 1;  // f32x4s per lane: accumulators, then (max, sum) of both query tiles
        f32x4 *part = reinterpret_cast<f32x4 *>(smem_raw) + (size_t)w * kPart * kWave + lane;
        static_assert((size_t)NW * kPart * kWave * sizeof(f32x4) <= G * sizeof(TileT), "partials fit the tiles' LDS");
        async_tile_wait();  // (copies past the last chunk)
        m_run[0] = reference(0), m_run[1] = reference(1);
        __syncthreads();
        if (grp == 1) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                part[(2 * dt) * kWave] = oacc[dt][0];
                part[(2 * dt + 1) * kWave] = oacc[dt][1];
            }
            part[2 * DT * kWave] = f32x4{m_run[0], l_run[0], m_run[1], l_run[1]};
        }
        __syncthreads();
        if (grp == 1) return;
        const f32x4 ml = part[2 * DT * kWave];
#pragma unroll
        for (int qt = 0; qt < 2; ++qt) {
            const float mo = ml[2 * qt], nm = fmaxf(m_run[qt], mo);
            const float ca = ex2((m_run[qt] - nm) * scale2), cb = ex2((mo - nm) * scale2);  // 0 where it saw no key
            l_run[qt] = l_run[qt] * ca + ml[2 * qt + 1] * cb;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) oacc[dt][qt] = oacc[dt][qt] * ca + part[(2 * dt + qt) * kWave] * cb;
        }
    }
    if (__builtin_expect(odd, 0)) {
        // The values left out of the products, for the rows that see them.  A probability is above 0 and a finite factor leaves such a
        // value as it is, so the value itself is added.
        const int lim[2] = {limit(row(0)), limit(row(1))};
#pragma unroll 1
        for (int key = wg_lo / KC * KC; key < whi; ++key) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const bf16x4 vv = *reinterpret_cast<const bf16x4 *>(v + (size_t)key * pr.mod.ldv + (size_t)kvh * D + 16 * dt + 4 * lb);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float val = fabsf((float)vv[r]) < INFINITY ? 0.f : (float)vv[r];
                    oacc[dt][0][r] += key < lim[0] ? val : 0.f;
                    oacc[dt][1][r] += key < lim[1] ? val : 0.f;
                }
            }
        }
    }
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
        const int tq = row(qt);
        if (tq < T) {
            const float inv = 1.f / l_run[qt];
            bf16_t *op = pr.o + ((row0 + tq) * pr.Hq + h) * D + 4 * lb;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                bf16x4 out;
#pragma unroll
                for (int e = 0; e < 4; ++e) out[e] = (bf16_t)(oacc[dt][qt][e] * inv);
                *reinterpret_cast<bf16x4 *>(op + 16 * dt) = out;
            }
        }
    }
}

template <int D, int NW, int NC, int KC, int G, bool CAP, bool BIAS>
int launch_mod(const Params &pr, long long units, hipStream_t st) {
    const size_t smem = G * sizeof(Tile<D, NC ? NC : NW, KC>);
    if (!allow_dynamic_lds(reinterpret_cast<const void *>(&attn_varlen_mfma_kernel<D, NW, NC, KC, G, CAP, BIAS>), smem)) return STRD_EHIP;
    attn_varlen_mfma_kernel<D, NW, NC, KC, G, CAP, BIAS><<<(unsigned)(units * pr.Hq), (G * NW + NC) * kWave, smem, st>>>(pr);
    return launch_status();
}

template <int D, int NW, int NC, int KC, int G>
int launch(Params &pr, const strd_seq *seqs, int nseq, hipStream_t st) {
    long long rows, units;
    if (!plan_attn(seqs, nseq, 32 * NW, pr.mod.tab, rows, units)) return STRD_EINVAL;
    if (units * pr.Hq > 0x7FFFFFFFLL) return STRD_EUNSUPPORTED;
    const bool cap = pr.mod.cap > 0.f, bias = pr.mod.slopes != nullptr;
    return cap    ? bias ? launch_mod<D, NW, NC, KC, G, true, true>(pr, units, st) : launch_mod<D, NW, NC, KC, G, true, false>(pr, units, st)
           : bias ? launch_mod<D, NW, NC, KC, G, false, true>(pr, units, st)
                  : launch_mod<D, NW, NC, KC, G, false, false>(pr, units, st);
}

template <int D>
int launch_d(Params &pr, const strd_seq *seqs, int nseq, long long blocks128, long long blocks256, int longest, hipStream_t st) {
    const int Hq = pr.Hq;
    const long long wgs128 = blocks128 * Hq, wgs256 = blocks256 * Hq;
    if constexpr (D == 64) {
        // Four workgroups of four waves fit a CU, and pass one of 256 rows (8320 tokens, 28 heads: 276 / 286 us;
        // six sequences of 3493 tokens and a prefix 43 / 50).  Few of them: two groups of waves with a copying one, each on half of the keys (2981
        // tokens, 28 heads 57 / 53 us; 2176 tokens, 32 heads 44 / 40, with a prefix 62 / 66; 3493 tokens in six, 28 heads 31 / 41).
        const bool one = longest <= 256 || wgs128 > (pr.mod.prefix ? 512 : 640 + 4 * blocks128);
        return one ? launch<D, 4, 0, 64, 1>(pr, seqs, nseq, st) : launch<D, 4, 4, 64, 2>(pr, seqs, nseq, st);
    } else {
        // In causal order as for one sequence (attn_mfma.hip).  With a prefix the blocks of a sequence cost the same, and what counts is the
        // rounds of the chip: one of 256 rows a workgroup takes 1.6 times one of 128 (2176 tokens, 32 heads, 2 rounds / 3: 106 / 103 us).
        const long long rounds256 = (wgs256 + 255) / 256, rounds128 = (wgs128 + 255) / 256;
        const bool big = pr.mod.prefix ? longest > 256 && 8 * rounds256 < 5 * rounds128 : wgs256 >= 384;
        const bool one = longest <= 256 || wgs128 > 512 + 7 * blocks128;
        return big   ? launch<D, 8, 4, 128, 1>(pr, seqs, nseq, st)
               : one ? launch<D, 4, 0, 64, 1>(pr, seqs, nseq, st)
                     : launch<D, 4, 4, 64, 2>(pr, seqs, nseq, st);
    }
}

}  // namespace

bool attn_varlen_mfma_supported(int Hq, int Hkv, int d, strd_dtype io) {
    (void)Hkv;
    return io == STRD_BF16 && (d == 64 || d == 128) && Hq <= 1 << 20;
}
// Staging uses 32-bit byte offsets into a sequence's keys and values.
bool attn_varlen_mfma_reaches(int longest, long long ldk, long long ldv) {
    return (unsigned long long)(longest + 256LL) * (unsigned long long)(ldk > ldv ? ldk : ldv) * 2 < 1ull << 32;
}

int attn_varlen_mfma(const void *q, const void *k, const void *v, void *o, int Hq, int Hkv, int d, const AttnMod &mod, const strd_seq *seqs,
                     int nseq, hipStream_t st) {
    Params pr;
    pr.q = (const bf16_t *)q, pr.k = (const bf16_t *)k, pr.v = (const bf16_t *)v, pr.o = (bf16_t *)o;
    pr.Hq = Hq, pr.Hkv = Hkv;
    pr.scale2 = mod.scale * kLog2e;
    pr.kappa = 2.f * kLog2e * mod.scale * mod.inv_cap;
    pr.c2 = mod.cap * kLog2e, pr.c2_twice = -2.f * pr.c2;
    // tanh(y) / y up to y = 0.25 and 0.5, of least relative error (4.0e-7, 5.5e-7: 5e-6 and 1.4e-5 of a score under a cap of 50, where the probability's
    // rounding to bf16 is 4e-3); y = ky raw goes into the coefficients.  Where those of the
    // higher powers leave fp32's range (a cap far above every score) the polynomials end before they count, where they are too large (a cap far
    // below) the exponential form, whose absolute error is a few steps of the cap, takes every score.
    const double near_y[3] = {0.99999960434, -0.33321908205, 0.12841613181}, half_y[4] = {0.999999452, -0.333263082, 0.131902465, -0.0444017053};
    const double ky = (double)mod.scale * mod.inv_cap;
    pr.half = ky > 1e4 ? -1.f : fminf((float)((ky > 1e-5 ? 0.5 : ky > 1e-9 ? 0.05 : 1e-3) / ky), 1e18f);
    pr.near = 0.5f * pr.half;
    double power = (double)mod.scale * kLog2e;
    for (int i = 0; i < 4; ++i, power *= ky * ky) {
        pr.tanh_half[i] = (float)(half_y[i] * power);
        if (i < 3) pr.tanh_near[i] = (float)(near_y[i] * power);
    }
    pr.mod = mod;
    // XCD-aware order when the kv heads per XCD and the query heads per kv head are powers of two
    const int per = Hkv / kXcd, gq = Hq / Hkv;
    const bool pow2 = Hkv % kXcd == 0 && (per & (per - 1)) == 0 && (gq & (gq - 1)) == 0 && per <= 128;
    pr.xcd_map = pow2 ? 1 + __builtin_ctz(per) + 8 * __builtin_ctz(gq) : 0;
    long long b128 = 0, b256 = 0;
    int longest = 0;
    for (int i = 0; i < nseq; ++i) {
        const int n = seqs[i].N + seqs[i].M;
        b128 += ceil_div(n, 128);
        b256 += ceil_div(n, 256);
        longest = max(longest, n);
    }
    return d == 128 ? launch_d<128>(pr, seqs, nseq, b128, b256, longest, st) : launch_d<64>(pr, seqs, nseq, b128, b256, longest, st);
}

}  // namespace strd
