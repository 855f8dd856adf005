// The rows of the cache that a drafted tree attends to (attn_tree.hip) on bf16 matrix cores, heads of 64, 96 or 128 channels.
//  * The query rows of a kv head -- m nodes times the query heads that share it -- are the columns of the products S^T = K Q^T and O^T = V^T P^T
//    (v_mfma_f32_16x16x32_bf16), 32 to a wave, up to 8 waves to a workgroup; keys and values pass through LDS once for all of them, so that
//    the cache is read from HBM once.  Accumulator rows are keys, then channels: a lane holds whole columns' parts, the softmax is its own.
//  * The nodes' keys follow the cache's in one row of blocks of 32, cut into splits; the masks are looked at in the blocks that hold nodes only.  A
//    weight of 0 takes a value out of the second product only if it is finite: in chunks with nodes the values are looked at when they have landed in
//    LDS, and those that are not finite are taken out and added at the end, row by row.
//  * A row's softmax has a reference that moves when eight of its weights add up to more than 2^8, or at its first keys.
// 64 nodes of 32 heads behind 131627 rows, capped and biased: 178 us for 541 MB and 138 GFLOP (775 TFLOP/s; 175 before capped
// references far from zero were taken off the scores; other shapes took the same), then 11 to join 32 splits; the matrix units are at
// work 35 % of the time and the vector units 50 % (10 instructions a score, one of them an exponential), at 2.0 GHz of 2.4.  Neither of the two alone bounds
// it: fewer instructions in the cap, other priorities of the waves and other chunks all take 175 +- 2.  Few rows are bound by HBM: 8 nodes 110 us, 4.9 TB/s.
#include <algorithm>

#include "attn_tree.h"

namespace strd {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr float kLazySum = 256.f, kFar = 1048576.f;  // a reference further from zero is taken off the scores themselves

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float quarters_max(float v) {  // over the four lanes 16 apart
    v = fmaxf(v, __shfl_xor(v, 16, kWave));
    return fmaxf(v, __shfl_xor(v, 32, kWave));
}

// K rows are read 16 bytes per lane, V with the transposing load: both run fastest at a row pitch of 8 words modulo 32 (two pad vectors, never
// copied; attn_varlen_mfma.hip).  NF: waves that fill the tiles.
template <int D, int NW, int NF, int KC>
struct Tile {
    using A = AsyncTile<KC, D / 8, NF, 2, true>;
    static constexpr int kPitch = A::kPitch;
    struct alignas(16) Half {
        bf16_t e[A::kBytes / 2];
        __device__ __forceinline__ const bf16_t *at(int r, int c) const { return e + r * kPitch + c; }
    };
    Half k[2], v[2];
    uint64_t nodes[32 * NW];    // the nodes that a row of the workgroup sees
    float2 bias[32 * NW];       // its position and slope
    // the keys' positions, eight to a row, in the padding of K
    static_assert((kPitch - D) * sizeof(bf16_t) >= 32, "eight numbers");
    __device__ __forceinline__ float *pos(int b, int key) { return reinterpret_cast<float *>(k[b].e + (key >> 3) * kPitch + D) + (key & 7); }
    // per wave that fills the tiles, whether it has taken values out, in that of V
    __device__ __forceinline__ int *odd() { return reinterpret_cast<int *>(v[0].e + D); }
};

// Takes the elements that are not finite out of the slots of a tile that this lane has copied (and that have landed); whether there were any, in
// any lane of the wave.
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
    TreeCall a;
    TreeWs ws;
    int nsplit, per;         // splits, blocks of 32 keys in each (the last: what is left)
    int row_blocks, nmain;   // workgroups' rows per kv head; workgroups
    float scale2;            // scale * log2 e
    // with a cap: raw scores that are a quarter and half of it, 2 log2 e * scale / cap, cap * log2 e, -2 cap * log2 e, and
    // cap log2 e tanh(raw scale / cap) / raw in powers of raw^2, up to those
    float near, half, kappa, c2, c2_twice, tanh_near[3], tanh_half[4];
};

// NW computing waves of 32 query rows; NC waves that copy (0: the computing ones do); chunks of KC keys.
template <int D, int NW, int NC, int KC, bool CAP, bool BIAS>
__global__ __launch_bounds__((NW + NC) * kWave) __attribute__((amdgpu_waves_per_eu(NC ? 3 : 2))) void tree_mfma_kernel(Params pr) {
    constexpr int KS = D / 32, DT = D / 16, NF = NC ? NC : NW;
    constexpr int kFours = DT / 4, kLast = DT % 4;  // tiles of V: four at a time, and the last two of 96 channels
    static_assert(kFours <= 2 && (kLast == 0 || kLast == 2), "the waits below");
    using TileT = Tile<D, NW, NF, KC>;
    using AT = typename TileT::A;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
    TileT &lds = *reinterpret_cast<TileT *>(smem_raw);
    const TreeCall &a = pr.a;
    const int rep = a.Hq / a.Hkv, R = a.m * rep;
    const int unit = xcd_swizzle(blockIdx.x, pr.nmain);
    if (unit >= pr.nmain) return;
    // the row blocks of a kv head and split are neighbours, then the kv heads of a split
    const int rb = unit % pr.row_blocks, hk = unit / pr.row_blocks % a.Hkv, split = unit / pr.row_blocks / a.Hkv;
    const int key0 = 32 * split * pr.per, nkeys = min(32 * pr.per, a.T + a.m - key0);
    const int plain = min(nkeys, a.T - key0);  // keys that every row sees (below 0: none)
    const int nchunk = (nkeys + KC - 1) / KC;
    auto chunk_at = [&](int i) { return BIAS ? nchunk - 1 - i : i; };  // nearest first: from far to near the reference would move in every block
    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lb = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);

    const uint32_t row_bytes = (uint32_t)a.Hkv * D * 2;
    const int cw = NC ? w - NW : w;
    // Where this lane's copies of a chunk start, from its first row, which copy waves hold (waves that compute as well have no registers for it).
    struct From {
        uint32_t at[AT::kIssues];
    } from;
    if (NC)
#pragma unroll
        for (int i = 0; i < AT::kIssues; ++i) {
            int row, cv;
            AT::slot(cw, lane, i, row, cv);
            from.at[i] = (uint32_t)row * row_bytes + (uint32_t)cv * 16;
        }
    // requests chunk c into buffer b; keys past the last node: that one again, hidden from everyone
    auto stage = [&](int c, int b) __attribute__((always_inline)) {
        const int first = key0 + c * KC, at = cw * kWave + lane;
        float where = 0.f;
        if (BIAS && at < KC) where = a.place(min(first + at, a.T + a.m - 1));  // (asked for before the copies, which it would else wait for)
        if (first + KC <= a.T) {  // uniform
            const size_t base = (size_t)first * row_bytes + (size_t)hk * D * 2;
            const char *const kc = reinterpret_cast<const char *>(a.k_cache) + base, *const vc = reinterpret_cast<const char *>(a.v_cache) + base;
#pragma unroll
            for (int i = 0; i < AT::kIssues; ++i) {
                uint32_t off;
                if constexpr (NC > 0) {
                    off = from.at[i];
                } else {
                    int row, cv;
                    AT::slot(cw, lane, i, row, cv);
                    off = (uint32_t)row * row_bytes + (uint32_t)cv * 16;
                }
                AT::issue(kc + off, &lds.k[b], cw, i);
                AT::issue(vc + off, &lds.v[b], cw, i);
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < AT::kIssues; ++i) {
                int row, cv;
                AT::slot(cw, lane, i, row, cv);
                const int j = min(first + row, a.T + a.m - 1);
                const size_t off = (size_t)(j < a.T ? j : j - a.T) * row_bytes + (size_t)hk * D * 2 + (uint32_t)cv * 16;
                AT::issue(reinterpret_cast<const char *>(j < a.T ? a.k_cache : a.k_new) + off, &lds.k[b], cw, i);
                AT::issue(reinterpret_cast<const char *>(j < a.T ? a.v_cache : a.v_new) + off, &lds.v[b], cw, i);
            }
        }
        if constexpr (BIAS) {
            static_assert(KC <= NF * kWave, "one position a lane");
            if (at < KC) *lds.pos(b, at) = where;
        }
    };
    // what has been requested has landed; in chunks with nodes values that are not finite are taken out before anyone reads them
    bool odd = false;  // uniform
    auto landed = [&](int c, int b) __attribute__((always_inline)) {
        async_tile_wait();
        if (key0 + (c + 1) * KC > a.T) odd |= hide_odd<AT>(lds.v[b].e, cw, NF);
        if (lane == 0) lds.odd()[cw] = odd;
    };
    if (NC && w >= NW) {
        stage(chunk_at(0), 0);
        landed(chunk_at(0), 0);
        lds_barrier();
        for (int i = 0; i < nchunk; ++i) {
            if (i + 1 < nchunk) {
                stage(chunk_at(i + 1), (i + 1) & 1);
                landed(chunk_at(i + 1), (i + 1) & 1);
            }
            lds_barrier();
        }
        return;
    }
    if (!NC) stage(chunk_at(0), 0);

    // query fragments: B operand, column = row lr of the tile, k slots d = 32 ks + 8 lb ..
    bf16x8 bq[2][KS];
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
        const int r = min(32 * (NW * rb + w) + 16 * qt + lr, R - 1), node = r / rep, h = hk * rep + r % rep;
        const bf16_t *q = (const bf16_t *)a.q + ((size_t)node * a.Hq + h) * D + 8 * lb;
        if (lb == 0) lds.nodes[32 * w + 16 * qt + lr] = a.mask[node] & (a.m < 64 ? (1ull << a.m) - 1 : ~0ull);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) bq[qt][ks] = *reinterpret_cast<const bf16x8 *>(q + 32 * ks);
        // (the slope in the scores' units; infinity times a distance of 0 is NaN)
        if (BIAS && lb == 0)
            lds.bias[32 * w + 16 * qt + lr] = {a.place(a.T + node), fminf(fmaxf(CAP ? a.slopes[h] * kTreeLog2e : a.slopes[h] / a.scale, -1e30f), 1e30f)};
    }
    // This lane's row in the workgroup, computed anew: nothing is held in registers for the few places that need it.
    auto row_anew = [&](int qt) {
        uint32_t none = 0, wave = w;
        asm volatile("" : "+s"(none), "+s"(wave));
        return 32 * wave + 16 * qt + (__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, none)) & 15);
    };
    // Which of the 32 keys from node `first` on (rows of the cache below 0) this lane's row sees.
    auto visible = [&](int qt, int first) -> uint32_t {
        const uint64_t nodes = lds.nodes[row_anew(qt)];
        if (first >= 0) return (uint32_t)(nodes >> first);
        return (uint32_t)(nodes << -first) | ((1u << -first) - 1);  // (first > -32: the block has a node)
    };
    // O^T tiles: oacc[dt][qt][e] = channel 16 dt + 4 lb + e of row (qt, lr)
    f32x4 oacc[DT][2];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) oacc[dt][0] = oacc[dt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    // per row: the reference, -infinity before the first key, and what is added to an exponent for it (with a cap to a score; 0 where it is far from zero);
    // l_run: this lane group's share of the sum
    float ref[2] = {-INFINITY, -INFINITY}, less[2] = {0.f, 0.f}, l_run[2] = {0.f, 0.f};
    const float scale2 = CAP ? 1.f : pr.scale2;  // scores' units -> log2 (with a cap the scores are in them)
    bool far_ref = false;  // uniform: some row's reference is far from zero
    // (or its capped scores may be: with a bias of their size a reference may be anywhere)
    auto is_far = [&](float r) { return r > -INFINITY && ((CAP && pr.c2 > kFar) || fabsf(r * scale2) > kFar); };
    const bool live = 32 * (NW * rb + w) < R;

    constexpr int kRowB = TileT::kPitch * 2;
    if (!NC) landed(chunk_at(0), 0);
    lds_barrier();
    for (int i = 0; i < nchunk; ++i) {
        const int cur = i & 1, c = chunk_at(i);
        if (!NC && i + 1 < nchunk) stage(chunk_at(i + 1), cur ^ 1);
#pragma unroll
        for (int kn = 0; kn < KC / 32; ++kn) {
            const int kt = BIAS ? KC / 32 - 1 - kn : kn;
            if (c * KC + 32 * kt >= nkeys || !live) continue;  // uniform
            // all key fragments of the 32 keys first: A operand, row = key lr of a 16-key tile, k slots d = 32 ks + 8 lb ..
            bf16x8 kf[2][KS];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) kf[j][ks] = *reinterpret_cast<const bf16x8 *>(lds.k[cur].at(32 * kt + 16 * j + lr, 32 * ks + 8 * lb));
            __builtin_amdgcn_sched_barrier(0);
            // s[qt][j][e] = score of key 16 j + 4 lb + e for row (qt, lr)
            f32x4 s[2][2];
#pragma unroll
            for (int qt = 0; qt < 2; ++qt) s[qt][0] = s[qt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
            __builtin_amdgcn_s_setprio(2);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int qt = 0; qt < 2; ++qt) s[qt][j] = mfma16(kf[j][ks], bq[qt][ks], s[qt][j]);
            __builtin_amdgcn_s_setprio(0);
            // the transposed V fragments are requested now and arrive during the softmax (with a cap or a bias once it is in): lane group lb passes
            // rows 4 lb + lr / 4 (then + 16) and columns 4 (lr % 4) of a 16-channel tile and receives, for channel lr, the keys
            // 4 lb .. 4 lb + 3 (then 16 + 4 lb ..): the slot order of P
            strd_s16x4 vr8[kFours][8], vr4[4];
            const bf16_t *vt = lds.v[cur].at(32 * kt + 4 * lb + (lr >> 2), 4 * (lr & 3));
            const bool edge = c * KC + 32 * kt + 32 > plain;  // uniform: some key of the block is hidden from some row
            if constexpr (!CAP && !BIAS) lds_issue_tr8<0, 16 * kRowB, 32, 16 * kRowB + 32, 64, 16 * kRowB + 64, 96, 16 * kRowB + 96>(vt, vr8[0]);
            auto each = [&](auto form) __attribute__((always_inline)) {
#pragma unroll
                for (int qt = 0; qt < 2; ++qt)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[qt][j][e] = form(qt, j, e, s[qt][j][e]);
            };
            if constexpr (CAP) {
                // up to a quarter of the cap a polynomial in the square, up to half of it one of four terms, else c - 2 c / (2^(2 log2 e x / cap) + 1)
                // (less the reference, added in the same instruction)
                auto near = [&](int qt, float y) { const float w = y * y; return fmaf(y, fmaf(w, fmaf(w, pr.tanh_near[2], pr.tanh_near[1]), pr.tanh_near[0]), less[qt]); };
                auto half = [&](int qt, float y) {
                    const float w = y * y;
                    return fmaf(y, fmaf(w, fmaf(w, fmaf(w, pr.tanh_half[3], pr.tanh_half[2]), pr.tanh_half[1]), pr.tanh_half[0]), less[qt]);
                };
                auto any = [&](int qt, float y) { return fmaf(pr.c2_twice, __builtin_amdgcn_rcpf(ex2(y * pr.kappa) + 1.f), pr.c2 + less[qt]); };
                float far = 0.f;
                each([&](int, int, int, float y) { far = fmaxf(far, fabsf(y)); return y; });
                if (__builtin_expect(!__any(far > pr.near), 1)) each([&](int qt, int, int, float y) { return near(qt, y); });
                else if (!__any(far > pr.half)) each([&](int qt, int, int, float y) { return fabsf(y) <= pr.near ? near(qt, y) : half(qt, y); });
                else each([&](int qt, int, int, float y) { return fabsf(y) <= pr.half ? half(qt, y) : any(qt, y); });
            }
            if constexpr (BIAS) {
                const float2 *const at = &lds.bias[row_anew(0)], own[2] = {at[0], at[16]};
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const f32x4 pk = *reinterpret_cast<const f32x4 *>(lds.pos(cur, 32 * kt + 16 * j + 4 * lb));
#pragma unroll
                    for (int qt = 0; qt < 2; ++qt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[qt][j][e] = fmaf(-own[qt].y, fabsf(pk[e] - own[qt].x), s[qt][j][e]);
                }
            }
            if (__builtin_expect(edge, 0)) {
                const int first = key0 + c * KC + 32 * kt - a.T;  // node of the block's first key, below 0: that many rows of the cache first
                uint32_t see[2];                                   // bit 16 j + e: key 16 j + 4 lb + e
#pragma unroll
                for (int qt = 0; qt < 2; ++qt) see[qt] = visible(qt, first) >> (4 * lb);
                each([&](int qt, int j, int e, float y) { return see[qt] & 1u << (16 * j + e) ? y : -INFINITY; });
            }
            if constexpr (CAP || BIAS) lds_issue_tr8<0, 16 * kRowB, 32, 16 * kRowB + 32, 64, 16 * kRowB + 64, 96, 16 * kRowB + 96>(vt, vr8[0]);
            // the weights against the reference as it is (before the first keys: 0), rounded to bf16 for the second product; the row's sum is taken of
            // them as they enter it
            bf16x8 pf[2];
            float ps[2];
            auto weights = [&](auto exponent) __attribute__((always_inline)) {
#pragma unroll
                for (int qt = 0; qt < 2; ++qt) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) pf[qt][4 * j + e] = (bf16_t)ex2(exponent(qt, s[qt][j][e]));
                    ps[qt] = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; e += 2)
                        ps[qt] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pf[qt][e], pf[qt][e + 1]}, bf16x2{(bf16_t)1.f, (bf16_t)1.f}, ps[qt], false);
                }
            };
            auto all_weights = [&]() __attribute__((always_inline)) {
                // A reference far from zero has no place in the instruction that gives an exponent or, with a cap, a score: what is rounded off it there
                // may be a power of two that a sum does not hold.  It is taken off the scores themselves.  (A row of the wave that has not seen a key yet
                // has none to take off: -infinity less itself is NaN.)
                if (__builtin_expect(far_ref, 0)) weights([&](int qt, float x) { return (x - ((CAP ? is_far(ref[qt]) : ref[qt] > -INFINITY) ? ref[qt] : 0.f)) * scale2; });
                else if constexpr (CAP) weights([&](int, float x) { return x; });
                else weights([&](int qt, float x) { return fmaf(x, scale2, BIAS ? ref[qt] == -INFINITY ? 0.f : -ref[qt] * scale2 : less[qt]); });  // (registers)
            };
            all_weights();
            if (__any(fmaxf(ps[0], ps[1]) > kLazySum || fminf(ref[0], ref[1]) == -INFINITY)) {
#pragma unroll
                for (int qt = 0; qt < 2; ++qt) {
                    float t = s[qt][0][0];
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) t = fmaxf(t, s[qt][j][e]);
                    t = quarters_max(t) - (CAP ? less[qt] : 0.f);  // (with a cap the scores have it off them)
                    const bool own = ref[qt] == -INFINITY || quarters_max(ps[qt]) > kLazySum;
                    const float old = ref[qt], now = own ? fmaxf(old, t) : old, corr = old == -INFINITY || now == old ? 1.f : ex2((old - now) * scale2);
                    l_run[qt] *= corr;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) oacc[dt][qt] *= corr;
                    ref[qt] = now;
                    const float add = now == -INFINITY || (CAP && is_far(now)) ? 0.f : -now * scale2;
                    if constexpr (CAP) {
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[qt][j][e] += add - less[qt];
                    }
                    less[qt] = add;
                }
                far_ref = __any(is_far(ref[0]) || is_far(ref[1]));
                all_weights();
            }
            l_run[0] += ps[0];
            l_run[1] += ps[1];
#pragma unroll
            for (int dp = 1; dp < kFours; ++dp)
                lds_issue_tr8<0, 16 * kRowB, 32, 16 * kRowB + 32, 64, 16 * kRowB + 64, 96, 16 * kRowB + 96>(vt + 64 * dp, vr8[dp]);
            if constexpr (kLast) lds_issue_tr4<0, 16 * kRowB, 32, 16 * kRowB + 32>(vt + 64 * kFours, vr4);
            constexpr int kLater = 8 * (kFours - 1) + 2 * kLast;
            auto add = [&](int dt, bf16x8 vf) __attribute__((always_inline)) {
                oacc[dt][0] = mfma16(vf, pf[0], oacc[dt][0]);
                oacc[dt][1] = mfma16(vf, pf[1], oacc[dt][1]);
            };
            __builtin_amdgcn_s_setprio(2);
#pragma unroll
            for (int dp = 0; dp < kFours; ++dp) {
                strd_s16x4(&r)[8] = vr8[dp];
                if (dp == 0 && kLater) lds_settle8_but<kLater>(r);  // LDS reads return in order: the later batch may still travel
                else lds_settle8(r);
#pragma unroll
                for (int dd = 0; dd < 4; ++dd) add(4 * dp + dd, tr_pair(r[2 * dd], r[2 * dd + 1]));
            }
            if constexpr (kLast) {
                lds_settle4(vr4);
                add(DT - 2, tr_pair(vr4[0], vr4[1]));
                add(DT - 1, tr_pair(vr4[2], vr4[3]));
            }
            __builtin_amdgcn_s_setprio(0);
        }
        if (!NC && i + 1 < nchunk) landed(chunk_at(i + 1), cur ^ 1);
        lds_barrier();  // the next chunk has landed, every wave is done with this one
    }
#pragma unroll
    for (int i = 0; i < NF; ++i) odd |= lds.odd()[i] != 0;
    if (__builtin_expect(odd, 0)) {
        // The values left out of the products, for the rows that see them.  A weight is above 0 and a finite factor leaves such a value as it is, so the
        // value itself is added.
#pragma unroll 1
        for (int j = key0 + max(plain, 0) / KC * KC; j < key0 + nkeys; ++j) {
            const bool sees[2] = {j < a.T || (visible(0, j - a.T) & 1), j < a.T || (visible(1, j - a.T) & 1)};
            const bf16_t *const v = (const bf16_t *)(j < a.T ? a.v_cache : a.v_new) + ((size_t)(j < a.T ? j : j - a.T) * a.Hkv + hk) * D + 4 * lb;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const bf16x4 vv = *reinterpret_cast<const bf16x4 *>(v + 16 * dt);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float val = fabsf((float)vv[e]) < INFINITY ? 0.f : (float)vv[e];
#pragma unroll
                    for (int qt = 0; qt < 2; ++qt) oacc[dt][qt][e] += sees[qt] ? val : 0.f;
                }
            }
        }
    }
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
        l_run[qt] += __shfl_xor(l_run[qt], 16, kWave);
        l_run[qt] += __shfl_xor(l_run[qt], 32, kWave);
        const int r = 32 * NW * rb + row_anew(qt);
        if (r < R) {
            const size_t at = (size_t)split * a.m * a.Hq + (size_t)(r / rep) * a.Hq + hk * rep + r % rep;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4 *>(pr.ws.part + at * D + 16 * dt + 4 * lb) = oacc[dt][qt];
            if (lb == 0) {
                pr.ws.ml[2 * at] = fmaxf(ref[qt] * scale2, kTreeNegBig);
                pr.ws.ml[2 * at + 1] = l_run[qt];
            }
        }
    }
}

// Rows of a workgroup, chunk of keys, workgroups per CU: as few waves as hold all rows of a kv head, so that the cache is read once; eight with four more that
// copy (the computing ones have no registers for the copies' addresses: 64 nodes 184 -> 222 us without), or two workgroups to a CU of up to four; a wave
// without a row waits (33 nodes 173 -> 149).  32 heads in 8 of 128 behind 131000 rows, us, against the next larger shape: 32 nodes 128 / 171, 16
// 122 / 124, 8 112 / 116; against the next smaller one and the cache read twice: 33 nodes 149 / 202, 17 126 / 171, 9 120 / 150.
struct Shape {
    int nw, kc, per_cu;
};
Shape shape_of(int R, int d) {
    if (R > 128) return {8, 128, 1};
    if (R > 64) return {4, 64, 2};
    if (R > 32) return {2, 64, 2};
    return {1, 64, 2};
}
int plan(int T, int m, int Hq, int Hkv, int d, Shape &sh, int &row_blocks, int &per) {
    const int R = m * (Hq / Hkv), blocks = ceil_div(T + m, 32);
    sh = shape_of(R, d);
    row_blocks = ceil_div(R, 32 * sh.nw);
    const int want = std::max(1, 256 * sh.per_cu / (row_blocks * Hkv));
    // As many splits as fill the chip, of two blocks at least, of six where their parts would be more than 8 MB, which are written and read again (us, two
    // or three blocks / six: 12751 rows, 52 nodes of 4 heads in 2 25.0 / 19.3; 5000, 16 of 32 in 8 20.6 / 17.9; below: 843, 16 of 32 in 8 12.0 / 14.0)
    per = std::max(ceil_div(blocks, want), std::min(2, blocks));
    if ((size_t)ceil_div(blocks, per) * m * Hq * d * sizeof(float) > 8u << 20) per = std::max(per, 6);
    return ceil_div(blocks, per);
}

template <int D, int NW, int NC, int KC>
int launch(const Params &pr, hipStream_t st) {
    auto go = [&](auto *kernel) {
        const size_t lds = sizeof(Tile<D, NW, NC ? NC : NW, KC>);
        if (!allow_dynamic_lds((const void *)kernel, lds)) return (int)STRD_EHIP;
        kernel<<<xcd_grid(pr.nmain), (NW + NC) * kWave, lds, st>>>(pr);
        return launch_status();
    };
    const bool cap = pr.a.cap > 0.f, bias = pr.a.slopes != nullptr;
    return cap    ? bias ? go(&tree_mfma_kernel<D, NW, NC, KC, true, true>) : go(&tree_mfma_kernel<D, NW, NC, KC, true, false>)
           : bias ? go(&tree_mfma_kernel<D, NW, NC, KC, false, true>)
                  : go(&tree_mfma_kernel<D, NW, NC, KC, false, false>);
}

// Splits of two blocks take them one at a time, the second on its way while the first is worked on (16 nodes behind 843 rows 13.4 -> 12.4 us).
template <int D>
int launch_d(const Params &pr, int nw, hipStream_t st) {
    if (nw == 8) return launch<D, 8, 4, 128>(pr, st);
    if (pr.per <= 2) return nw == 4 ? launch<D, 4, 0, 32>(pr, st) : nw == 2 ? launch<D, 2, 0, 32>(pr, st) : launch<D, 1, 0, 32>(pr, st);
    return nw == 4 ? launch<D, 4, 0, 64>(pr, st) : nw == 2 ? launch<D, 2, 0, 64>(pr, st) : launch<D, 1, 0, 64>(pr, st);
}

}  // namespace

bool tree_mfma_supported(int Hq, int Hkv, int d, strd_dtype io) {
    (void)Hq;
    return io == STRD_BF16 && (d == 64 || d == 96 || d == 128) && Hkv <= 4096;  // a chunk's rows are reached by 32-bit offsets
}

int tree_mfma_splits(int T, int m, int Hq, int Hkv, int d) {
    Shape sh;
    int row_blocks, per;
    return plan(T, m, Hq, Hkv, d, sh, row_blocks, per);
}

int tree_mfma(const TreeCall &a, const TreeWs &ws, hipStream_t st) {
    Params pr;
    Shape sh;
    pr.a = a, pr.ws = ws;
    pr.nsplit = plan(a.T, a.m, a.Hq, a.Hkv, a.d, sh, pr.row_blocks, pr.per);
    pr.nmain = pr.nsplit * a.Hkv * pr.row_blocks;
    pr.scale2 = a.scale * kTreeLog2e;
    pr.kappa = 2.f * kTreeLog2e * a.scale * a.inv_cap;
    pr.c2 = a.cap * kTreeLog2e, pr.c2_twice = -2.f * pr.c2;
    // tanh(y) / y up to y = 0.25 and 0.5, of least relative error (4.0e-7, 5.5e-7); y = ky raw goes into the coefficients.  Where the higher powers'
    // leave fp32's range (a cap far above every score) the polynomials end before they count, where they are too large (a cap far below) the
    // exponential form takes every score.  (As in attn_varlen_mfma.hip.)
    const double near_y[3] = {0.99999960434, -0.33321908205, 0.12841613181}, half_y[4] = {0.999999452, -0.333263082, 0.131902465, -0.0444017053};
    const double ky = (double)a.scale * a.inv_cap;
    pr.half = ky > 1e4 ? -1.f : fminf((float)((ky > 1e-5 ? 0.5 : ky > 1e-9 ? 0.05 : 1e-3) / ky), 1e18f);
    pr.near = 0.5f * pr.half;
    double power = (double)a.scale * kTreeLog2e;
    for (int i = 0; i < 4; ++i, power *= ky * ky) {
        pr.tanh_half[i] = (float)(half_y[i] * power);
        if (i < 3) pr.tanh_near[i] = (float)(near_y[i] * power);
    }
    return a.d == 128 ? launch_d<128>(pr, sh.nw, st) : a.d == 96 ? launch_d<96>(pr, sh.nw, st) : launch_d<64>(pr, sh.nw, st);
}

}  // namespace strd
