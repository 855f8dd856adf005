// ssd_prefill_varlen on bf16 matrix cores: the Mamba-2 recurrence (paper Eqs. "ssm_state_update", "ssm_output") over a packed batch of sequences,
// each from a state of its own, with final states that count as fp32.
//
// The walk is that of ssd_quad_mfma.hip -- four whole heads (P = 64) of one group per workgroup, 32-token steps, products (a) to (e), waves and tiles --
// over one segment of one sequence.  What differs:
//  * States first.  A kernel before the walk makes what each segment leaves in the state behind it, another the states at the segments' starts, and the
//    walk sets out from those: every output is added up in fp32 and rounded once, and no segment waits for another.  (A walk from a zero state whose outputs
//    are completed later reads and rounds most outputs twice where heads remember for long.)  The same sums are the final states, fp32 numbers.
//  * w x in pieces.  S += b^T (w x) has exact bf16 numbers b and x, but w = dt 2^(decay to the end) has 24 bits.  w x goes into the product as bf16 numbers, each
//    the rest of those before it: three for the states, two in the walk, whose outputs then pass two roundings to bf16 on any way (of a weight or of
//    the state, and their own).  One, and three roundings of what passes through the state, where all four heads forget within every step of the segment:
//    there that is a few tokens' part of an output.
//  * States in units.  Where heads remember a state decays by its unit, which the weights of tokens and the factors of outputs take in; it is multiplied only
//    where the unit has gone 2^48 away: 64 multiplications of a wave and step less (33280 tokens of slow heads 353 -> 293 us; where heads forget within a
//    step it would be multiplied as often, and not between the products: 277 -> 334).
//
// 33280 tokens of 128 heads of 64 x 128 in three sequences, a quarter of the heads slow: decays 15 us, parts 88-104, states before segments 25, walk 260-300, final
// states 14, 391 us among calls (350 TFLOP/s, 3.2 TB/s); 3493 tokens in six 87.  The walk is bound by the products (33 % of a SIMD's time) and vector
// instructions (44 %) of two compute waves, one after the other, at 1.8 GHz, the parts by the same where heads remember (32 and 42 %).
//
// Values that are not finite are never forgotten: a segment that ends with one in a channel says so, and the last kernel writes NaN to that channel's later
// outputs and final state, whatever the decays.
#include <algorithm>
#include <functional>

#include "carry.h"
#include "ssd_quad.h"

namespace strd {
namespace {

constexpr float kGone = -150.f;     // log2 of a decay that leaves nothing in fp32
constexpr float kApart = 48.f;      // log2 of how far a state's unit may be from 1
constexpr float kForgets = -12.f;  // log2 of the decay over every step of a segment from which on w x is taken in one piece

struct PackArgs {
    const bf16_t *x;
    const float *dt, *A;
    const bf16_t *B, *C;
    const float *D, *S_in;
    bf16_t *y;
    float *S_out;
    float *init;      // [segments of sequences with several, H, P, n]: the state before a segment (the first one's is not used)
    float *ends;      // [parts, H, P, n]: what parts of segments leave in the states behind the segments
    uint32_t *alive;  // [parts, H / 4]: whether a part has left anything
    float *total;     // [segments, H]: log2 decay over a segment
    float *decay;     // [steps, H]: log2 decay over a step
    float *weight;    // [steps, H, 32]: dt 2^(decay from the token to its step's end), in slot order
    uint32_t *lost;   // [segments, H, 2]: channels that end with a value that is not finite
    int H, G, wg;     // wg = H / 4
    // Sequences, those with several segments first: rows, slot of the pools, steps per segment (the last one: what is left), segments before, the first one in
    // `init`, parts before, steps of all segments before.
    int row0[kMaxSeqs], len[kMaxSeqs], slot[kMaxSeqs], steps[kMaxSeqs], base[kMaxSeqs + 1], first[kMaxSeqs], parts[kMaxSeqs + 1], step0[kMaxSeqs + 1];
    // The order of launches: all segments of full length (full[s] before those of sequence s), then what is left of sequences, by falling length.
    int full[kMaxSeqs + 1];
    unsigned char rest[kMaxSeqs];
    unsigned long long fresh;
    int nseq, nmulti, part_steps;
    // Sequence and segment of a workgroup's rank: the ranks are dealt to the XCDs forth and back.
    __device__ __forceinline__ bool segment_of(int round, int xcd, int &s, int &seg) const {
        const int rank = round * kXcd + (round & 1 ? kXcd - 1 - xcd : xcd), left = rank - full[nseq];
        if (rank >= base[nseq]) return false;
        s = 0;
        if (left >= 0) {
            s = rest[left], seg = count(s) - 1;
        } else {
            while (s + 1 < nseq && rank >= full[s + 1]) ++s;  // uniform
            seg = rank - full[s];
        }
        return true;
    }
    __device__ __forceinline__ int count(int s) const { return base[s + 1] - base[s]; }
    __device__ __forceinline__ int parts_of(int s) const { return (steps[s] + part_steps - 1) / part_steps; }  // of a segment
};

template <int NS>
struct LdsP : LdsQ<NS> {
    int remembers[kThreads / 64];  // per wave, whether it has seen a step beyond which a head remembers
    float anew[3][kHeads];         // what a state is multiplied by in a step for its new unit, or 1
};
static_assert(sizeof(LdsP<128>) <= 160 * 1024, "one workgroup must fit the 160 KB of LDS of a CU");

// ---- compute wave: slab cw (32 channels) of head hh of the workgroup: (d), (c), (e), the outputs ----
template <int NS, bool MORE>
__device__ __forceinline__ void compute_wave(LdsP<NS> &lds, const PackArgs &a, int hh, int cw, int h, int row0, int row_end, int nloc,
                                             const float *s_src, uint32_t *lost) {
    using L = LdsP<NS>;
    constexpr int KS = NS / 32;  // k-steps of the products contracted over n
    constexpr int NT = NS / 16;  // 16-row tiles of the state
    const int lane = threadIdx.x & 63, lr = lane & 15, lb = lane >> 4;

    // state: S^T[n][p] tiles, rows n = 16 nt + 4 lb + i, columns p = chan_of(cw, pt, lr)
    f32x4 sacc[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int pt = 0; pt < 2; ++pt) {
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
            if (s_src) v = *reinterpret_cast<const f32x4 *>(s_src + ((size_t)h * kP + chan_of(cw, pt, lr)) * NS + 16 * nt + 4 * lb);
            sacc[nt][pt] = v;
        }
    const uint32_t HP = (uint32_t)a.H * kP;
    // Places of this lane in the tiles (bytes): 8 channels of x and 4 columns of b of the row it passes to the transposing reads of a 16-token
    // block, in even and in odd tiles of the state; the first and second 8-byte piece of a k-step of its own row of c.
    using TB = typename L::TB;
    using TX = typename L::TX;
    const int trow = state_tok(lb, lr >> 2), q4 = lr & 3;
    const int x_at = TX::row_at(trow) + 2 * (kP * hh + 32 * cw + 8 * q4);
    const int b_at = TB::row_at(trow) + 16 * ((q4 >> 1) ^ (trow & 3)) + 8 * (q4 & 1);  // odd tiles: ^ 32
    const int c_at = TB::row_at(lr) + 16 * ((lb >> 1) ^ (lr & 3)) + 8 * (lb & 1);      // second piece: ^ 32
    // this lane's 8 channels of its token in the first rows of a step's outputs (elements)
    const uint32_t y_at = lr * HP + (uint32_t)(h * kP + 32 * cw + 8 * lb);
    bf16_t *yp = a.y + (size_t)row0 * HP;  // uniform

    strd_s16x4 cr[2][2 * KS];  // c pieces of a step's two query blocks, requested a step ahead (as are the tiles, for the G waves)
    using First = std::integral_constant<int, 0>;
    using Second = std::integral_constant<int, 1>;
    auto request_c = [&](int i, auto tt) __attribute__((always_inline)) {
        const uint32_t ct = lds_offset(lds.c[i % kRB].v) + c_at;
        issue_c_pieces<KS, tt.value * TB::kBlock>(ct, ct ^ 32, cr[tt.value]);
    };
    lds_barrier();
    lds_barrier();  // first copies landed, scans of steps 0 and 1 |
    request_c(0, First());
    request_c(0, Second());
    lds_barrier();  // weights of step 0

    for (int i = 0; i < nloc; ++i) {
        settle_c_pieces<KS>(cr[0]);  // (the barrier before has waited for them)
        settle_c_pieces<KS>(cr[1]);
        const typename L::Scan &sc = lds.scan[i % 3][hh];
        const uint32_t bt = lds_offset(lds.b[i % kRB].v) + b_at;
        // Everything that (d), (c) and the weights of (e) need is requested at the start of the step.
        strd_s16x4 xr[4];
        lds_issue_tr4<0, TX::kBlock, 8, TX::kBlock + 8>(lds.x[i % kRX].v + x_at, xr);
        const float anew = read_lane_f32(lds.anew[i % 3][hh], 0);
        const f32x4 w0 = *reinterpret_cast<const f32x4 *>(&sc.w[8 * lb]), w1 = *reinterpret_cast<const f32x4 *>(&sc.w[8 * lb + 4]);
        const float cr0 = sc.carry[lr], cr1 = sc.carry[16 + lr];
        __builtin_amdgcn_sched_barrier(0);
        // (d): Y^T[p, t] = sum_n S[p, n] c_t[n].  A operand straight from the accumulators: the lane holds rows
        // 4 lb .. 4 lb + 3 of state tiles 2 ks and 2 ks + 1 for column p = lr, i.e. the k slots n = 32 ks + 4 lb + s (s < 4),
        // 32 ks + 16 + 4 lb + s - 4 (s >= 4); the c fragments are read in the same slot order (two 8-byte reads).
        // The vector work of a step is dealt out between its products, four or five instructions to each: the state's conversion and the
        // weights of x here, the state's decay in (e).
        f32x4 yacc[2][2];  // [query block][tile]
        bf16x8 xf[2], xwf[2];
        auto decay = [&](int nt, int pt) __attribute__((always_inline)) {
            if constexpr (!MORE) sacc[nt][pt] *= anew;
        };
        auto half = [&](int ks, int pt, int hi) __attribute__((always_inline)) { return to_bf16x4(sacc[2 * ks + hi][pt]); };
        bf16x4 sb[2][2][2];  // [ks % 2][tile][half]: the state's fragments of this k-step and the next
#pragma unroll
        for (int pt = 0; pt < 2; ++pt)
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) sb[0][pt][hi] = half(0, pt, hi);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int tt = j >> 1, pt = j & 1;
                yacc[tt][pt] = mfma16(cat8(sb[ks & 1][pt][0], sb[ks & 1][pt][1]), tr_pair(cr[tt][2 * ks], cr[tt][2 * ks + 1]), ks ? yacc[tt][pt] : f32x4{0.f, 0.f, 0.f, 0.f});
                if (ks + 1 < KS) sb[(ks + 1) & 1][pt][tt] = half(ks + 1, pt, tt);
                if (ks == 0) {
                    decay(tt, pt);
                } else {
                    // a twelfth (n = 64: a quarter) of the weights of x
                    constexpr int kSlots = 4 * (KS - 1);
                    const int from = 16 * (4 * (ks - 1) + j) / kSlots, to = 16 * (4 * (ks - 1) + j + 1) / kSlots;
#pragma unroll
                    for (int e = from; e < to; ++e) xwf[e >> 3][e & 7] = (bf16_t)((float)xf[e >> 3][e & 7] * ((e & 7) < 4 ? w0[e & 3] : w1[e & 3]));
                }
                if (ks == 0 && j == 3) {
                    // x fragments: A operand of (c) as they are, B operand of (e) once weighted
                    __builtin_amdgcn_s_waitcnt(lgkm_wait_imm(0));  // (in the compiler's books, too: a wait of its own later on would count the b fragments)
                    lds_settle4(xr);
                    xf[0] = tr_pair(xr[0], xr[1]);
                    xf[1] = tr_pair(xr[2], xr[3]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        strd_s16x4 ba[8], bb[8], m0;
        i32x4 m1;
        asm volatile("ds_read_b64 %0, %2\n\tds_read_b128 %1, %3"
                     : "=&v"(m0), "=&v"(m1) : "v"(lds_offset(&lds.m0[i & 1][hh][lane])), "v"(lds_offset(&lds.m1[i & 1][hh][lane])) : "memory");
        issue_b_frags<0, TB::kBlock>(bt, bt ^ 32, ba);
        if constexpr (NT == 8 && !MORE) issue_b_frags<128, TB::kBlock>(bt, bt ^ 32, bb);
        // (c) on top of the carried part
#pragma unroll
        for (int pt = 0; pt < 2; ++pt) {
            yacc[0][pt] *= cr0;
            yacc[1][pt] *= cr1;
        }
        asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(m0), "+v"(m1) : "i"(NT == 8 && !MORE ? 15 : 8) : "memory");  // the b fragments after them may be on their way
#pragma unroll
        for (int pt = 0; pt < 2; ++pt) {
            yacc[0][pt] = mfma16(xf[pt], cat8(__builtin_bit_cast(bf16x4, m0), bf16x4{}), yacc[0][pt]);
            yacc[1][pt] = mfma16(xf[pt], __builtin_bit_cast(bf16x8, m1), yacc[1][pt]);
        }
        bf16x8 out[2];
        auto round = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) out[tt] = cat8(to_bf16x4(yacc[tt][0]), to_bf16x4(yacc[tt][1]));
        };
        if constexpr (MORE) round();
        // (e): S^T = 2^(l_Q) S^T + b^T (w x), w x in as many pieces as the step is worth.  With several pieces the state decays by its unit.
        if (MORE && anew != 1.f) {  // uniform
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sacc[nt][0] *= anew, sacc[nt][1] *= anew;
        }
        bf16x8 mid[2];
        if constexpr (MORE) {
            // (read again: eight registers less in between)
            const f32x4 v0 = *reinterpret_cast<const f32x4 *>(&sc.w[8 * lb]), v1 = *reinterpret_cast<const f32x4 *>(&sc.w[8 * lb + 4]);
#pragma unroll
            for (int pt = 0; pt < 2; ++pt)
#pragma unroll
                for (int e = 0; e < 8; ++e) mid[pt][e] = (bf16_t)fmaf((float)xf[pt][e], e < 4 ? v0[e & 3] : v1[e & 3], -(float)xwf[pt][e]);
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (NT == 8) {
            if constexpr (MORE) issue_b_frags<128, TB::kBlock>(bt, bt ^ 32, bb);
            lds_settle8_but<8>(ba);
        } else {
            lds_settle8(ba);
            if constexpr (!MORE) request_c(i + 1, Second());
        }
        // the c pieces of the next step (the last step reads a tile that was never requested, into registers that nobody uses)
        if constexpr (!MORE) request_c(i + 1, First());
#pragma unroll
        for (int d = 0; d < 4; ++d) {
#pragma unroll
            for (int pt = 0; pt < 2; ++pt) sacc[d][pt] = mfma16(tr_pair(ba[2 * d], ba[2 * d + 1]), xwf[pt], sacc[d][pt]);
            if (d + 2 < NT) decay(d + 2, 0), decay(d + 2, 1);
        }
        if constexpr (!MORE) eight_products_with_vector_work();
        __builtin_amdgcn_sched_barrier(0);
        auto add = [&](const strd_s16x4 (&b)[8], int d0, const bf16x8 (&piece)[2]) __attribute__((always_inline)) {
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int pt = 0; pt < 2; ++pt) sacc[(d0 + d) % NT][pt] = mfma16(tr_pair(b[2 * d], b[2 * d + 1]), piece[pt], sacc[(d0 + d) % NT][pt]);
        };
        if constexpr (MORE) {
            add(ba, 0, mid);
            request_c(i + 1, First());
        }
        if constexpr (NT == 8) {
            lds_settle8_but<2 * KS>(bb);
            if constexpr (!MORE) request_c(i + 1, Second());
#pragma unroll
            for (int d = 4; d < 8; ++d) {
#pragma unroll
                for (int pt = 0; pt < 2; ++pt)
                    sacc[d % NT][pt] = mfma16(tr_pair(bb[2 * (d - 4)], bb[2 * (d - 4) + 1]), xwf[pt], sacc[d % NT][pt]);
                if (d + 2 < NT) decay(d + 2, 0), decay(d + 2, 1);
            }
            if constexpr (!MORE) eight_products_with_vector_work();
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (MORE) add(bb, 4, mid);
        }
        if constexpr (MORE) request_c(i + 1, Second());
        else round();
        // outputs: 16 bytes of this lane's token
        const int left = row_end - (row0 + i * kQ);  // uniform: tokens from the step's first to the segment's end
        if (left >= kQ) {
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) *reinterpret_cast<bf16x8 *>(yp + (size_t)16 * tt * HP + y_at) = out[tt];
        } else {
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
                if (lr + 16 * tt < left) *reinterpret_cast<bf16x8 *>(yp + (size_t)16 * tt * HP + y_at) = out[tt];
        }
        yp += (size_t)kQ * HP;
        lds_barrier();  // the step is over
    }

    if (lost) {  // which channels of the slab hold a value that is not finite: bit lr + 16 pt
        uint32_t bits = 0;
#pragma unroll
        for (int pt = 0; pt < 2; ++pt) {
            bool odd = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) odd |= !(__builtin_fabsf(sacc[nt][pt][e]) < __builtin_inff());
            unsigned long long any = __ballot(odd);
            any |= any >> 32;
            any |= any >> 16;
            bits |= (uint32_t)(any & 0xFFFF) << (16 * pt);
        }
        if (lane == 0) lost[2 * h + cw] = bits;
    }
}

// ---- helper wave: dt copies, the scans of the workgroup's heads (two at a time, lane = 32 * (head % 2) + token) ----
template <int NS>
__device__ __forceinline__ void helper_wave(LdsP<NS> &lds, const PackArgs &a, int h0, int row0, int row_end, int nloc, bool units) {
    using L = LdsP<NS>;
    const int lane = threadIdx.x & 63, half = lane >> 5, j = lane & 31;
    float Al2[2], unit[2] = {0.f, 0.f};  // log2 of the units that the states are in
#pragma unroll
    for (int k = 0; k < 2; ++k) Al2[k] = a.A[h0 + 2 * k + half] * kLog2e;
    __builtin_amdgcn_s_setprio(3);
    auto request_dt = [&](int i) __attribute__((always_inline)) {  // 64 lanes x 4 bytes per pair; rows past the end re-read the last row
        const size_t row = min(row0 + i * kQ + j, row_end - 1);
#pragma unroll
        for (int k = 0; k < 2; ++k)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(a.dt + row * a.H + (h0 + 2 * k + half)),
                                             (__attribute__((address_space(3))) void *)lds.dt[i % kRD][k], 4, 0, 0);
    };
    auto make_scan = [&](int k, int i, float raw) __attribute__((always_inline)) {
        const float dv = row0 + i * kQ + j < row_end ? raw : 0.f;
        float inc = step_decay(dv * Al2[k]);  // inclusive prefix sum over the 32 lanes of a head
#define STRD_DPP_FADD(ctrl, row_mask) \
    inc += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, inc), ctrl, row_mask, 0xF, true))
        STRD_DPP_FADD(0x111, 0xF);  // row_shr:1
        STRD_DPP_FADD(0x112, 0xF);  // row_shr:2
        STRD_DPP_FADD(0x114, 0xF);  // row_shr:4
        STRD_DPP_FADD(0x118, 0xF);  // row_shr:8
        STRD_DPP_FADD(0x142, 0xA);  // row_bcast:15 into rows 1 and 3
#undef STRD_DPP_FADD
        typename L::Scan &m = lds.scan[i % 3][2 * k + half];
        const float tot = half ? read_lane_f32(inc, 63) : read_lane_f32(inc, 31);
        const float l15 = half ? read_lane_f32(inc, 47) : read_lane_f32(inc, 15);
        m.ell[j] = inc;
        m.dtv[j] = dv;
        const float from = inc + unit[k], after = unit[k] + tot;
        const bool anew = !(units && __builtin_fabsf(after) <= kApart);
        m.w[slot_of(j)] = dv * fast_exp2(anew ? tot - inc : -from);
        m.carry[j] = fast_exp2(from);
        if (j == 0) lds.anew[i % 3][2 * k + half] = anew ? fast_exp2(after) : 1.f;
        unit[k] = anew ? 0.f : after;
        if (j < 16) m.fw[j] = dv * fast_exp2(l15 - inc);  // the exponent is <= 0 for these
    };
    constexpr int kNewest = 2;  // copies requested per step

    lds_barrier();
#pragma unroll
    for (int i = 0; i < kRD; ++i)
        if (i < nloc) request_dt(i);
    async_tile_wait();
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (i < nloc) {
#pragma unroll
            for (int k = 0; k < 2; ++k) make_scan(k, i, lds.dt[i][k][lane]);
        }
    lds_barrier();  // first copies landed, scans of steps 0 and 1
    lds_barrier();
    for (int i = 0; i < nloc; ++i) {
        // dt of step i + 2 landed before the barrier that ended the previous step (or in the prologue)
        float raw[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) raw[k] = lds.dt[(i + 2) % kRD][k][lane];
        __builtin_amdgcn_sched_barrier(0);
        const bool more = i + 4 < nloc;  // uniform; nothing past the segment is requested
        if (more) request_dt(i + 4);     // slot last read in step i - 2
        if (i + 2 < nloc) {              // slot last read in step i - 1
#pragma unroll
            for (int k = 0; k < 2; ++k) make_scan(k, i + 2, raw[k]);
        }
        if (more)
            __builtin_amdgcn_s_waitcnt(vm_wait_imm(kNewest));  // everything requested in earlier steps has landed
        else
            async_tile_wait();
        lds_barrier();
    }
}

// ---- copy wave: the B, C and x tiles three steps ahead of the compute waves (B and C two ahead of the G waves) ----
template <int NS>
__device__ __forceinline__ void copy_wave(LdsP<NS> &lds, const PackArgs &a, int g, int h0, int row0, int row_end, int nloc) {
    using L = LdsP<NS>;
    using TB = typename L::TB;
    using TX = typename L::TX;
    const int lane = threadIdx.x & 63;
    __builtin_amdgcn_s_setprio(3);
    const uint32_t x_row = (uint32_t)a.H * kP * 2, bc_row = (uint32_t)a.G * NS * 2;
    const char *xs = reinterpret_cast<const char *>(a.x) + (size_t)h0 * kP * 2;
    const char *bs = reinterpret_cast<const char *>(a.B) + (size_t)g * NS * 2, *cs = reinterpret_cast<const char *>(a.C) + (size_t)g * NS * 2;
    // The row this lane copies from with its first instruction of a tile, and where in the row; the k-th one is k * kRows rows on.
    const int xr0 = lane / (64 / TX::kRows), br0 = lane / (64 / TB::kRows);
    const uint32_t xc = lane % (64 / TX::kRows) * 16, bc = ((lane % (64 / TB::kRows)) ^ (br0 & 3)) * 16;
    uint32_t xo[TX::kIssues], bo[TB::kIssues];  // byte offsets inside the rows of a step, which are a uniform pointer
#pragma unroll
    for (int k = 0; k < TX::kIssues; ++k) xo[k] = (xr0 + k * TX::kRows) * x_row + xc;
#pragma unroll
    for (int k = 0; k < TB::kIssues; ++k) bo[k] = (br0 + k * TB::kRows) * bc_row + bc;
    auto stream = [&](auto *tile, const char *src, uint32_t row_bytes, const uint32_t *off, int r0, uint32_t col, int i) __attribute__((always_inline)) {
        using TT = typename std::remove_pointer<decltype(tile)>::type;
        const int t0 = row0 + i * kQ;
        if (t0 + kQ <= row_end) {  // uniform: every row of the step exists
            const char *base = src + (size_t)t0 * row_bytes;
#pragma unroll
            for (int k = 0; k < TT::kIssues; ++k) copy16(base + off[k], tile->v + 1088 * k);
        } else {  // past the end: the last row again
#pragma unroll
            for (int k = 0; k < TT::kIssues; ++k) {
                const uint32_t row = (uint32_t)min(t0 + r0 + k * TT::kRows, row_end - 1);
                copy16(src + (size_t)row * row_bytes + col, tile->v + 1088 * k);
            }
        }
    };
    auto request_x = [&](int i) __attribute__((always_inline)) { stream(&lds.x[i % kRX], xs, x_row, xo, xr0, xc, i); };
    auto request_bc = [&](int i) __attribute__((always_inline)) {
        stream(&lds.b[i % kRB], bs, bc_row, bo, br0, bc, i);
        stream(&lds.c[i % kRB], cs, bc_row, bo, br0, bc, i);
    };
    constexpr int kX = TX::kIssues, kBC = 2 * TB::kIssues;
    constexpr int kAll = 3 * kX + 2 * kBC;
    static_assert(2 * kX + kBC < 64, "vmcnt has 6 bits");

    lds_barrier();
    request_bc(0);
    request_x(0);
    if (nloc > 1) request_bc(1);
    if (nloc > 1) request_x(1);
    if (nloc > 2) request_bc(2);
    if (nloc > 2) request_x(2);
    if (nloc > 2)
        __builtin_amdgcn_s_waitcnt(vm_wait_imm(kAll < 63 ? kAll : 63));  // b and c of step 0
    else
        async_tile_wait();
    lds_barrier();
    if (nloc > 2) __builtin_amdgcn_s_waitcnt(vm_wait_imm(2 * kX + kBC));  // x of step 0, b and c of step 1
    lds_barrier();

    for (int i = 0; i < nloc; ++i) {
        // At the end of step i there are x of step i + 1 and b and c of step i + 2: of what was requested later, x of steps i + 2 and
        // i + 3 and b and c of step i + 3 may still be on their way (b and c of step i + 2 were requested before x of step i + 2).
        if (i + 3 < nloc) {                   // slots last read in step i - 1
            request_bc(i + 3);
            request_x(i + 3);
            __builtin_amdgcn_s_waitcnt(vm_wait_imm(2 * kX + kBC));
        } else if (i + 2 < nloc) {
            __builtin_amdgcn_s_waitcnt(vm_wait_imm(kX));
        } else {
            async_tile_wait();
        }
        lds_barrier();  // publishes it; the copies stay in flight
    }
}

template <int NS>
__global__ __launch_bounds__(kThreads) void ssd_packed_kernel(PackArgs a) {
    using L = LdsP<NS>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
    L &lds = *reinterpret_cast<L *>(smem_raw);
    // The heads of a segment, which share tiles of B and C, on one XCD.
    const int place = blockIdx.x / kXcd, h0 = place % a.wg * kHeads, g = h0 / (a.H / a.G);
    int s, seg;
    if (!a.segment_of(place / a.wg, blockIdx.x % kXcd, s, seg)) return;
    const int useg = a.base[s] + seg;
    const int row0 = a.row0[s] + seg * a.steps[s] * kQ, row_end = min(a.row0[s] + a.len[s], row0 + a.steps[s] * kQ), nloc = (row_end - row0 + kQ - 1) / kQ;
    const size_t state = (size_t)a.H * kP * NS;
    const float *s_src = seg ? a.init + (size_t)(a.first[s] + seg) * state : a.S_in && !(a.fresh >> s & 1) ? a.S_in + (size_t)a.slot[s] * state : nullptr;
    uint32_t *lost = a.lost + (size_t)useg * a.H * 2;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    // Whether some head remembers beyond some step (other than the last, whose state nothing reads: resets on the way do not speak for the rest).
    bool mine = false;
    for (int i = (int)threadIdx.x; i + 1 < nloc; i += kThreads) {
        const f32x4 d = *reinterpret_cast<const f32x4 *>(a.decay + (size_t)(a.step0[s] + seg * a.steps[s] + i) * a.H + h0);
#pragma unroll
        for (int k = 0; k < kHeads; ++k) mine |= !(d[k] <= kForgets);
    }
    mine = __any(mine);
    if ((threadIdx.x & 63) == 0) lds.remembers[wave] = mine;
    lds_barrier();
    bool more = false;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) more |= lds.remembers[w] != 0;
    more = __builtin_amdgcn_readfirstlane(more);
    // Wave i runs on SIMD i % 4: every SIMD has two compute waves and one of the others.
    if (wave < 8 && more)
        compute_wave<NS, true>(lds, a, wave >> 1, wave & 1, h0 + (wave >> 1), row0, row_end, nloc, s_src, lost);
    else if (wave < 8)
        compute_wave<NS, false>(lds, a, wave >> 1, wave & 1, h0 + (wave >> 1), row0, row_end, nloc, s_src, lost);
    else if (wave < 10)
        g_wave<NS>(lds, a.D, wave - 8, h0, nloc);
    else if (wave == 10)
        copy_wave<NS>(lds, a, g, h0, row0, row_end, nloc);
    else
        helper_wave<NS>(lds, a, h0, row0, row_end, nloc, more);
}

// ---- decays over steps, and the weights of their tokens: a workgroup per step and 64 heads -----------------------------------------------------------
// Sums of decays that a weight takes are added up from the step's end, so that those that count are not differences of large ones.
__global__ __launch_bounds__(256) void ssd_packed_steps_kernel(PackArgs a) {
    constexpr int kRow = 33;
    __shared__ float dt[kQ][64 + 1], w[64][kRow], part[4][64];
    const int step = blockIdx.x, hb = blockIdx.y * 64, tid = threadIdx.x, h = tid & 63, q = tid >> 6;  // q: 8 tokens of the step
    int s = 0;
    while (s + 1 < a.nseq && step >= a.step0[s + 1]) ++s;  // uniform
    const int row0 = a.row0[s] + (step - a.step0[s]) * kQ, rows = min(kQ, a.row0[s] + a.len[s] - row0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int t = 4 * i + q;
        dt[t][h] = t < rows && hb + h < a.H ? a.dt[(size_t)(row0 + t) * a.H + hb + h] : 0.f;
    }
    const float Al2 = hb + h < a.H ? a.A[hb + h] * kLog2e : 0.f;
    __syncthreads();
    float d[8], behind[8], run = 0.f;
#pragma unroll
    for (int e = 7; e >= 0; --e) {
        d[e] = dt[8 * q + e][h];
        behind[e] = run;
        run += d[e] * Al2;
    }
    part[q][h] = run;
    __syncthreads();
    float after = 0.f;
    for (int i = 3; i > q; --i) after += part[i][h];
    if (q == 0 && hb + h < a.H) a.decay[(size_t)step * a.H + hb + h] = after + run;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[h][slot_of(8 * q + e)] = d[e] == 0.f ? 0.f : d[e] * fast_exp2(after + behind[e]);
    __syncthreads();
    for (int i = tid; i < 64 * kQ; i += 256)
        if (hb + i / kQ < a.H) a.weight[((size_t)step * a.H + hb) * kQ + i] = w[i / kQ][i % kQ];
}

// ---- what a part of a segment leaves in the state behind the segment:  sum_j (dt_j 2^(decay from j to the segment's end) x_j) b_j^T -----------------
// A workgroup per (part, four heads): 8 waves as the walk's compute waves, every one requesting a share of the tiles; from the part's last step to the first
// whose weights are not all zero.  A part whose decay up to the segment's end leaves nothing says so and ends.  w x goes into the product in three pieces
// where the sequence ends less than 2^-10 of a decay, or less than 64 steps behind the segment, further on, else in two: what two leave out is 2^-17 of it.
constexpr int kEndThreads = 512, kRE = 3, kMostPart = 64;
template <int NS>
struct LdsE {
    using TB = typename LdsQ<NS>::TB;
    using TX = typename LdsQ<NS>::TX;
    float sums[kEndThreads / 64][kHeads];
    float f[kMostPart][kHeads];  // decay from a step's end to the segment's; negative: three pieces
    int first[kHeads];
    alignas(16) float w[kRE][kHeads * kQ];
    TB b[kRE];
    TX x[kRE];
};

static_assert(2 * sizeof(LdsE<128>) <= 160 * 1024, "two workgroups must fit the 160 KB of LDS of a CU");

template <int NS>
__global__ __launch_bounds__(kEndThreads) __attribute__((amdgpu_waves_per_eu(4, 4))) void ssd_packed_ends_kernel(PackArgs a) {
    using L = LdsE<NS>;
    using TB = typename L::TB;
    using TX = typename L::TX;
    constexpr int NT = NS / 16;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
    L &lds = *reinterpret_cast<L *>(smem_raw);
    // The heads of a segment on one XCD; every segment's last parts first, which are those that count where heads forget.
    const int place = blockIdx.x / kXcd, quad = place % a.wg, h0 = quad * kHeads, g = h0 / (a.H / a.G);
    int s, seg;
    if (!a.segment_of(place / a.wg, blockIdx.x % kXcd, s, seg)) return;
    const int useg = a.base[s] + seg, per = a.parts_of(s), rank = blockIdx.y;
    if (rank >= per) return;
    const int all = (a.len[s] + kQ - 1) / kQ, seg_stop = min(all, (seg + 1) * a.steps[s]), here = (seg_stop - seg * a.steps[s] + a.part_steps - 1) / a.part_steps;
    const int u = rank < here ? here - 1 - rank : rank, upart = a.parts[s] + seg * per + u, begin0 = seg * a.steps[s] + u * a.part_steps;  // steps of the sequence
    const int nloc = min(seg_stop - begin0, a.part_steps), row0 = a.row0[s] + begin0 * kQ, row_end = a.row0[s] + a.len[s];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float *const decay = a.decay + (size_t)a.step0[s] * a.H + h0;  // of step i: + i H
    if (nloc <= 0) {  // (a sequence's last segment is shorter)
        if (tid == 0) a.alive[(size_t)upart * a.wg + quad] = 0;
        return;
    }
    // A share of the tiles of step i: 1 KB per instruction, B's pieces permuted as in the walk's tiles; rows behind the end: the last one, of weight 0.
    constexpr int kX = TX::kIssues / 8;  // (and one of B, with n = 64 of four waves)
    auto request = [&](int i) __attribute__((always_inline)) {
        const int r0 = row0 + i * kQ;
#pragma unroll
        for (int q = 0; q < kX; ++q) {
            const int k = kX * wave + q, row = min(r0 + k * TX::kRows + lane / (64 / TX::kRows), row_end - 1);
            copy16(reinterpret_cast<const char *>(a.x + ((size_t)row * a.H + h0) * kP) + lane % (64 / TX::kRows) * 16, lds.x[i % kRE].v + 1088 * k);
        }
        if (wave < TB::kIssues) {
            const int in_tile = lane / (64 / TB::kRows), row = min(r0 + wave * TB::kRows + in_tile, row_end - 1);
            copy16(reinterpret_cast<const char *>(a.B + ((size_t)row * a.G + g) * NS) + ((lane % (64 / TB::kRows)) ^ (in_tile & 3)) * 16,
                   lds.b[i % kRE].v + 1088 * wave);
        }
        if (wave >= 6)  // the weights of four heads are 512 bytes
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(a.weight + ((size_t)(a.step0[s] + begin0 + i) * a.H + h0) * kQ + 64 * (wave - 6) + lane),
                                             (__attribute__((address_space(3))) void *)(lds.w[i % kRE] + 64 * (wave - 6)), 4, 0, 0);
    };
    auto landed = [&](bool later) __attribute__((always_inline)) {  // all copies, or (later) all but those of the step requested last
        const int copies = kX + (wave < TB::kIssues) + (wave >= 6);  // uniform
        if (!later) async_tile_wait();
        else if (copies == 4) __builtin_amdgcn_s_waitcnt(vm_wait_imm(4));
        else if (copies == 3) __builtin_amdgcn_s_waitcnt(vm_wait_imm(3));
        else __builtin_amdgcn_s_waitcnt(vm_wait_imm(2));
    };
    static_assert(kX == 2 && TB::kIssues <= 8, "two to four copies of a wave and step");
    // decay from the part's end to the segment's, until nothing is left of any head
    float behind[kHeads] = {};
    bool gone = false;
    for (int i0 = begin0 + nloc; i0 < seg_stop && !gone; i0 += kEndThreads) {
        f32x4 d = {0.f, 0.f, 0.f, 0.f};
        if (i0 + tid < seg_stop) d = *reinterpret_cast<const f32x4 *>(decay + (size_t)(i0 + tid) * a.H);
#pragma unroll
        for (int k = 0; k < kHeads; ++k) {
            const float sum = wave_inclusive_scan_f32(d[k]);
            if (lane == 63) lds.sums[wave][k] = sum;
        }
        lds_barrier();
        gone = true;
#pragma unroll
        for (int k = 0; k < kHeads; ++k) {
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < kEndThreads / 64; ++w) sum += lds.sums[w][k];
            behind[k] += sum;
            gone &= behind[k] <= kGone;  // (NaN is never gone)
        }
        lds_barrier();
    }
    if (tid == 0) a.alive[(size_t)upart * a.wg + quad] = !gone;
    if (gone) {
        if (u == 0 && tid < kHeads) a.total[(size_t)useg * a.H + h0 + tid] = kGone;
        return;
    }
    request(nloc - 1);
    if (nloc > 1) request(nloc - 2);
    if (wave < kHeads) {  // a wave per head, a lane per step, from the last
        float sum = wave == 0 ? behind[0] : wave == 1 ? behind[1] : wave == 2 ? behind[2] : behind[3];
        const float next = seg_stop + lane < all ? decay[(size_t)(seg_stop + lane) * a.H + wave] : 0.f;  // behind the segment
        const float beyond = read_lane_f32(wave_inclusive_scan_f32(next), 63);
        int first = nloc;
        for (int b0 = 0; b0 < nloc; b0 += 64) {
            const int i = nloc - 1 - b0 - lane;
            const float inc = wave_inclusive_scan_f32(i >= 0 ? decay[(size_t)(begin0 + i) * a.H + wave] : 0.f);
            float before = __shfl_up(inc, 1, 64);
            if (lane == 0) before = 0.f;
            const float left = sum + before, f = fast_exp2(left);
            if (i >= 0) {
                lds.f[i][wave] = left + beyond <= -10.f ? f : -f;
                if (f != 0.f) first = min(first, i);
            }
            sum += read_lane_f32(inc, 63);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) first = min(first, __shfl_xor(first, o, 64));
        if (lane == 0) {
            lds.first[wave] = first;
            if (u == 0) a.total[(size_t)useg * a.H + h0 + wave] = sum;
        }
    }
    lds_barrier();
    const int begin = min(min(lds.first[0], lds.first[1]), min(lds.first[2], lds.first[3]));  // (nloc: nothing at all)
    const int lr = lane & 15, lb = lane >> 4, hh = wave >> 1, cw = wave & 1;
    const int trow = state_tok(lb, lr >> 2), q4 = lr & 3;
    const int x_at = TX::row_at(trow) + 2 * (kP * hh + 32 * cw + 8 * q4);
    const int b_at = TB::row_at(trow) + 16 * ((q4 >> 1) ^ (trow & 3)) + 8 * (q4 & 1);  // odd tiles: ^ 32
    f32x4 sacc[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) sacc[nt][0] = sacc[nt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    float f_next = lds.f[nloc - 1][hh];
    for (int i = nloc - 1; i >= begin; --i) {
        landed(i > 0 && i - 1 >= min(begin, nloc - 2));
        lds_barrier();  // the tiles of step i are there, everyone is done with those of step i + 1
        if (i - 2 >= begin) request(i - 2);
        const float f = read_lane_f32(f_next, 0), scale = __builtin_fabsf(f);
        f_next = lds.f[max(i - 1, 0)][hh];
        if (scale == 0.f) continue;  // uniform: nothing of this head
        const uint32_t bt = lds_offset(lds.b[i % kRE].v) + b_at;
        strd_s16x4 xr[4], ba[8];
        lds_issue_tr4<0, TX::kBlock, 8, TX::kBlock + 8>(lds.x[i % kRE].v + x_at, xr);
        const float *const wp = &lds.w[i % kRE][hh * kQ + 8 * lb];
        const f32x4 w0 = *reinterpret_cast<const f32x4 *>(wp), w1 = *reinterpret_cast<const f32x4 *>(wp + 4);
        __builtin_amdgcn_s_waitcnt(lgkm_wait_imm(0));
        lds_settle4(xr);
        issue_b_frags<0, TB::kBlock>(bt, bt ^ 32, ba);
        bf16x8 wx[3][2];
        const f32x4 v0 = w0 * scale, v1 = w1 * scale;
#pragma unroll
        for (int pt = 0; pt < 2; ++pt) {
            const bf16x8 xf = tr_pair(xr[2 * pt], xr[2 * pt + 1]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = (float)xf[e], w = e < 4 ? v0[e & 3] : v1[e & 3];
                wx[0][pt][e] = (bf16_t)(x * w);
                const float rest = fmaf(x, w, -(float)wx[0][pt][e]);
                wx[1][pt][e] = (bf16_t)rest;
                wx[2][pt][e] = (bf16_t)(rest - (float)wx[1][pt][e]);
            }
        }
        const bool third = !(f >= 0.f);  // uniform
        lds_settle8(ba);
        auto products = [&](int d0) __attribute__((always_inline)) {
            auto add = [&](int piece) __attribute__((always_inline)) {
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int pt = 0; pt < 2; ++pt) sacc[(d0 + d) % NT][pt] = mfma16(tr_pair(ba[2 * d], ba[2 * d + 1]), wx[piece][pt], sacc[(d0 + d) % NT][pt]);
            };
            add(0);
            add(1);
            if (third) add(2);
        };
        products(0);
        if constexpr (NT == 8) {
            __builtin_amdgcn_sched_barrier(0);
            issue_b_frags<128, TB::kBlock>(bt, bt ^ 32, ba);
            lds_settle8(ba);
            products(4);
        }
    }
    async_tile_wait();  // (nothing lands in LDS that is no longer this workgroup's)
    float *dst = a.ends + (size_t)upart * a.H * kP * NS;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int pt = 0; pt < 2; ++pt)
            *reinterpret_cast<f32x4 *>(dst + ((size_t)(h0 + hh) * kP + chan_of(cw, pt, lr)) * NS + 16 * nt + 4 * lb) = sacc[nt][pt];
}

// A thread of the next two kernels has kVecs times four entries of a state, a workgroup 1024 kVecs of one head, those of a thread 1024 apart.
constexpr int kVecs = 4;
struct Entries {
    f32x4 v[kVecs];
    __device__ __forceinline__ void load(const float *p) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) v[i] = *reinterpret_cast<const f32x4 *>(p + 1024 * i);
    }
    __device__ __forceinline__ void store(float *p) const {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) *reinterpret_cast<f32x4 *>(p + 1024 * i) = v[i];
    }
};

// The state behind a segment (entries from element `at` on, head h); run is the one before it.  Which parts have left something is asked for at once, 64
// of them at a time, what they have left two at a time.
template <int NS>
__device__ __forceinline__ void pass_segment(const PackArgs &a, int s, int seg, size_t at, int h, Entries &run) {
    const size_t state = (size_t)a.H * kP * NS;
    const int per = a.parts_of(s), quad = h / kHeads, lane = threadIdx.x & 63;
    const size_t part0 = a.parts[s] + (size_t)seg * per;
    const float total = a.total[(size_t)(a.base[s] + seg) * a.H + h];
    bool scaled = false;
    for (int u0 = 0; u0 < per; u0 += 64) {
        const int u = min(u0 + lane, per - 1);
        unsigned long long left = __ballot(u0 + lane < per && a.alive[(part0 + u) * a.wg + quad]);
        if (!scaled) {
            const float f = fast_exp2(total);
#pragma unroll
            for (int i = 0; i < kVecs; ++i) run.v[i] *= f;
            scaled = true;
        }
        const float *const from = a.ends + (part0 + u0) * state + at;
        while (left) {
            const int k0 = __builtin_ctzll(left);
            left &= left - 1;
            const bool two = left != 0;
            const int k1 = two ? __builtin_ctzll(left) : k0;
            left &= left - 1;
            Entries x, y;
            x.load(from + (size_t)k0 * state);
            y.load(from + (size_t)k1 * state);
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                run.v[i] += x.v[i];
                if (two) run.v[i] += y.v[i];
            }
        }
    }
}

// ---- the states before the segments of a sequence, one after the other ---------------------------------------------------------------------------
template <int NS>
__global__ __launch_bounds__(256) void ssd_packed_chain_kernel(PackArgs a) {
    const int s = blockIdx.y, nseg = a.count(s);
    const size_t state = (size_t)a.H * kP * NS, at = (size_t)blockIdx.x * (1024 * kVecs) + 4 * threadIdx.x;
    static_assert(kP * NS % (1024 * kVecs) == 0, "a workgroup's entries are of one head");
    const int h = (int)(at / (kP * NS));
    Entries run = {};
    if (a.S_in && !(a.fresh >> s & 1)) run.load(a.S_in + (size_t)a.slot[s] * state + at);
    for (int seg = 0; seg + 1 < nseg; ++seg) {
        pass_segment<NS>(a, s, seg, at, h, run);
        run.store(a.init + (size_t)(a.first[s] + seg + 1) * state + at);
    }
}

// ---- final states; what is not finite stays for good --------------------------------------------------------------------------------------------
template <int NS>
__global__ __launch_bounds__(256) void ssd_packed_finish_kernel(PackArgs a) {
    constexpr int kPer = kP * NS / (1024 * kVecs);  // workgroups per head
    const int s = blockIdx.y, h = blockIdx.x / kPer, nseg = a.count(s);
    const size_t state = (size_t)a.H * kP * NS, at = (size_t)blockIdx.x * (1024 * kVecs) + 4 * threadIdx.x;
    Entries run = {};
    if (a.S_out) {
        const bool forgotten = fast_exp2(a.total[(size_t)(a.base[s] + nseg - 1) * a.H + h]) == 0.f;  // (and not NaN, nor a state that is lost)
        if (forgotten) ;
        else if (nseg > 1) run.load(a.init + (size_t)(a.first[s] + nseg - 1) * state + at);
        else if (a.S_in && !(a.fresh >> s & 1)) run.load(a.S_in + (size_t)a.slot[s] * state + at);
        pass_segment<NS>(a, s, nseg - 1, at, h, run);
    }
    auto is_lost = [](const uint32_t (&m)[2], int p) { return m[p >> 5] >> (16 * (p >> 2 & 1) + 4 * ((p & 31) >> 3) + (p & 3)) & 1; };  // channel p (chan_of)
    uint32_t m[2] = {0, 0};
    for (int seg = 0; seg < nseg; ++seg) {
        const uint32_t *l = a.lost + ((size_t)(a.base[s] + seg) * a.H + h) * 2;
        m[0] |= l[0], m[1] |= l[1];
        if (!(m[0] | m[1]) || seg + 1 == nseg || blockIdx.x % kPer) continue;  // uniform
        const int r0 = a.row0[s] + (seg + 1) * a.steps[s] * kQ, r1 = min(a.row0[s] + a.len[s], r0 + a.steps[s] * kQ);
        const int p = threadIdx.x % kP;
        if (is_lost(m, p))
            for (int r = r0 + (int)threadIdx.x / kP; r < r1; r += 256 / kP) a.y[((size_t)r * a.H + h) * kP + p] = (bf16_t)__builtin_nanf("");
    }
    if (!a.S_out) return;
    if (m[0] | m[1]) {
        const float nan = __builtin_nanf("");
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
            if (is_lost(m, (int)((at + 1024 * i) % (kP * NS)) / NS)) run.v[i] = f32x4{nan, nan, nan, nan};
    }
    run.store(a.S_out + (size_t)a.slot[s] * state + at);
}

struct Layout {
    int steps[kMaxSeqs], nseg[kMaxSeqs];  // by sequence
    int take;                             // steps of a full segment
    int part_steps;                       // of a part of a segment, whose contribution to the state behind the segment one workgroup makes
    long long segs = 0, multi_segs = 0, parts = 0, steps_all = 0;
    int most_parts = 0;                   // of a segment
    size_t init, ends, alive, total, lost, decay, weight;  // bytes of the parts of the workspace
    size_t bytes() const { return init + ends + alive + total + lost + decay + weight; }
};

// How the sequences are cut: the length of a segment, in steps, is what is estimated to end first.  A segment's workgroups are one XCD's, of 32 CUs with
// one workgroup at a time, which takes about 3 steps to start; cutting costs a launch, about 4 steps, and every segment of a sequence that is cut leaves and
// reads states, on all CUs about 9 steps' time for one each.  (3493 tokens of six sequences of 128 heads in segments of 22 steps 91 us, of 30 98, of 20 and
// two rounds 104, of 10 109.)
Layout lay_out(const CarryTab &t, int H, int n) {
    constexpr int kCUs = 32, kMinSegSteps = 8, kStart = 3, kCut = 4, kMostParts = 80;
    constexpr double kState = 9. / (kXcd * kCUs);
    const int wg = H / kHeads;
    int longest = 1, steps = 0;
    for (int s = 0; s < t.nseq; ++s) longest = std::max(longest, ceil_div(t.len[s], kQ)), steps += ceil_div(t.len[s], kQ);
    double best = 0.;
    int take = 0;
    auto look_at = [&](int len) {
        len = std::min(std::max(len, kMinSegSteps), longest);
        int fulls = 0, multi = 0, nrest = 0, rest[kMaxSeqs];
        for (int s = 0; s < t.nseq; ++s) {
            const int k = ceil_div(t.len[s], kQ);
            fulls += k / len;
            if (k % len) rest[nrest++] = k % len;
            if (k > len) multi += ceil_div(k, len);
        }
        std::sort(rest, rest + nrest, std::greater<int>());
        double worst = 0.;
        for (int x = 0; x < kXcd; ++x) {
            double sum = (double)(fulls / kXcd) * (len + kStart), first = fulls >= kXcd ? len + kStart : 0;
            for (int round = fulls / kXcd; round * kXcd < fulls + nrest; ++round) {
                const int rank = round * kXcd + (round & 1 ? kXcd - 1 - x : x);
                if (rank >= fulls + nrest) continue;
                const double here = (rank < fulls ? len : rest[rank - fulls]) + kStart;
                sum += here, first = std::max(first, here);
            }
            worst = std::max(worst, std::max(first, sum * wg / kCUs));
        }
        const double est = worst + (multi ? kCut + multi * wg * kState * n / 128 : 0);
        if (!take || est < best) best = est, take = len;
    };
    look_at(longest);
    for (int rounds = 1; rounds <= 4; ++rounds) {  // workgroups one after the other on a CU
        const int places = rounds * kXcd * std::max(1, kCUs / wg);
        // equal shares, and the shortest segments of which there are no more than places
        look_at(ceil_div(steps, places));
        int lo = 1, hi = longest;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            int segs = 0;
            for (int s = 0; s < t.nseq; ++s) segs += ceil_div(ceil_div(t.len[s], kQ), mid);
            if (segs <= places) hi = mid;
            else lo = mid + 1;
        }
        look_at(lo);
    }
    Layout l;
    l.take = take;
    // Equal parts of a full segment, of about 24 steps, of more where there were too many of them (each is a state in the workspace).  (33280 tokens in
    // segments of 130 steps: parts of 22 steps 413 us, of 16 and 32 435 and 427, of 44 431, of 64 461.)
    int part = 24;
    while (part < kMostPart && steps / part > kMostParts) part = std::min(2 * part, kMostPart);
    l.part_steps = ceil_div(take, ceil_div(take, part));
    for (int s = 0; s < t.nseq; ++s) {
        const int k = ceil_div(t.len[s], kQ);
        l.steps[s] = std::min(k, take);
        l.nseg[s] = k ? ceil_div(k, take) : 0;
        l.segs += l.nseg[s];
        if (l.nseg[s] > 1) l.multi_segs += l.nseg[s];
        l.parts += (long long)l.nseg[s] * ceil_div(l.steps[s], l.part_steps);
        l.most_parts = std::max(l.most_parts, ceil_div(l.steps[s], l.part_steps));
    }
    l.steps_all = steps;
    const size_t state = (size_t)H * kP * n * sizeof(float);
    l.init = l.multi_segs * state;
    l.ends = l.parts * state;
    l.alive = align_up(l.parts * wg * sizeof(uint32_t), 256);
    l.total = align_up(l.segs * H * sizeof(float), 256);
    l.lost = align_up(l.segs * H * 2 * sizeof(uint32_t), 256);
    l.decay = align_up((size_t)steps * H * sizeof(float), 256);
    l.weight = (size_t)steps * H * kQ * sizeof(float);
    return l;
}

template <int NS>
int launch(const PackArgs &a, const Layout &l, hipStream_t st) {
    const int grid = ceil_div((int)l.segs, kXcd) * kXcd * a.wg, pieces = a.H * kP * NS / (1024 * kVecs);
    const size_t lds = sizeof(LdsP<NS>), lds_ends = sizeof(LdsE<NS>);
    if (!allow_dynamic_lds((const void *)&ssd_packed_kernel<NS>, lds) || !allow_dynamic_lds((const void *)&ssd_packed_ends_kernel<NS>, lds_ends))
        return STRD_EHIP;
    ssd_packed_steps_kernel<<<dim3((unsigned)l.steps_all, ceil_div(a.H, 64)), 256, 0, st>>>(a);
    if (a.nmulti || a.S_out) ssd_packed_ends_kernel<NS><<<dim3(grid, l.most_parts), kEndThreads, lds_ends, st>>>(a);
    if (a.nmulti) ssd_packed_chain_kernel<NS><<<dim3(pieces, a.nmulti), 256, 0, st>>>(a);
    ssd_packed_kernel<NS><<<grid, kThreads, lds, st>>>(a);
    if (a.nmulti || a.S_out) ssd_packed_finish_kernel<NS><<<dim3(pieces, a.S_out ? a.nseq : a.nmulti), 256, 0, st>>>(a);
    return launch_status();
}

}  // namespace

// bf16, heads of 64 channels in groups of a multiple of four, state sizes 64 and 128.
bool ssd_packed_supported(long long rows, int H, int P, int G, int n, strd_dtype io) {
    return io == STRD_BF16 && P == kP && (n == 64 || n == 128) && H / G % kHeads == 0 && H <= 65535 && rows <= kMostCarryRows &&
           // rows of a step are reached by 32-bit offsets, states of a launch by the grid
           (long long)H * kP * 2 * kQ < 1LL << 31;
}

size_t ssd_packed_ws(const CarryTab &t, int H, int n) { return lay_out(t, H, n).bytes(); }

int ssd_packed(const void *x, const float *dt, const float *A, const void *B, const void *C, const float *D, const float *S_in, float *S_out, const CarryTab &t,
               void *y, int H, int G, int n, void *ws, hipStream_t st) {
    const Layout l = lay_out(t, H, n);
    if ((l.segs + kXcd) * (H / kHeads) > 1 << 22 || l.steps_all > 1 << 23 || l.most_parts > 65535) return STRD_EUNSUPPORTED;  // threads of a launch have 32 bits
    PackArgs a = {};
    a.x = (const bf16_t *)x, a.dt = dt, a.A = A, a.B = (const bf16_t *)B, a.C = (const bf16_t *)C, a.D = D, a.S_in = S_in, a.y = (bf16_t *)y, a.S_out = S_out;
    a.H = H, a.G = G, a.wg = H / kHeads;
    char *w = (char *)ws;
    a.init = (float *)w, w += l.init;
    a.ends = (float *)w, w += l.ends;
    a.alive = (uint32_t *)w, w += l.alive;
    a.total = (float *)w, w += l.total;
    a.lost = (uint32_t *)w, w += l.lost;
    a.decay = (float *)w, w += l.decay;
    a.weight = (float *)w;
    int order[kMaxSeqs], count = 0;
    for (int s = 0; s < t.nseq; ++s)
        if (t.len[s]) order[count++] = s;
    std::stable_partition(order, order + count, [&](int s) { return l.nseg[s] > 1; });
    int fulls = 0, nrest = 0;
    auto rest_of = [&](int i) { return ceil_div(a.len[i], kQ) % l.take; };
    int segs = 0, parts = 0, firsts = 0, steps = 0;
    for (int i = 0; i < count; ++i) {
        const int s = order[i];
        a.row0[i] = t.row0[s], a.len[i] = t.len[s], a.slot[i] = t.slot[s], a.steps[i] = l.steps[s];
        a.base[i] = segs, a.parts[i] = parts, a.step0[i] = steps, a.full[i] = fulls;
        fulls += ceil_div(t.len[s], kQ) / l.take;
        if (rest_of(i)) a.rest[nrest++] = (unsigned char)i;
        steps += ceil_div(t.len[s], kQ);
        a.fresh |= (t.fresh >> s & 1) << i;
        a.first[i] = -1;
        segs += l.nseg[s];
        if (l.nseg[s] > 1) {
            a.first[i] = firsts;
            firsts += l.nseg[s];
            ++a.nmulti;
        }
        parts += l.nseg[s] * ceil_div(l.steps[s], l.part_steps);
    }
    a.nseq = count, a.part_steps = l.part_steps;
    a.base[count] = segs, a.parts[count] = parts, a.step0[count] = steps, a.full[count] = fulls;
    std::stable_sort(a.rest, a.rest + nrest, [&](int p, int q) { return rest_of(p) > rest_of(q); });
    if (S_out) {
        const int rc = copy_empty_slots(t, S_in, S_out, (size_t)H * kP * n, st);
        if (rc != STRD_OK) return rc;
    }
    if (count == 0) return launch_status();
    return n == 128 ? launch<128>(a, l, st) : launch<64>(a, l, st);
}

}  // namespace strd
