// What the decode steps over a cache with capped or biased scores and gathered weights share.
#pragma once
#include "kv4.h"

namespace strd {

constexpr int kDecMaxSplits = 512;
constexpr float kDecNegBig = -3.0e38f;

// x = scale * q.k -> score: the cap first, then the bias (see strd.h).
struct ScoreMod {
    float scale, cap, inv_cap;      // cap == 0: none
    const float *slopes;            // [Hq] or null
    const int32_t *pos;             // [T] or null: the row number
};
struct CacheView {
    const void *k, *km, *v, *vm;  // plain: k and v; 4-bit: codes and (s, z) pairs
};

// Partial results of a decode step in its workspace: per split and query head the weighted values [d], the reference and the
// sum of the softmax; then, for the weights, the scores of every (query head, token) in units of log2 e.
struct DecWs {
    float *part, *ml, *scores;  // scores: null if no weights are wanted
    long long ldt;              // floats between the scores of two heads
};
inline size_t dec_ws_bytes(int nsplit, int Hq, int d, long long ldt, bool weights) {
    return align_up((size_t)nsplit * Hq * (d + 2) * sizeof(float), 256) + (weights ? (size_t)Hq * ldt * sizeof(float) : 0);
}
inline long long dec_ldt(int T) { return ((long long)T + 63) / 64 * 64; }

struct DecCall {
    const void *q;
    CacheView c;
    void *o;
    int T, Hq, Hkv, d;
    ScoreMod mod;
    const float *w_in;
    float *w_out;
    strd_dtype io;
    bool kv4;
};

// Workgroup b runs on XCD b % 8, each with an L2 of its own: the kv heads of one split, which share lines of the cache -- a row's
// (s, z) pairs of 8 heads of 128 channels are one line -- go to one XCD, one after the other.
__device__ __forceinline__ void dec_place(int b, int Hkv, int &hk, int &split) {
    const int u = b / kXcd;
    hk = u % Hkv;
    split = b % kXcd + kXcd * (u / Hkv);
}
inline int dec_grid(int Hkv, int nsplit) { return Hkv * ((nsplit + kXcd - 1) / kXcd * kXcd); }

bool dec_mfma_supported(int T, int Hq, int Hkv, int d, bool kv4, strd_dtype io);
int dec_mfma_splits(int T, int Hkv, int d, bool kv4, int &tps);
int dec_mfma(const DecCall &a, const DecWs &ws, int nsplit, int tps, hipStream_t st);
int dec_splits_general(int T, int Hq, int Hkv, int &tps);
int dec_combine(const DecCall &a, const DecWs &ws, int nsplit, hipStream_t st);

}  // namespace strd
