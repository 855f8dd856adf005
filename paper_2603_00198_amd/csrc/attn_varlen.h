// Packed batches of sequences for attention: which rows a workgroup takes, and how scores are changed.
#pragma once
#include <algorithm>

#include "common.h"

namespace strd {

// Sequences by falling length, cut into blocks of the kernel's rows.  Blocks are issued by level, the highest (in causal
// order the longest) first: on a level are the blocks with that number of every sequence that has as many.  Sequences 0 .. s
// are on the levels nb[s + 1] .. nb[s] - 1, whose blocks are base[s] .. base[s + 1] - 1.
struct AttnTab {
    int row0[kMaxSeqs], len[kMaxSeqs], vis[kMaxSeqs];  // first row, rows, vision rows
    int nb[kMaxSeqs], base[kMaxSeqs];
    int nseq;
    __device__ __forceinline__ void locate(int block, int &level, int &s) const {
        int top = 0;
        for (int i = 1; i < nseq; ++i) top = block >= base[i] ? i : top;  // (base never falls; equal: the later one holds the block)
        const int rem = block - base[top], row = rem / (top + 1);
        level = nb[top] - 1 - row;
        s = rem - row * (top + 1);
    }
};

constexpr int kMostRows = 1 << 30;

// Sequences with rows, longest first, in blocks of `bm` rows; false if the descriptors are inconsistent.
inline bool plan_attn(const strd_seq *seqs, int nseq, int bm, AttnTab &t, long long &rows, long long &units) {
    if (!seqs || nseq < 1 || nseq > STRD_VARLEN_MAX) return false;
    int order[STRD_VARLEN_MAX], n = 0;
    long long row0[STRD_VARLEN_MAX];
    rows = units = 0;
    for (int b = 0; b < nseq; ++b) {
        if (seqs[b].N < 0 || seqs[b].M < 0) return false;
        row0[b] = rows;
        rows += (long long)seqs[b].N + seqs[b].M;
        if (rows > kMostRows) return false;
        if (seqs[b].N + seqs[b].M > 0) order[n++] = b;
    }
    std::stable_sort(order, order + n, [&](int a, int b) { return seqs[a].N + seqs[a].M > seqs[b].N + seqs[b].M; });
    t = AttnTab();
    t.nseq = n;
    for (int i = 0; i < n; ++i) {
        const strd_seq &s = seqs[order[i]];
        t.row0[i] = (int)row0[order[i]];
        t.len[i] = s.N + s.M;
        t.vis[i] = s.N;
        t.nb[i] = ceil_div(t.len[i], bm);
        if (i) units += (long long)(t.nb[i - 1] - t.nb[i]) * i;
        t.base[i] = (int)std::min(units, (long long)kMostRows);
    }
    if (n) units += (long long)t.nb[n - 1] * n;
    return true;
}

struct AttnMod {
    AttnTab tab;
    long long ldq, ldk, ldv;    // elements between rows
    float scale, cap, inv_cap;  // cap == 0: none
    const float *slopes;        // [Hq] or null
    const int32_t *pos;         // [rows] or null: the row's number in its sequence
    int prefix;                 // vision rows see every vision row of their sequence
};

}  // namespace strd
