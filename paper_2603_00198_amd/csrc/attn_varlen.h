// Packed batches of sequences for attention: which rows a workgroup takes, and how scores are changed.
#pragma once
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

struct AttnMod {
    AttnTab tab;
    long long ldq, ldk, ldv;    // elements between rows
    float scale, cap, inv_cap;  // cap == 0: none
    const float *slopes;        // [Hq] or null
    const int32_t *pos;         // [rows] or null: the row's number in its sequence
    int prefix;                 // vision rows see every vision row of their sequence
};

}  // namespace strd
