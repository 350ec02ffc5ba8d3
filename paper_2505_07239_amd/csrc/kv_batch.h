// A batch of sequences over a paged cache, as the attention kernels see it (comet_kv_batch in comet_ring.h).
#pragma once

#include "common.h"

namespace comet_attn {

struct Batch {
    int n_seq, n_tok, n_heads, n_kv_heads, group;   // group: query heads of a key head
    int page_size, max_pages, n_pages;
    int max_q, causal;
    int ld, kv_cap;                                 // words in a row of a score matrix; longest readable sequence
    const int* q_start;
    const int* kv_len;
    const int* block_table;
    const unsigned char* head_mask;
};

// One sequence, everything clamped to what the operands hold.
struct Sequence {
    int q0, nq, kv;          // first token, tokens, cached rows
    const int* pages;

    __device__ __forceinline__ Sequence(const Batch& b, int s) {
        int lo = b.q_start[s], hi = b.q_start[s + 1];
        lo = lo < 0 ? 0 : lo > b.n_tok ? b.n_tok : lo;
        hi = hi < lo ? lo : hi > b.n_tok ? b.n_tok : hi;
        q0 = lo;
        nq = hi - lo;
        const int n = b.kv_len[s];
        kv = n < 0 ? 0 : n > b.kv_cap ? b.kv_cap : n;
        pages = b.block_table + (size_t)s * b.max_pages;
    }
    // keys that head h of the j-th token sees
    __device__ __forceinline__ int sees(const Batch& b, int j, int h) const {
        int v = kv;
        if (b.causal) {
            v = kv - nq + j + 1;
            v = v < 0 ? 0 : v;                      // (at most kv: j < nq)
        }
        if (b.head_mask && !b.head_mask[(size_t)(q0 + j) * b.n_heads + h]) v = 0;
        return v;
    }
    // slot of key j < kv
    __device__ __forceinline__ size_t slot(const Batch& b, int j) const {
        const int i = j / b.page_size;
        int pg = pages[i];
        pg = (unsigned)pg < (unsigned)b.n_pages ? pg : 0;
        return (size_t)pg * b.page_size + (j - i * b.page_size);
    }
};

__device__ __forceinline__ u64 rescale(int party, u64 v, int f) {
    return party == 0 ? (u64)((long long)v >> f) : (u64)0 - (u64)((long long)((u64)0 - v) >> f);
}

}  // namespace comet_attn
