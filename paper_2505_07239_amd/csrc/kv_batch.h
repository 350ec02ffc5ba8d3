// A batch of sequences over a paged cache, as the attention kernels see it (comet_kv_batch in comet_ring.h).
#pragma once

#include "common.h"

namespace comet_attn {

struct Batch {
    int n_seq, n_tok, n_heads, n_kv_heads, group;   // group: query heads of a key head
    int page_size, max_pages, n_pages;
    int max_q;
    bool causal, by_sequence;                       // (by_sequence: Place)
    int ld, kv_cap;                                 // words in a row of a score matrix; longest readable sequence
    const int* q_start;
    const int* kv_len;
    const int* block_table;
    const unsigned char* head_mask;
};

// Where the tokens of sequence s begin (s = n_seq: where the last one's end).
__device__ __forceinline__ int sequence_start(const Batch& b, int s) {
    const int q = b.q_start[s];
    return q < 0 ? 0 : q > b.n_tok ? b.n_tok : q;
}

// One sequence, everything clamped to what the operands hold.
struct Sequence {
    int q0, nq, kv;          // first token, tokens, cached rows
    const int* pages;

    __device__ __forceinline__ Sequence(const Batch& b, int s) {
        const int end = sequence_start(b, s + 1);
        q0 = sequence_start(b, s);
        nq = end < q0 ? 0 : end - q0;
        const int n = b.kv_len[s];
        kv = n < 0 ? 0 : n > b.kv_cap ? b.kv_cap : n;
        pages = b.block_table + (size_t)s * b.max_pages;
    }
    // rows of a key head that are computed
    __device__ __forceinline__ int rows(const Batch& b) const { return (nq < b.max_q ? nq : b.max_q) * b.group; }
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

// Kernels with rows of their own count places (sequence, j < max_q), or, where less than half of those could be taken, tokens,
// whose sequence has to be searched for: one long prompt among many sequences must not cost as many workgroups as a batch of
// such prompts (tiles_before: the same for tiles of rows).  (The weights of four prompts of up to 512 tokens: 91 us by places, 93 by tokens.)
struct Place {
    int s, token;
    __device__ __forceinline__ Place(const Batch& b, unsigned i) {
        if (b.by_sequence) {
            s = (int)(i / (unsigned)b.max_q);
            token = -1;
            return;
        }
        // the last sequence that begins at or before token i
        int hi = b.n_seq;
        s = 0;
        token = (int)i;
        while (hi - s > 1) {
            const int mid = s + (hi - s) / 2;
            if (b.q_start[mid] <= token) s = mid;
            else hi = mid;
        }
    }
    // the token's number in the sequence, -1 if it is not one of those that are computed
    __device__ __forceinline__ int of(const Batch& b, const Sequence& sq, unsigned i) const {
        const int j = token < 0 ? (int)(i % (unsigned)b.max_q) : token - sq.q0;
        return j >= 0 && j < sq.nq && j < b.max_q ? j : -1;
    }
    static bool by_sequence(const Batch& b) {
        const int64_t n = (int64_t)b.n_seq * b.max_q;
        return n <= 2ll * b.n_tok && n * b.n_heads <= 0x7fffffffll;
    }
    static int64_t count(const Batch& b) { return b.by_sequence ? (int64_t)b.n_seq * b.max_q : b.n_tok; }
};

// A grid has fewer than 2^32 threads along x; more workgroups than fit get a second axis, with as many as 2^20 - 1 at the end
// that have nothing to do.  (2^20 is a multiple of eight: the XCDs take turns as along one axis.)
__device__ __forceinline__ unsigned block_number() { return (blockIdx.y << 20) + blockIdx.x; }
template <class... Args>
int launch_all(comet_ctx* ctx, const char* what, void (*kern)(Args...), int64_t grid, int threads, Args... args) {
    if (grid > 0x7fffffffll) return comet_fail(ctx, COMET_ECAP, "%s: too many rows", what);
    const bool one = grid <= 1 << 20;
    const dim3 blocks(one ? (unsigned)grid : 1u << 20, one ? 1u : (unsigned)((grid + (1 << 20) - 1) >> 20));
    hipLaunchKernelGGL(kern, blocks, dim3(threads), 0, ctx->stream, args...);
    COMET_LAUNCH_CHECK(ctx, what);
    return COMET_OK;
}

__device__ __forceinline__ u64 rescale(int party, u64 v, int f) {
    return party == 0 ? (u64)((long long)v >> f) : (u64)0 - (u64)((long long)((u64)0 - v) >> f);
}

}  // namespace comet_attn
