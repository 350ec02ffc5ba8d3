// A batch of sequences over a paged cache, as the attention kernels see it (comet_kv_batch in comet_ring.h).
#pragma once

#include "common.h"

namespace comet_attn {

struct Batch {
    int n_seq, n_tok, n_heads, n_kv_heads, group;   // group: query heads of a key head
    int page_size, max_pages, n_pages;
    int max_q, causal;
    int ld, kv_cap;                                 // words in a row of a score matrix; longest readable sequence
    unsigned block0;                                // workgroups of the call in launches before this one (launch_all)
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

// Kernels with rows of their own count places (sequence, j < max_q), or tokens where those are fewer: one long prompt among
// many sequences must not cost as many workgroups as a batch of such prompts.
struct Place {
    int s, token;
    __device__ __forceinline__ Place(const Batch& b, unsigned i) {
        if (by_sequence(b)) {
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
    static __host__ __device__ __forceinline__ bool by_sequence(const Batch& b) { return (int64_t)b.n_seq * b.max_q <= b.n_tok; }
    static int64_t count(const Batch& b) { return by_sequence(b) ? (int64_t)b.n_seq * b.max_q : b.n_tok; }
};

// A launch has fewer than 2^32 threads; more workgroups than that allows go in several, each a multiple of eight of them, so
// that the XCDs take turns as in one.
template <class Params, class... More>
int launch_all(comet_ctx* ctx, const char* what, void (*kern)(Params, More...), int64_t grid, int threads, Params& p, More... more) {
    if (grid > 0x7fffffffll) return comet_fail(ctx, COMET_ECAP, "%s: too many rows", what);
    const int64_t most = ((1ll << 32) - 1) / threads / 8 * 8;
    for (int64_t at = 0; at < grid; at += most) {
        p.b.block0 = (unsigned)at;
        hipLaunchKernelGGL(kern, dim3((unsigned)(grid - at < most ? grid - at : most)), dim3(threads), 0, ctx->stream, p, more...);
        COMET_LAUNCH_CHECK(ctx, what);
    }
    return COMET_OK;
}

__device__ __forceinline__ u64 rescale(int party, u64 v, int f) {
    return party == 0 ? (u64)((long long)v >> f) : (u64)0 - (u64)((long long)((u64)0 - v) >> f);
}

}  // namespace comet_attn
