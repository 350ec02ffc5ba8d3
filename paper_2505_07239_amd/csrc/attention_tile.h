// What the matrix-core kernels of attention over a cache of shares have in common.
//
// A product of words is 36 products of signed base-256 digits (t + u <= 7, the others vanish mod 2^64), summed in
// eight int32 planes s = t + u and recombined at the end.  v_mfma_i32_16x16x64_i8 contracts 64 words of 16 rows and
// 16 columns; a lane holds, for one row (or column) and one digit, the sixteen words of its lane group g = lane / 16.
// Which sixteen is free as long as both operands agree: here word 2 j + b of group g is word 8 j + 2 g + b of the 64, so
// that the four groups of a row read 64 consecutive bytes at a time.
#pragma once

#include "digits.h"
#include "kv_batch.h"

namespace comet_attn {

using comet_gemm::digits_to_planes;
using comet_gemm::to_digits;

typedef int v4i __attribute__((ext_vector_type(4)));
typedef u64 u64x2 __attribute__((ext_vector_type(2)));

struct ProductParams {
    Batch b;
    int party, d, ldp, frac;
    const u64* E;
    const u64* A;
    const u64* F;
    const u64* X;
    const u64* C;
    const u64* M;
    u64* Z;
    u64* part;           // partial sums [split][row][d] of the values, null when the keys are not split
    int tiles;           // row tiles of one key head (host bound)
    int groups;          // column groups of the values
    int chunks, chunk;   // pieces the keys are cut into, keys of a piece
};

// Sixteen words of a lane in slot order -> its unit of every digit.
__device__ __forceinline__ void to_units(const u64x2 (&w)[8], v4i (&f)[8]) {
    u64 plane[2][8];
#pragma unroll
    for (int o = 0; o < 2; ++o) {
        u64 v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = to_digits(w[4 * o + i].x);
            v[2 * i + 1] = to_digits(w[4 * o + i].y);
        }
        digits_to_planes(v, plane[o]);
    }
#pragma unroll
    for (int t = 0; t < 8; ++t)
        f[t] = v4i{(int)(u32)plane[0][t], (int)(plane[0][t] >> 32), (int)(u32)plane[1][t], (int)(plane[1][t] >> 32)};
}

// The eight planes of an output word -> the word.
__device__ __forceinline__ u64 word_of(const v4i (&acc)[8], int e) {
    long long lo = (long long)acc[0][e];
    lo += (long long)acc[1][e] * (1 << 8);
    lo += (long long)acc[2][e] * (1 << 16);
    lo += (long long)acc[3][e] * (1 << 24);
    const u32 hi = (u32)acc[4][e] + ((u32)acc[5][e] << 8) + ((u32)acc[6][e] << 16) + ((u32)acc[7][e] << 24);
    return (u64)lo + ((u64)hi << 32);
}

// The work of a workgroup: a piece of the keys (chunk) of a (sequence, key head), and which of the `inner` units that read
// the same cached rows it is.  Those follow each other on one of the eight XCDs, to which workgroups are dealt in turn.
struct Unit {
    int s, kvh, chunk, inner;
    bool live;
    __device__ __forceinline__ Unit(const Batch& b, int n_inner, int chunks) {
        const unsigned q = blockIdx.x >> 3, group = (q / (unsigned)n_inner) * 8 + (blockIdx.x & 7);
        const unsigned pair = group / (unsigned)chunks;
        inner = (int)(q % (unsigned)n_inner);
        chunk = (int)(group % (unsigned)chunks);
        live = pair < (unsigned)(b.n_seq * b.n_kv_heads);
        s = (int)(pair / (unsigned)b.n_kv_heads);
        kvh = (int)(pair % (unsigned)b.n_kv_heads);
    }
    static int64_t grid(const Batch& b, int64_t n_inner, int64_t chunks) {
        return ((int64_t)b.n_seq * b.n_kv_heads * chunks + 7) / 8 * 8 * n_inner;
    }
};

// Rows r0 .. r0 + R of a (sequence, key head): row number and keys seen of each, in LDS.  Row r is query head
// kvh * group + r % group of token r / group.
template <int R>
struct RowTile {
    int row[R], sees[R];
    __device__ __forceinline__ void fill(const Batch& b, const Sequence& sq, int kvh, int r0) {
        const int r = r0 + (int)threadIdx.x;
        if ((int)threadIdx.x < R) {
            const int n = (sq.nq < b.max_q ? sq.nq : b.max_q) * b.group;
            const int j = r / b.group, h = kvh * b.group + r - j * b.group;
            row[threadIdx.x] = r < n ? (sq.q0 + j) * b.n_heads + h : -1;
            sees[threadIdx.x] = r < n ? sq.sees(b, j, h) : 0;
        }
    }
    // (behind a barrier) the most and the fewest keys that a row sees
    __device__ __forceinline__ void span(int& most, int& least) const {
        int hi = sees[threadIdx.x % R], lo = hi;
#pragma unroll
        for (int n = 1; n < 64; n *= 2) {
            const int a = __shfl_xor(hi, n), c = __shfl_xor(lo, n);
            hi = a > hi ? a : hi;
            lo = c < lo ? c : lo;
        }
        most = __builtin_amdgcn_readfirstlane(hi);
        least = __builtin_amdgcn_readfirstlane(lo);
    }
};

// One block of 64 words: acc[i] += rows 16 i .. 16 i + 15 (digits in LDS, `at` the lane's unit of digit 0 of the first) times the
// lane's column f.  The rows' units are read DEPTH ahead of their use, and the digits taken from both ends in turn, so that
// every two units feed nine instructions.
template <int RF>
__device__ __forceinline__ void multiply_block(v4i (&acc)[RF][8], const v4i (&f)[8], const unsigned char* at) {
    constexpr int N = 8 * RF, DEPTH = RF == 1 ? 2 : 4, R = 16 * RF;
    auto digit = [](int n) { const int q = n / (2 * RF); return n & 1 ? 7 - q : q; };
    auto sub = [](int n) { return n % (2 * RF) / 2; };
    auto read = [&](int n) { return *reinterpret_cast<const v4i*>(at + (digit(n) * 4 * R + sub(n) * 16) * 16); };
    v4i a[DEPTH];
#pragma unroll
    for (int n = 0; n < DEPTH; ++n) a[n] = read(n);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int t = digit(n), i = sub(n);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (t + u < 8) acc[i][t + u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[n % DEPTH], f[u], acc[i][t + u], 0, 0, 0);
        if (n + DEPTH < N) a[n % DEPTH] = read(n + DEPTH);
        __builtin_amdgcn_sched_barrier(0);
    }
}

int launch_scores(comet_ctx* ctx, const char* what, ProductParams& p);
int launch_values(comet_ctx* ctx, const char* what, ProductParams& p, void* ws, size_t ws_bytes);
size_t values_workspace_bytes(int64_t m, int64_t ld, int64_t d);

constexpr int MAX_D = 576;       // words of a cached row that a product contracts, or of a row of values

}  // namespace comet_attn
