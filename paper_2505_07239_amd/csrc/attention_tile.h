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

#include <type_traits>

namespace comet_attn {

using comet_gemm::digits_to_planes;
using comet_gemm::to_digits;

typedef int v4i __attribute__((ext_vector_type(4)));
typedef u32 v2u __attribute__((ext_vector_type(2)));
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
    int tiles;           // row tiles of one key head (host bound): of a sequence, or, with split < 0, of the batch (tiles_before)
    int groups;          // column groups of the values
    int chunks, chunk;   // pieces the keys are cut into, keys of a piece
    int parts;           // XCDs that share the units of a piece
    bool far_rows;       // scores: the rows of a tile may be 2 GB apart or more
    signed char split;   // > 0: of the sequences those of up to so many new tokens, < 0: those of more than -split (launch_split)
    __device__ __forceinline__ bool takes(const Sequence& sq) const { return split == 0 || (split > 0 ? sq.nq <= split : sq.nq > -split); }
};

// One prompt among sequences of a single token each: planned together, the single tokens would get tiles of 64 rows, mostly empty,
// and long pieces of keys.  So where less than half of the places for tokens can be taken, the sequences whose rows fit a
// small tile (or a single token) have a launch of their own, planned for them.  One prompt of 512 tokens and 31 sequences of 8000
// down to 6890 keys, 32 query and 8 key heads of 128 words: scores 2660 us together, 789 apart (floor 680), values 2800
// and 639 (floor 674 at the rate of a copy; reading alone is faster).
template <class Launch>
int launch_split(ProductParams& p, Launch launch) {
    const Batch& b = p.b;
    const int few = b.group < 16 ? 16 / b.group : 1;
    p.split = 0;
    if (b.by_sequence || b.max_q <= few) return launch(b.max_q);
    p.split = (signed char)few;
    const int rc = launch(few);
    if (rc != COMET_OK) return rc;
    p.split = (signed char)-few;
    return launch(b.max_q);
}
// The prompts of a split batch have their row tiles numbered along its tokens, so that a launch has as many as there can be, whatever
// the number of sequences that might have been prompts: the tiles of a sequence that begins at token q have the numbers from
// tiles_before(q) on.  A prompt of n > -split tokens ends before the numbers of the next one, as
// floor((q + n) g / R) - floor(q g / R) + 1 >= ceil(n g / R).  (A prompt of 1024 tokens of 128 heads over one row of 576 words among
// 255 single tokens, score rows of 4096 words: scores 8.6 ms, values 3.4; with a prompt's tiles for every sequence 50.4 and 11.5.)
__host__ __device__ inline int tiles_before(const Batch& b, int few, int R, int q) {
    return (int)((int64_t)q * b.group / R) + q / (few + 1);
}
// Row tiles of one key head that a launch may find rows for, over all sequences.
inline int64_t filled_tiles(const ProductParams& p, int R) {
    const Batch& b = p.b;
    const int64_t all = (int64_t)b.n_seq * p.tiles, most = p.split < 0 ? b.n_tok / -p.split : b.n_seq;
    const int64_t by_token = (int64_t)b.n_tok * b.group / R + (most < b.n_seq ? most : b.n_seq);
    return all < by_token ? all : by_token;
}

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
// the same cached rows it is.  Those follow each other on one of the eight XCDs, to which workgroups are dealt in turn; where
// there are few pieces, a piece's units are dealt to several XCDs (parts), so that all have the same number.
// With split < 0 the tiles of all sequences are one row of units.
struct Unit {
    int s, kvh, chunk, tile, cg;   // tile: of the sequence, those whose rows see most first; cg: column group
    bool live;
    __device__ __forceinline__ Unit(const ProductParams& p, int R) {
        const Batch& b = p.b;
        const unsigned n_inner = (unsigned)(p.tiles * p.groups), chunks = (unsigned)p.chunks, parts = (unsigned)p.parts;
        const unsigned per = (n_inner + parts - 1) / parts;
        const unsigned block = block_number(), q = block >> 3, group = (q / per) * 8 + (block & 7);
        const unsigned piece = group / parts, pair = piece / chunks, inner = q % per * parts + group % parts;
        chunk = (int)(piece % chunks);
        live = pair < (unsigned)pairs(p) && inner < n_inner;
        s = (int)(pair / (unsigned)b.n_kv_heads);
        kvh = (int)(pair % (unsigned)b.n_kv_heads);
        tile = p.tiles - 1 - (int)(inner / (unsigned)p.groups);
        cg = (int)(inner % (unsigned)p.groups);
        // (expected rare: otherwise the allocator takes the search for as hot as the main loops, and spills registers in those)
        if (__builtin_expect(p.split < 0 && live, 0)) find(b, -p.split, R);
    }
    // The sequence of tile number `tile`: the last whose tiles begin at or before it.
    __device__ __forceinline__ void find(const Batch& b, int few, int R) {
        const int number = tile;
        s = 0;
        for (int end = b.n_seq; end - s > 1;) {
            const int mid = s + (end - s) / 2;
            if (tiles_before(b, few, R, sequence_start(b, mid)) <= number) s = mid;
            else end = mid;
        }
        tile -= tiles_before(b, few, R, sequence_start(b, s));
        live = tile >= 0;
    }
    static __host__ __device__ int pairs(const ProductParams& p) { return (p.split < 0 ? 1 : p.b.n_seq) * p.b.n_kv_heads; }
    // Workgroups of a launch whose pieces and tiles of a sequence are set; deals them out.
    static int64_t grid(ProductParams& p, int R) {
        if (p.split < 0) p.tiles = tiles_before(p.b, -p.split, R, p.b.n_tok);
        const int64_t pieces = (int64_t)pairs(p) * p.chunks;
        p.parts = pieces >= 64 || pieces % 8 == 0 ? 1 : pieces % 4 == 0 ? 2 : pieces % 2 == 0 ? 4 : 8;
        return (pieces * p.parts + 7) / 8 * 8 * (((int64_t)p.tiles * p.groups + p.parts - 1) / p.parts);
    }
};

// Rows r0 .. r0 + R of a (sequence, key head): row number and keys seen of each, in LDS.  Row r is query head
// kvh * group + r % group of token r / group.
template <int R>
struct RowTile {
    __align__(16) int row[R];      // -1 beyond the last
    __align__(16) int sees[R];
    int row0;                      // the first row (a uniform value, the smallest there is)
    __device__ __forceinline__ void fill(const Batch& b, const Sequence& sq, int kvh, int r0) {
        if (threadIdx.x == 0) row0 = (sq.q0 + r0 / b.group) * b.n_heads + kvh * b.group;
        const int r = r0 + (int)threadIdx.x;
        if ((int)threadIdx.x < R) {
            const int n = sq.rows(b);
            const int j = r / b.group, h = kvh * b.group + r - j * b.group;
            row[threadIdx.x] = r < n ? (sq.q0 + j) * b.n_heads + h : -1;
            sees[threadIdx.x] = r < n ? sq.sees(b, j, h) : 0;
        }
    }
    // (behind a barrier) the most and the fewest keys that a row sees
    __device__ __forceinline__ void span(int& most, int& least) const {
        int hi = sees[threadIdx.x % R], lo = hi;
#pragma unroll
        for (int n = 1; n < R; n *= 2) {
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
    auto digit = [](int n) { const int q = n / (2 * RF); return n / RF & 1 ? 7 - q : q; };
    auto sub = [](int n) { return n % RF; };
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

// LDS accesses done, then meet the other wavefronts (loads from memory stay in flight).
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Words 2 J .. 2 J + 2 N - 1 of the sixteen of the lane's row in a block of 64 that begins at key0 (ld is even: rows are 16-byte
// aligned), and what does not count of them made zero.  The second step uses the words, so it stays away from the loads.
template <int J, int N>
__device__ __forceinline__ void load_row(const u64* row, int key0, int ld, int g, u64x2 (&w)[N]) {
    if (key0 + 64 <= ld) {
#pragma unroll
        for (int j = 0; j < N; ++j) w[j] = *reinterpret_cast<const u64x2*>(row + key0 + 8 * (J + j) + 2 * g);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int key = key0 + 8 * (J + j) + 2 * g;
            w[j] = *reinterpret_cast<const u64x2*>(row + (key < ld ? key : ld - 2));
        }
    }
}
template <int J, int N>
__device__ __forceinline__ void clear_beyond(u64x2 (&w)[N], int key0, int n, int g) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int key = key0 + 8 * (J + j) + 2 * g;
        w[j].x = key < n ? w[j].x : 0;
        w[j].y = key + 1 < n ? w[j].y : 0;
    }
}

// The blocks of a workgroup of eight wavefronts that multiplies 16 RF rows with sixteen columns of each, block by block: the rows'
// digits of both halves of the stacked contraction ([E | A]) go through one of two LDS stages while the other is
// multiplied; a wavefront's column words go straight into its registers, half a block ahead.
//   * WORKS: the wavefront has columns;  FEEDS: it has rows to convert, of the half and at the place that `put_at` says.
//   * The two wavefronts of a SIMD are out of step: one converts its column behind the barrier, the other (LATE) ahead of it,
//     so that one multiplies while the other converts.
//   * HALVES = 2: a wavefront multiplies both halves, and half a unit of every digit of the rows is on its way at a time, so
//     that the words fit the registers beside the rest.  HALVES = 1: it multiplies half h0 only.
// Source: row<J>(block, w) and clear<J>(block, w), words 2 J .. of the lane's row (load_row); column(half, block, w).
// Blocks are taken from `start` on, around the end.
template <int RF, int HALVES, bool WORKS, bool FEEDS, bool LATE, class Source>
__device__ __forceinline__ void sweep_blocks(v4i (&acc)[RF][8], const Source& src, int blocks, int start, int h0,
                                             unsigned char* put_at, const unsigned char* get_at) {
    constexpr int R = 16 * RF, HALF = R * 512, STAGE = 2 * HALF, WORDS = HALVES == 2 ? 4 : 8;
    u64x2 w[WORDS], v[8];
    v4i f[8];
    auto request = [&]<int J>(std::integral_constant<int, J>, int blk) {
        if constexpr (FEEDS) src.template row<J>(blk, w);
    };
    auto feed = [&]<int J>(std::integral_constant<int, J>, int blk, int st) {
        if constexpr (FEEDS) {
            src.template clear<J>(blk, w);
#pragma unroll
            for (int o = 0; o < WORDS / 4; ++o) {
                u64 x[8], plane[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) { x[2 * i] = to_digits(w[4 * o + i].x); x[2 * i + 1] = to_digits(w[4 * o + i].y); }
                digits_to_planes(x, plane);
#pragma unroll
                for (int t = 0; t < 8; ++t)
                    *reinterpret_cast<u64*>(put_at + st * STAGE + t * 4 * R * 16 + 8 * (J / 4 + o)) = plane[t];
            }
        }
    };
    const std::integral_constant<int, 0> lower{};
    const std::integral_constant<int, 4> upper{};
    int blk = start;
    request(lower, blk);
    if constexpr (WORKS) src.column(h0, blk, v);
    feed(lower, blk, 0);
    if constexpr (HALVES == 2) {
        request(upper, blk);
        feed(upper, blk, 0);
    }
    if constexpr (WORKS && LATE) to_units(v, f);
    for (int n = 0; n < blocks; ++n) {
        lds_barrier();
        const int next = blk + 1 < blocks ? blk + 1 : 0, st = (n + 1) & 1;
        const unsigned char* const from = get_at + (n & 1) * STAGE;
        if constexpr (WORKS) {
            if constexpr (!LATE) to_units(v, f);
            __builtin_amdgcn_sched_barrier(0);
            src.column(HALVES == 2 ? 1 : h0, HALVES == 2 ? blk : next, v);
        }
        request(lower, next);
        if constexpr (WORKS) multiply_block<RF>(acc, f, HALVES == 2 ? from : from + h0 * HALF);
        if constexpr (HALVES == 2) {
            if constexpr (WORKS) {
                to_units(v, f);
                __builtin_amdgcn_sched_barrier(0);
                src.column(0, next, v);
            }
            feed(lower, next, st);
            request(upper, next);
            if constexpr (WORKS) multiply_block<RF>(acc, f, from + HALF);
            feed(upper, next, st);
        } else {
            feed(lower, next, st);
        }
        if constexpr (WORKS && LATE) to_units(v, f);
        blk = next;
    }
}

int launch_scores(comet_ctx* ctx, const char* what, ProductParams& p);
int launch_values(comet_ctx* ctx, const char* what, ProductParams& p, void* ws, size_t ws_bytes);
size_t values_workspace_bytes(int64_t m, int64_t ld, int64_t d);

constexpr int MAX_D = 4096;      // words of a cached row that a product contracts (an int32 plane takes 8191), or of a row of values

}  // namespace comet_attn
