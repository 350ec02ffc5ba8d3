// Weights times cached values (comet_attention_values) on the int8 matrix cores:
//     Z(r, c) = t(C(r, c) + sum_j E(r, j) X(j, c) + A(r, j) F(j, c)) - M(r, c).
//
// The contraction runs over the keys, in blocks of 64, for E X and A F in turn.  A lane loads the sixteen words of
// its column in sixteen cached rows (consecutive lanes read consecutive columns) and of its row of weights, and splits and
// transposes both in registers.  Two kernels:
//   * values_few_kernel, up to 16 rows (a decoding step): a wavefront has 16 rows x 16 CT columns and every eighth block of
//     keys; nothing is shared, so there is no barrier until the eight wavefronts of a workgroup add their sums up in LDS.
//     Bound by HBM: 16 sequences of up to 8193 keys, 8 key heads of 128 words, 4 rows each: 288 us (floor 258 at 5.9 TB/s; 311 without
//     loads past the caches).  One token of 12 heads of 64 over 201 keys: 5.9 us, a chain of six dependent loads.
//   * values_many_kernel: 16 RF rows x 16 COLW columns.  A wavefront has 16 columns, whose cached words only it reads; the
//     weights, which all of them need, are converted once by all threads into one of two LDS stages while the other is
//     multiplied (sweep_blocks in attention_tile.h).  With at most 64 columns four wavefronts take E X and four A F.
//     Bound by the matrix units and power: 512 tokens of 32 heads over 4608 keys, 560 us (floor 337 at 3.9 POP/s of random
//     operands), matrix units busy 61 % of the cycles at 1.84 GHz.  With 48 rows 648, with the two wavefronts of a SIMD in step
//     and 64 rows 830; a barrier that waits for memory, or a spilled register in the loop, costs as much.
// Long sequences with few rows are cut into pieces, whose sums (of words, so that their order changes nothing)
// values_finish_kernel adds up.
#include "attention_tile.h"

using namespace comet_attn;

namespace {

constexpr int NT = 512, W = NT / 64;
constexpr int MAX_CHUNK = 8128;       // keys whose digit products an int32 plane can take: 2 * 8 * 8128 * 2^14 < 2^31
constexpr int GROUPS16 = MAX_CHUNK / 16 + 4;

// First slots of the groups of 16 keys (which lie in one page) from `first` on, in LDS; slot 0 beyond the last.
__device__ __forceinline__ void find_slots(int (&slots)[GROUPS16], const Batch& b, const Sequence& sq, int first, int end) {
    for (int i = threadIdx.x; i < GROUPS16; i += NT) {
        const int key = first + 16 * i;
        slots[i] = key < end ? (int)sq.slot(b, key) : 0;
    }
}

// The sixteen words of the lane's column in a block of 64 keys: key 8 j + 2 g + b is word 2 j + b.
// `slots`: those of the block's four groups; `lane_at`: byte offset of the lane's first row and column.  Buffer loads, so
// that a lane holds one offset for all of them.
template <int AUX = 0>
__device__ __forceinline__ void load_column(const u64* pool, const int* slots, u32 row_bytes, u32 lane_at, u64x2 (&w)[8]) {
    const v4i four = *reinterpret_cast<const v4i*>(slots);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const size_t at = (size_t)(u32)__builtin_amdgcn_readfirstlane(four[i]) * row_bytes;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(reinterpret_cast<const char*>(pool) + at), 0, -1, 0x00027000);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            w[2 * i + j].x = __builtin_bit_cast(u64, __builtin_amdgcn_raw_buffer_load_b64(rsrc, lane_at, 8 * j * row_bytes, AUX));
            w[2 * i + j].y = __builtin_bit_cast(u64, __builtin_amdgcn_raw_buffer_load_b64(rsrc, lane_at, (8 * j + 1) * row_bytes, AUX));
        }
    }
}

// CT: tiles of 16 columns of a wavefront.
template <int CT>
__global__ __launch_bounds__(NT) void values_few_kernel(ProductParams p) {
    constexpr int R = 16, COLS = 16 * CT;
    __shared__ __align__(16) int slots[GROUPS16];
    __shared__ RowTile<R> tile;
    __shared__ u64 sums[R * COLS];
    const Batch& b = p.b;
    const Unit unit(p, R);
    if (!unit.live) return;
    const int cg = unit.cg;
    const Sequence sq(b, unit.s);
    if (!p.takes(sq) || (int64_t)unit.tile * R >= sq.rows(b)) return;
    tile.fill(b, sq, unit.kvh, unit.tile * R);
    const int first = unit.chunk * p.chunk;
    find_slots(slots, b, sq, first, first + p.chunk < sq.kv ? first + p.chunk : sq.kv);
    for (int i = threadIdx.x; i < R * COLS; i += NT) sums[i] = 0;
    __syncthreads();
    int most, least;
    tile.span(most, least);
    const int end = most < first + p.chunk ? most : first + p.chunk;
    if (first >= end && unit.chunk > 0) return;

    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int row = tile.row[r] < 0 ? 0 : tile.row[r], sees = tile.sees[r];
    const u64* const e = p.E + (size_t)row * b.ld;
    const u64* const a = p.A + (size_t)row * b.ld;
    const u32 row_bytes = (u32)(b.n_kv_heads * p.ldp) * 8u;
    u32 lane_at[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        int col = cg * COLS + c * 16 + r;
        col = col < p.d ? col : p.d - 1;                      // (never written)
        lane_at[c] = (u32)(2 * g) * row_bytes + (u32)(unit.kvh * p.ldp + col) * 8u;
    }
    v4i acc[CT][8];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int s = 0; s < 8; ++s) acc[c][s] = v4i{0, 0, 0, 0};
    for (int key0 = first + 64 * wave; key0 < end; key0 += 64 * W) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u64x2 w[8];
            v4i x[8];
            load_row<0>(h ? a : e, key0, b.ld, g, w);
            if (key0 + 64 > least) clear_beyond<0>(w, key0, sees, g);
            to_units(w, x);
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                v4i f[8];
                load_column<2>(h ? p.F : p.X, slots + (key0 - first) / 16, row_bytes, lane_at[c], w);
                to_units(w, f);
#pragma unroll
                for (int t = 0; t < 8; ++t)
#pragma unroll
                    for (int u = 0; t + u < 8; ++u)
                        acc[c][t + u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[t], f[u], acc[c][t + u], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) atomicAdd(&sums[(4 * g + e4) * COLS + c * 16 + r], word_of(acc[c], e4));
    // (C and M are on their way while the sums come together)
    constexpr int EACH = (R * COLS + NT - 1) / NT;
    u64 c[EACH], m[EACH];
    size_t at[EACH];
    bool live[EACH];
#pragma unroll
    for (int n = 0; n < EACH; ++n) {
        const int i = n * NT + (int)threadIdx.x, col = cg * COLS + i % COLS, to = tile.row[i / COLS % R];
        live[n] = i < R * COLS && to >= 0 && col < p.d;
        at[n] = live[n] ? (size_t)to * p.d + col : 0;
        c[n] = p.part ? 0 : p.C[at[n]];
        m[n] = p.part || !p.M ? 0 : p.M[at[n]];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < EACH; ++n) {
        if (!live[n]) continue;
        const u64 sum = sums[n * NT + (int)threadIdx.x];
        if (p.part) p.part[(size_t)unit.chunk * b.n_tok * b.n_heads * p.d + at[n]] = sum;
        else p.Z[at[n]] = rescale(p.party, c[n] + sum, p.frac) - m[n];
    }
}

// What a wavefront of values_many_kernel reads: its row of weights, its column of the cached rows.
struct Source {
    const u64 *weights, *X, *F;
    const int* slots;
    int first, ld, sees, least, g;
    u32 row_bytes, lane_at;
    template <int J, int N>
    __device__ __forceinline__ void row(int blk, u64x2 (&w)[N]) const { load_row<J>(weights, first + 64 * blk, ld, g, w); }
    template <int J, int N>
    __device__ __forceinline__ void clear(int blk, u64x2 (&w)[N]) const {
        if (first + 64 * blk + 64 > least) clear_beyond<J>(w, first + 64 * blk, sees, g);
    }
    __device__ __forceinline__ void column(int h, int blk, u64x2 (&v)[8]) const {
        load_column(h ? F : X, slots + 4 * blk, row_bytes, lane_at, v);
    }
};

// COLW: wavefronts side by side along the columns; 4: the two halves of the workgroup take E X and A F.
template <int RF, int COLW>
__global__ __launch_bounds__(NT) void values_many_kernel(ProductParams p) {
    constexpr int R = 16 * RF, COLS = 16 * COLW, HALF = R * 512, STAGE = 2 * HALF;
    __shared__ __align__(16) unsigned char stage[2 * STAGE];
    __shared__ __align__(16) int slots[GROUPS16];
    __shared__ RowTile<R> tile;
    const Batch& b = p.b;
    const Unit unit(p, R);
    if (!unit.live) return;
    const int rt = unit.tile, cg = unit.cg;
    const Sequence sq(b, unit.s);
    if (!p.takes(sq) || (int64_t)rt * R >= sq.rows(b)) return;
    tile.fill(b, sq, unit.kvh, rt * R);
    const int first = unit.chunk * p.chunk;
    find_slots(slots, b, sq, first, first + p.chunk < sq.kv ? first + p.chunk : sq.kv);
    __syncthreads();
    int most, least;
    tile.span(most, least);
    const int end = most < first + p.chunk ? most : first + p.chunk;
    if (first >= end && unit.chunk > 0) return;

    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    // what this thread converts: its sixteen weights of row cr, of E (ch = 0) or A
    const bool feeds = wave < 2 * RF;
    const int ch = wave / RF, cr = (wave % RF) * 16 + r;
    const int crow = feeds && tile.row[cr] >= 0 ? tile.row[cr] : 0;
    const int csees = feeds ? tile.sees[cr] : 0;
    const u64* const weights = (ch ? p.A : p.E) + (size_t)crow * b.ld;
    unsigned char* const put_at = stage + (ch & 1) * HALF + (g * R + cr) * 16;
    // what it multiplies
    const int cw = wave % COLW, h0 = COLW == 8 ? 0 : wave / COLW;
    const u32 row_bytes = (u32)(b.n_kv_heads * p.ldp) * 8u;
    const int col = cg * COLS + cw * 16 + r;
    const bool works = cg * COLS + cw * 16 < p.d;
    const u32 lane_at = (u32)(2 * g) * row_bytes + (u32)(unit.kvh * p.ldp + (col < p.d ? col : p.d - 1)) * 8u;
    const unsigned char* const get_at = stage + (g * R + r) * 16;

    v4i acc[RF][8];
#pragma unroll
    for (int i = 0; i < RF; ++i)
#pragma unroll
        for (int s = 0; s < 8; ++s) acc[i][s] = v4i{0, 0, 0, 0};
    const int blocks = end > first ? (end - first + 63) / 64 : 0;
    // Every second row tile begins in the middle: rows of weights are a few pages of memory apart, and workgroups that all read
    // the same columns of them meet in the same few channels (512 rows of 4608 words: 784 us, and 559 with two
    // beginnings; four and eight are no better, and cost hits in L2).
    const int start = rt & 1 ? blocks / 2 : 0;
    const Source src = {weights, p.X, p.F, slots, first, b.ld, csees, least, g, row_bytes, lane_at};
    auto sweep = [&]<bool WORKS, bool FEEDS, bool LATE>() {
        sweep_blocks<RF, COLW == 8 ? 2 : 1, WORKS, FEEDS, LATE>(acc, src, blocks, start, h0, put_at, get_at);
    };
    if (blocks > 0) {
        if (wave < 4) {                                       // (these feed, whatever RF is)
            if (works) sweep.template operator()<true, true, false>();
            else sweep.template operator()<false, true, false>();
        } else if (feeds) {
            if (works) sweep.template operator()<true, true, true>();
            else sweep.template operator()<false, true, true>();
        } else {
            if (works) sweep.template operator()<true, false, true>();
            else sweep.template operator()<false, false, true>();
        }
    }
    u64* const sums = reinterpret_cast<u64*>(stage);
    if constexpr (COLW == 4) {
        // the halves of the workgroup meet in LDS
        __syncthreads();
        if (h0 == 1 && works)
#pragma unroll
            for (int i = 0; i < RF; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) sums[(16 * i + 4 * g + e) * COLS + cw * 16 + r] = word_of(acc[i], e);
        __syncthreads();
        if (h0 == 1) return;
    }
    if (!works || col >= p.d) return;
    // all loads first: Z may be C or M, so the compiler would wait for every store before the next load
    u64 c[RF][4], m[RF][4];
    if (!p.part)
#pragma unroll
        for (int i = 0; i < RF; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = tile.row[16 * i + 4 * g + e];
                const size_t at = (size_t)(row < 0 ? 0 : row) * p.d + col;
                c[i][e] = p.C[at];
                m[i][e] = p.M ? p.M[at] : 0;
            }
#pragma unroll
    for (int i = 0; i < RF; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int rr = 16 * i + 4 * g + e, row = tile.row[rr];
            u64 z = word_of(acc[i], e);
            if constexpr (COLW == 4) z += sums[rr * COLS + cw * 16 + r];
            if (row < 0) continue;
            if (p.part) p.part[((size_t)unit.chunk * b.n_tok * b.n_heads + row) * p.d + col] = z;
            else p.Z[(size_t)row * p.d + col] = rescale(p.party, c[i][e] + z, p.frac) - m[i][e];
        }
}

// n: Place::count().  Adds up the pieces of a row that have been written: those that begin before the last key it sees, and the first.
__global__ __launch_bounds__(256) void values_finish_kernel(ProductParams p, int pieces, unsigned n) {
    const Batch& b = p.b;
    unsigned w = block_number();
    const int piece = (int)(w % (unsigned)pieces); w /= (unsigned)pieces;
    const int h = (int)(w % (unsigned)b.n_heads); w /= (unsigned)b.n_heads;
    if (w >= n) return;
    const Place place(b, w);
    const Sequence sq(b, place.s);
    const int j = place.of(b, sq, w), col = piece * 256 + threadIdx.x;
    if (j < 0 || col >= p.d || !p.takes(sq)) return;
    const int row = (sq.q0 + j) * b.n_heads + h, sees = sq.sees(b, j, h);
    const size_t all = (size_t)b.n_tok * b.n_heads * p.d;
    const u64* from = p.part + (size_t)row * p.d + col;
    u64 sum = from[0];
    for (int c = 1; c * p.chunk < sees; ++c) sum += from[c * all];
    const size_t at = (size_t)row * p.d + col;
    const u64 z = rescale(p.party, p.C[at] + sum, p.frac);
    p.Z[at] = p.M ? z - p.M[at] : z;
}

// Pieces that the workspace of a call may hold: as many as a plane needs, and more while the partial sums of all rows
// stay small (32 M words).
int64_t max_chunks(int64_t m, int64_t ld, int64_t d) {
    const int64_t needed = (ld + MAX_CHUNK - 1) / MAX_CHUNK;
    int64_t n = m * d > 0 ? (32ll << 20) / (m * d) : 1;
    if (n > 64) n = 64;
    if (n > (ld + 255) / 256) n = (ld + 255) / 256;
    return n < needed ? needed : n;
}

}  // namespace

size_t comet_attn::values_workspace_bytes(int64_t m, int64_t ld, int64_t d) {
    if (m < 0 || ld < 2 || (ld & 1) || d < 1 || (d & 1) || d > MAX_D || ld > COMET_DIM_MAX || m > 0x7fffffffll) return 0;
    const int64_t n = max_chunks(m, ld, d);
    return n < 2 ? 0 : (size_t)n * m * d * 8;
}

static int launch_part(comet_ctx* ctx, const char* what, ProductParams& p, int max_q, void* ws) {
    const Batch& b = p.b;
    const int64_t n_rows = (int64_t)max_q * b.group, m = (int64_t)b.n_tok * b.n_heads;
    int R, cols, step;
    void (*kern)(ProductParams);
    // Up to 16 rows: four column tiles a wavefront, for whose sake the weights are loaded and split once; one where there are
    // not workgroups for every second compute unit, and the launch is as long as a wavefront's chain of loads.
    if (n_rows <= 16) {
        const bool small = (int64_t)b.n_seq * b.n_kv_heads * ((p.d + 63) / 64) * ((b.kv_cap + 64 * W - 1) / (64 * W)) * 2 <= ctx->num_cu;
        kern = small ? values_few_kernel<1> : values_few_kernel<4>;
        R = 16; cols = small ? 16 : 64; step = 64 * W;
    }
    // More: tiles of 64 rows, which convert a cached word half as often as tiles of 32; those where tiles of 64 would occupy up to two
    // thirds of the compute units (512 tokens of 12 heads of 64: 30 us, with 64 43; 100 tokens of 32/8 heads of 128: 15 and 22; 200 tokens
    // of 40 heads 26 and 33; 4 x 200 of 12 heads of 64, three quarters, 27 and 25).
    else {
        cols = p.d <= 64 ? 64 : 128;
        p.tiles = (int)((n_rows + 63) / 64);
        R = n_rows <= 32 || filled_tiles(p, 64) * b.n_kv_heads * ((p.d + cols - 1) / cols) * 3 <= 2 * ctx->num_cu ? 32 : 64;
        if (cols == 64) kern = R == 32 ? values_many_kernel<2, 4> : values_many_kernel<4, 4>;
        else kern = R == 32 ? values_many_kernel<2, 8> : values_many_kernel<4, 8>;
        step = 64;
    }
    p.tiles = (int)((n_rows + R - 1) / R);
    p.groups = (p.d + cols - 1) / cols;
    // Pieces of the keys: what the longest-working compute unit does, in steps of `step` keys, with two steps for the beginning
    // and the end of a workgroup, four for the second launch, which more than one piece needs, and one for every 2 M words
    // of partial sums, written and read again.
    const int64_t units = filled_tiles(p, R) * b.n_kv_heads * p.groups;
    const int64_t cap = max_chunks(m, b.ld, p.d), needed = (b.kv_cap + MAX_CHUNK - 1) / MAX_CHUNK;
    const int64_t steps = (b.kv_cap + step - 1) / step;
    const int64_t rows = filled_tiles(p, R) * R * b.n_kv_heads, words = (rows < m ? rows : m) * p.d;
    int64_t chunks = 1, best = INT64_MAX;
    for (int64_t n = needed > 1 ? needed : 1; n <= cap && (n <= steps || n <= needed); ++n) {
        // (the units of a mixed batch's prompts are a guess, not worth cutting for the last round of workgroups)
        if (p.split < 0 && n > needed && units * (n - 1) >= ctx->num_cu) break;
        const int64_t cost = (units * n + ctx->num_cu - 1) / ctx->num_cu * ((steps + n - 1) / n + 2) + (n > 1 ? 4 + n * words / (2 << 20) : 0);
        if (cost < best) { best = cost; chunks = n; }
    }
    p.chunk = (int)(((b.kv_cap + chunks - 1) / chunks + 63) / 64 * 64);
    if (p.chunk > MAX_CHUNK) p.chunk = MAX_CHUNK;
    if (p.chunk < 64) p.chunk = 64;
    p.chunks = b.kv_cap > 0 ? (b.kv_cap + p.chunk - 1) / p.chunk : 1;
    p.part = p.chunks > 1 ? (u64*)ws : nullptr;
    const int64_t grid = Unit::grid(p, R);
    const int pieces = (p.d + 255) / 256;
    const int64_t finish = Place::count(b) * b.n_heads * pieces;
    if (finish > 0x7fffffffll) return comet_fail(ctx, COMET_ECAP, "%s: too many rows", what);
    const int rc = launch_all(ctx, what, kern, grid, NT, p);
    return rc != COMET_OK || !p.part ? rc : launch_all(ctx, what, values_finish_kernel, finish, 256, p, pieces, (unsigned)Place::count(b));
}

int comet_attn::launch_values(comet_ctx* ctx, const char* what, ProductParams& p, void* ws, size_t ws_bytes) {
    const size_t need = values_workspace_bytes((int64_t)p.b.n_tok * p.b.n_heads, p.b.ld, p.d);
    if (need > 0 && (!ws || ws_bytes < need))
        return comet_fail(ctx, COMET_EWORKSPACE, "%s: needs %zu bytes of workspace", what, need);
    if (need > 0 && (reinterpret_cast<uintptr_t>(ws) & 255u) != 0)
        return comet_fail(ctx, COMET_EALIGN, "%s: the workspace must be 256-byte aligned", what);
    return launch_split(p, [&](int max_q) { return launch_part(ctx, what, p, max_q, ws); });
}
