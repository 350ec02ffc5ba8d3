// Queries times cached keys (comet_attention_scores) on the int8 matrix cores:
//     Z(r, j) = t(C(r, j) + [E | A](r, :) . [X | F](j, :)) - M(r, j).
//
// scores_kernel, d <= 256: a workgroup holds R = 16 RF rows in LDS, as digits, for the whole stacked contraction (E and A, each
// filled up to whole blocks of 64 words); behind the barrier that follows, its wavefronts are on their own.  Each takes every
// W-th tile of 16 keys: it loads its keys' words straight into registers, a block ahead of their use, splits them into
// digits and transposes them there (no other wavefront of the workgroup wants them), and multiplies them with the rows'
// digits, read from LDS in operand order.  So a cached word is fetched once per row tile, a query word once per workgroup.
// scores_many_kernel, d > 256: the rows' digits would not fit; both sides are streamed (sweep_blocks in attention_tile.h).
//
// What bounds them (us of a call; the floor at 5.9 TB/s and 3.9 POP/s):
//   * few rows, the cache read once: HBM.  16 sequences of up to 8193 keys, 8 key heads of 128 words, 4 rows each: 280 (floor 262,
//     5.5 TB/s).  Loads past the caches are slower here (374): a load takes half a line, the next one the other half.
//   * prompts, 4 of up to 512 tokens, 32 heads of 128: 153 (floor 75, matrix units busy 30 %).  By time stamps a workgroup of 64 rows
//     takes 7 us to begin (its row's digits 5), then per tile and pair of wavefronts 10 us of multiplying, in which the matrix units
//     are busy for nine tenths, and 7 of writing out, in which they are not.  Tried, without gain: 32 and 48 rows, more
//     workgroups of fewer rows or keys, C and M requested early (registers, or their lines into L2), priorities.
//   * latent rows, 64 heads of 4 sequences over 576 words: 62 (floor 22): a chain of nine blocks whose loads one wavefront per SIMD
//     cannot cover; smaller tiles that would add wavefronts split the keys more often (85).
//   * latent rows, 37 tokens of 64 heads over 2037 keys: 243 to 254 (floor 102): the conversion of both sides, and 36 registers of
//     scores_many_kernel<4, 8> that do not fit and are reloaded in its loop.
#include "attention_tile.h"

using namespace comet_attn;

namespace {

// A wavefront's tile: Z = t(C + sum) - M for the keys that its rows see.  All loads come before the first store: Z may be C or M,
// so the compiler would keep them in order, and a load behind a store is not there before the store has been acknowledged
// (the hardware counts both in order).  What a row does not see gets an offset outside the buffer, where loads give
// zero and stores nothing.
template <int RF>
__device__ __forceinline__ void write_out(const ProductParams& p, const RowTile<16 * RF>& tile, const v4i (&acc)[RF][8], int key0,
                                          int lane) {
    const int r = lane & 15, g = lane >> 4, key = key0 + r;
    if (!p.far_rows) {
        const int row0 = __builtin_amdgcn_readfirstlane(tile.row0);
        const size_t base = (size_t)row0 * p.b.ld + key0;
        const auto at = [&](const u64* q) {
            return __builtin_amdgcn_make_buffer_rsrc(const_cast<u64*>(q + base), 0, 0x7fffffff, 0x00027000);
        };
        const auto rc = at(p.C), rm = at(p.M ? p.M : p.C), rz = at(p.Z);
        u32 off[RF][4];
        u64 c[RF][4], m[RF][4];
#pragma unroll
        for (int i = 0; i < RF; ++i) {
            const v4i row = *reinterpret_cast<const v4i*>(tile.row + 16 * i + 4 * g);
            const v4i sees = *reinterpret_cast<const v4i*>(tile.sees + 16 * i + 4 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                off[i][e] = key < sees[e] ? (u32)(row[e] - row0) * ((u32)p.b.ld * 8u) + (u32)r * 8u : 0xffffffffu;
                c[i][e] = __builtin_bit_cast(u64, __builtin_amdgcn_raw_buffer_load_b64(rc, off[i][e], 0, 2));
                m[i][e] = p.M ? __builtin_bit_cast(u64, __builtin_amdgcn_raw_buffer_load_b64(rm, off[i][e], 0, 2)) : 0;
            }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < RF; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const u64 z = rescale(p.party, c[i][e] + word_of(acc[i], e), p.frac) - m[i][e];
                __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(v2u, z), rz, off[i][e], 0, 2);
            }
    } else {
        // rows of a tile 2 GB apart or more
#pragma unroll
        for (int i = 0; i < RF; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int rr = 16 * i + 4 * g + e;
                if (key < tile.sees[rr]) {
                    const size_t at = (size_t)tile.row[rr] * p.b.ld + key;
                    const u64 m = p.M ? p.M[at] : 0;
                    p.Z[at] = rescale(p.party, p.C[at] + word_of(acc[i], e), p.frac) - m;
                }
            }
    }
}

// KT: blocks of 64 words that fit the rows' place in LDS.  NT: threads.
template <int RF, int KT, int NT>
__global__ __launch_bounds__(NT, RF == 1 ? 4 : 2) void scores_kernel(ProductParams p) {
    constexpr int R = 16 * RF, W = NT / 64;
    __shared__ __align__(16) unsigned char rows[KT * R * 512];
    __shared__ RowTile<R> tile;
    const Batch& b = p.b;
    const Unit unit(p, R);
    if (!unit.live) return;
    const Sequence sq(b, unit.s);
    if (!p.takes(sq) || (int64_t)unit.tile * R >= sq.rows(b)) return;
    const int kvh = unit.kvh, r0 = unit.tile * R;
    const int first = unit.chunk * p.chunk;
    if (first >= sq.kv) return;
    tile.fill(b, sq, kvh, r0);

    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int d = p.d, half = (d + 63) / 64, blocks = 2 * half;

    // A tile's 16 keys lie in one page: a uniform address, and one offset per lane.  Buffer loads that end with the page's 16
    // rows: the last block may reach beyond d, where the rows' digits are zero, but never beyond the pool.
    const u32 row_bytes = (u32)(b.n_kv_heads * p.ldp) * 8u, head_at = (u32)(kvh * p.ldp) * 8u;
    const u32 lane_at = (u32)r * row_bytes + (u32)g * 16u, bytes = 16u * row_bytes - head_at;
    auto locate = [&](int key0) {
        return (size_t)(u32)__builtin_amdgcn_readfirstlane((int)sq.slot(b, key0)) * row_bytes + head_at;
    };
    auto block_at = [&](size_t off, int kb) {
        const u32 at = (u32)(kb < half ? kb : kb - half) * 512u;
        const char* const pool = reinterpret_cast<const char*>(kb < half ? p.X : p.F) + off + at;
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(pool), 0, (int)(bytes - at), 0x00027000);
    };
    auto load = [&](size_t off, int kb, u64x2 (&w)[8]) {
        const auto rsrc = block_at(off, kb);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            w[j] = __builtin_bit_cast(u64x2, __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane_at + 64 * j, 0, 0));
    };

    int key0 = first + 16 * wave;
    size_t off = key0 < sq.kv ? locate(key0) : 0;
    u64x2 w[8];
    load(off, 0, w);                                          // (under way while the rest is found out)
    __syncthreads();
    int most, least;
    tile.span(most, least);
    const int end = most < first + p.chunk ? most : first + p.chunk;
    if (first >= end) return;
    // the rows' digits: block kb, digit t, lane group g, row
    auto fetch_rows = [&](int i, u64x2 (&w)[8]) {
        const int kb = i / RF, row = tile.row[(i % RF) * 16 + r];
        const u64* const src = (kb < half ? p.E : p.A) + (size_t)(row < 0 ? 0 : row) * d;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int k = 64 * (kb < half ? kb : kb - half) + 8 * j + 2 * g;
            w[j] = u64x2{0, 0};
            if (row >= 0 && k < d) w[j] = *reinterpret_cast<const u64x2*>(src + k);
        }
    };
    {
        u64x2 now[8], next[8];
        if (wave < blocks * RF) fetch_rows(wave, now);
        for (int i = wave; i < blocks * RF; i += W) {
            if (i + W < blocks * RF) fetch_rows(i + W, next);
            v4i f[8];
            to_units(now, f);
            unsigned char* const to = rows + ((size_t)(i / RF * 32 + g) * R + (i % RF) * 16 + r) * 16;
#pragma unroll
            for (int t = 0; t < 8; ++t) *reinterpret_cast<v4i*>(to + t * 4 * R * 16) = f[t];
#pragma unroll
            for (int j = 0; j < 8; ++j) now[j] = next[j];
        }
    }
    __syncthreads();
    const unsigned char* mine = rows + (g * R + r) * 16;
    for (; key0 < end; key0 += 16 * W) {
        const int next0 = key0 + 16 * W;
        const size_t off_next = next0 < end ? locate(next0) : off;
        v4i acc[RF][8];
#pragma unroll
        for (int i = 0; i < RF; ++i)
#pragma unroll
            for (int s = 0; s < 8; ++s) acc[i][s] = v4i{0, 0, 0, 0};
        for (int kb = 0; kb < blocks; ++kb) {
            v4i f[8];
            to_units(w, f);
            __builtin_amdgcn_sched_barrier(0);
            const bool last = kb + 1 == blocks;
            load(last ? off_next : off, last ? 0 : kb + 1, w);
            multiply_block<RF>(acc, f, mine + (size_t)kb * (R * 512));
        }
        off = off_next;
        write_out<RF>(p, tile, acc, key0, lane);
    }
}

// What a wavefront of scores_many_kernel reads: its row of E or A, its 16 keys.
struct Source {
    const u64* rows;
    const char *X, *F;             // the keys' rows of the head
    int d, g;
    u32 lane_at, bytes;
    template <int J, int N>
    __device__ __forceinline__ void row(int blk, u64x2 (&w)[N]) const { load_row<J>(rows, 64 * blk, d, g, w); }
    template <int J, int N>
    __device__ __forceinline__ void clear(int blk, u64x2 (&w)[N]) const {
        if (64 * blk + 64 > d) clear_beyond<J>(w, 64 * blk, d, g);
    }
    __device__ __forceinline__ void column(int h, int blk, u64x2 (&v)[8]) const {
        const u32 at = (u32)blk * 512u;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>((h ? F : X) + at), 0, (int)(bytes - at), 0x00027000);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] = __builtin_bit_cast(u64x2, __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane_at + 64 * j, 0, 0));
    }
};

// Rows whose digits do not fit LDS: 16 RF rows x 16 W keys, the contraction streamed (sweep_blocks).
template <int RF, int W>
__global__ __launch_bounds__(64 * W) void scores_many_kernel(ProductParams p) {
    constexpr int R = 16 * RF, HALF = R * 512;
    __shared__ __align__(16) unsigned char stage[4 * HALF];
    __shared__ RowTile<R> tile;
    const Batch& b = p.b;
    const Unit unit(p, R);
    if (!unit.live) return;
    const Sequence sq(b, unit.s);
    if (!p.takes(sq) || (int64_t)unit.tile * R >= sq.rows(b)) return;
    tile.fill(b, sq, unit.kvh, unit.tile * R);
    __syncthreads();
    int most, least;
    tile.span(most, least);
    if (unit.chunk * p.chunk >= most) return;

    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int key0 = unit.chunk * p.chunk + 16 * wave;        // (a chunk is 16 W keys)
    const bool works = key0 < most, feeds = wave < 2 * RF;
    const int ch = (wave / RF) & 1, cr = (wave % RF) * 16 + r, row = tile.row[cr] < 0 ? 0 : tile.row[cr];
    const u32 row_bytes = (u32)(b.n_kv_heads * p.ldp) * 8u, head_at = (u32)(unit.kvh * p.ldp) * 8u;
    const size_t off = works ? (size_t)(u32)__builtin_amdgcn_readfirstlane((int)sq.slot(b, key0)) * row_bytes + head_at : 0;
    const Source src = {(ch ? p.A : p.E) + (size_t)row * p.d, reinterpret_cast<const char*>(p.X) + off,
                        reinterpret_cast<const char*>(p.F) + off, p.d, g, (u32)r * row_bytes + (u32)g * 16u,
                        16u * row_bytes - head_at};
    unsigned char* const put_at = stage + ch * HALF + (g * R + cr) * 16;
    const unsigned char* const get_at = stage + (g * R + r) * 16;
    v4i acc[RF][8];
#pragma unroll
    for (int i = 0; i < RF; ++i)
#pragma unroll
        for (int s = 0; s < 8; ++s) acc[i][s] = v4i{0, 0, 0, 0};
    auto sweep = [&]<bool WORKS, bool FEEDS, bool LATE>() {
        sweep_blocks<RF, 2, WORKS, FEEDS, LATE>(acc, src, (p.d + 63) / 64, 0, 0, put_at, get_at);
    };
    if (wave < 4) {                                           // (these feed, whatever RF is)
        if (works) sweep.template operator()<true, true, false>();
        else sweep.template operator()<false, true, false>();
    } else if (feeds) {
        if (works) sweep.template operator()<true, true, true>();
        else sweep.template operator()<false, true, true>();
    } else {
        if (works) sweep.template operator()<true, false, true>();
        else sweep.template operator()<false, false, true>();
    }
    if (works) write_out<RF>(p, tile, acc, key0, lane);
}

}  // namespace

static int launch_part(comet_ctx* ctx, const char* what, ProductParams& p, int max_q) {
    const Batch& b = p.b;
    const int blocks = (p.d + 63) / 64 * 2;
    const int64_t n_rows = (int64_t)max_q * b.group;
    int R, W;
    void (*kern)(ProductParams);
    // d > 256: the rows' digits would fill LDS (and 16 rows of them would leave one workgroup on a compute unit): the contraction is
    // streamed, with tiles of 64 x 128 where there is one for every compute unit, smaller ones, of which a compute unit holds several,
    // below.  576 words, when this was settled: 37 tokens of 64 heads over 2037 keys 273 us (32 x 64: 313; resident rows 807), one token of 64 heads of 4
    // sequences of 4000 keys 69 us (64 x 128: 131), of 16 heads 39 us (resident 64).
    // d <= 256: resident rows (192 words, 512 tokens of 32 heads: 115 us, streamed 197; d = 128: 151 and 172).
    p.tiles = (int)((n_rows + 63) / 64);
    const int64_t units64 = filled_tiles(p, 64) * b.n_kv_heads;
    // Resident rows: tiles of 64, of which a compute unit holds one, where there is one for each or the keys make several pieces of
    // each; else 32, of which it holds two (100 tokens of 32/8 heads of 128: 12 us, with 64 21; 200 tokens of 40 heads 32 and 42;
    // 64 tokens of 32 heads over 1000 keys 30.5 and 27.5).
    const bool wide = n_rows > 32 && (units64 > ctx->num_cu || b.kv_cap >= 1024);
    if (blocks > 8) {
        const bool large = n_rows > 32 && units64 * ((b.kv_cap + 127) / 128) >= ctx->num_cu;
        if (large) { kern = scores_many_kernel<4, 8>; R = 64; W = 8; }
        else { kern = n_rows > 16 ? scores_many_kernel<2, 4> : scores_many_kernel<1, 4>; R = n_rows > 16 ? 32 : 16; W = 4; }
    }
    else if (wide && blocks <= 2) { kern = scores_kernel<4, 2, 256>; R = 64; W = 4; }
    else if (wide && blocks <= 4) { kern = scores_kernel<4, 4, 512>; R = 64; W = 8; }
    else if (n_rows > 16 && blocks <= 4) { kern = scores_kernel<2, 4, 256>; R = 32; W = 4; }
    else if (n_rows > 16) { kern = scores_kernel<2, 8, 512>; R = 32; W = 8; }
    else if (blocks <= 4) { kern = scores_kernel<1, 4, 256>; R = 16; W = 4; }
    else { kern = scores_kernel<1, 8, 512>; R = 16; W = 8; }
    p.tiles = (int)((n_rows + R - 1) / R);
    const int64_t tokens = R / b.group + 2 < b.max_q ? R / b.group + 2 : b.max_q;    // that a tile of rows may touch
    p.far_rows = tokens * b.n_heads * b.ld * 8 >= 0x7fffffffll;
    // Enough workgroups to fill the chip several times over (sequences differ in length), each with a tile of keys per
    // wavefront at least.
    const int64_t units = filled_tiles(p, R) * b.n_kv_heads, wanted = (blocks <= 4 && R == 16 ? 32ll : 2ll) * ctx->num_cu;
    int64_t chunks = (wanted + units - 1) / units;
    const int64_t most = (b.kv_cap + 16 * W - 1) / (16 * W);
    if (chunks > most || blocks > 8) chunks = most;
    if (chunks < 1) chunks = 1;
    p.chunk = (int)(((b.kv_cap + chunks - 1) / chunks + 16 * W - 1) / (16 * W) * (16 * W));
    p.chunks = (b.kv_cap + p.chunk - 1) / p.chunk;
    return launch_all(ctx, what, kern, Unit::grid(p, R), 64 * W, p);
}

int comet_attn::launch_scores(comet_ctx* ctx, const char* what, ProductParams& p) {
    return launch_split(p, [&](int max_q) { return launch_part(ctx, what, p, max_q); });
}
