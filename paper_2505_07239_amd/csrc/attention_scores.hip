// Queries times cached keys (comet_attention_scores) on the int8 matrix cores:
//     Z(r, j) = t(C(r, j) + [E | A](r, :) . [X | F](j, :)) - M(r, j).
//
// A workgroup holds R = 16 RF rows in LDS, as digits, for the whole stacked contraction (E and A, each filled up to whole blocks of 64 words); behind
// the barrier that follows, its wavefronts are on their own.  Each takes every W-th tile of 16 keys: it loads its keys' words
// straight into registers, a block of 64 words ahead of their use, splits them into digits and transposes them there (no
// other wavefront of the workgroup wants them), and multiplies them with the rows' digits, read from LDS in operand
// order.  So a cached word is fetched once per row tile, a query word once per workgroup, and while one
// wavefront of a SIMD writes its tile out the other multiplies.
#include "attention_tile.h"

using namespace comet_attn;

namespace {

// KT: blocks of 64 words that fit the rows' place in LDS.  NT: threads.
template <int RF, int KT, int NT>
__global__ __launch_bounds__(NT, RF == 1 && KT <= 8 ? 4 : 2) void scores_kernel(ProductParams p) {
    constexpr int R = 16 * RF, W = NT / 64, AHEAD = KT > 8 ? 2 : 1;
    __shared__ __align__(16) unsigned char rows[KT * R * 512];
    __shared__ RowTile<R> tile;
    const Batch& b = p.b;
    const Unit unit(b, p.tiles, p.chunks);
    if (!unit.live) return;
    const Sequence sq(b, unit.s);
    const int kvh = unit.kvh;
    const int rt = p.tiles - 1 - unit.inner;       // (the rows that see most come first)
    const int r0 = rt * R;
    if (r0 >= sq.nq * b.group) return;
    tile.fill(b, sq, kvh, r0);
    __syncthreads();
    int most, least;
    tile.span(most, least);
    const int first = unit.chunk * p.chunk;
    const int end = most < first + p.chunk ? most : first + p.chunk;
    if (first >= end) return;

    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int d = p.d, half = (d + 63) / 64, blocks = 2 * half;

    // the rows' digits: block kb, digit t, lane group g, row
    for (int i = wave; i < blocks * RF; i += W) {
        const int kb = i / RF, rr = (i % RF) * 16 + r;
        const int row = tile.row[rr];
        const u64* const src = (kb < half ? p.E : p.A) + (size_t)(row < 0 ? 0 : row) * d;
        u64x2 w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int k = 64 * (kb < half ? kb : kb - half) + 8 * j + 2 * g;
            w[j] = u64x2{0, 0};
            if (row >= 0 && k < d) w[j] = *reinterpret_cast<const u64x2*>(src + k);
        }
        v4i f[8];
        to_units(w, f);
#pragma unroll
        for (int t = 0; t < 8; ++t) *reinterpret_cast<v4i*>(rows + ((size_t)((kb * 8 + t) * 4 + g) * R + rr) * 16) = f[t];
    }
    __syncthreads();

    // A tile's 16 keys lie in one page: a uniform address, and one offset per lane.  Buffer loads that end with the page's 16
    // rows: the last block may reach beyond d, where the rows' digits are zero, but never beyond the pool.
    const u32 row_bytes = (u32)(b.n_kv_heads * p.ldp) * 8u, head_at = (u32)(kvh * p.ldp) * 8u;
    const u32 lane_at = (u32)r * row_bytes + (u32)g * 16u, bytes = 16u * row_bytes - head_at;
    auto locate = [&](int key0) {
        return (size_t)(u32)__builtin_amdgcn_readfirstlane((int)sq.slot(b, key0)) * row_bytes + head_at;
    };
    auto load = [&](size_t off, int kb, u64x2 (&w)[8]) {
        const u32 at = (u32)(kb < half ? kb : kb - half) * 512u;
        const char* const pool = reinterpret_cast<const char*>(kb < half ? p.X : p.F) + off + at;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(pool), 0, (int)(bytes - at), 0x00027000);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            w[j] = __builtin_bit_cast(u64x2, __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane_at + 64 * j, 0, 0));
    };

    int key0 = first + 16 * wave;
    if (key0 >= end) return;
    size_t off = locate(key0);
    u64x2 w[AHEAD][8];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) load(off, n, w[n]);       // (there are two blocks at least)
    const unsigned char* mine = rows + (g * R + r) * 16;
    for (; key0 < end; key0 += 16 * W) {
        const int next0 = key0 + 16 * W;
        const size_t off_next = next0 < end ? locate(next0) : off;
        v4i acc[RF][8];
#pragma unroll
        for (int i = 0; i < RF; ++i)
#pragma unroll
            for (int s = 0; s < 8; ++s) acc[i][s] = v4i{0, 0, 0, 0};
        for (int kb0 = 0; kb0 < blocks; kb0 += AHEAD) {       // (blocks is even, AHEAD one or two)
#pragma unroll
            for (int n = 0; n < AHEAD; ++n) {
                v4i f[8];
                to_units(w[n], f);
                __builtin_amdgcn_sched_barrier(0);
                const int kb = kb0 + n, then = kb + AHEAD;
                const bool over = then >= blocks;
                load(over ? off_next : off, over ? then - blocks : then, w[n]);
                multiply_block<RF>(acc, f, mine + (size_t)kb * (R * 512));
            }
        }
        off = off_next;
        // the loads of several rows first: Z may be C or M, so the compiler would wait for every store before the next load
        constexpr int BATCH = RF < 2 ? RF : 2;
        const int key = key0 + r;
#pragma unroll
        for (int i0 = 0; i0 < RF; i0 += BATCH) {
            size_t at[BATCH][4];
            bool live[BATCH][4];
            u64 c[BATCH][4], m[BATCH][4];
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int rr = 16 * (i0 + i) + 4 * g + e;
                    live[i][e] = key < tile.sees[rr];
                    at[i][e] = live[i][e] ? (size_t)tile.row[rr] * b.ld + key : 0;
                    c[i][e] = __builtin_nontemporal_load(p.C + at[i][e]);
                    m[i][e] = p.M ? __builtin_nontemporal_load(p.M + at[i][e]) : 0;
                }
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (live[i][e]) __builtin_nontemporal_store(rescale(p.party, c[i][e] + word_of(acc[i0 + i], e), p.frac) - m[i][e], p.Z + at[i][e]);
        }
    }
}

}  // namespace

int comet_attn::launch_scores(comet_ctx* ctx, const char* what, ProductParams& p) {
    const Batch& b = p.b;
    const int blocks = (p.d + 63) / 64 * 2;
    const int64_t n_rows = (int64_t)b.max_q * b.group;
    int R, W;
    void (*kern)(ProductParams);
    if (n_rows > 32 && blocks <= 4) { kern = scores_kernel<4, 4, 512>; R = 64; W = 8; }
    else if (n_rows > 16 && blocks <= 8) { kern = scores_kernel<2, 8, 512>; R = 32; W = 8; }
    else if (blocks <= 4) { kern = scores_kernel<1, 4, 256>; R = 16; W = 4; }
    else if (blocks <= 8) { kern = scores_kernel<1, 8, 512>; R = 16; W = 8; }
    else { kern = scores_kernel<1, 18, 768>; R = 16; W = 12; }
    p.tiles = (int)((n_rows + R - 1) / R);
    // Enough workgroups to fill the chip several times over (sequences differ in length), each with a tile of keys per
    // wavefront at least.
    const int64_t units = (int64_t)b.n_seq * b.n_kv_heads * p.tiles, wanted = (W == 4 ? 32ll : 2ll) * ctx->num_cu;
    int64_t chunks = (wanted + units - 1) / units;
    const int64_t most = (b.kv_cap + 16 * W - 1) / (16 * W);
    if (chunks > most) chunks = most;
    if (chunks < 1) chunks = 1;
    p.chunk = (int)(((b.kv_cap + chunks - 1) / chunks + 16 * W - 1) / (16 * W) * (16 * W));
    p.chunks = (b.kv_cap + p.chunk - 1) / p.chunk;
    const int64_t grid = Unit::grid(b, p.tiles, p.chunks);
    if (grid > 0x7fffffffll) return comet_fail(ctx, COMET_ECAP, "%s: too many rows", what);
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(64 * W), 0, ctx->stream, p);
    COMET_LAUNCH_CHECK(ctx, what);
    return COMET_OK;
}
