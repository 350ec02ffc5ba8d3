// Queries times cached keys (comet_attention_scores) on the int8 matrix cores:
//     Z(r, j) = t(C(r, j) + [E | A](r, :) . [X | F](j, :)) - M(r, j).
//
// A workgroup holds R = 16 RF rows in LDS, as digits, for the whole stacked contraction of 2 d words; behind
// the barrier that follows, its wavefronts are on their own.  Each takes every W-th tile of 16 keys: it loads its keys' words
// straight into registers, a block of 64 ahead of their use, splits them into digits and transposes them there (no
// other wavefront of the workgroup wants them), and multiplies them with the rows' digits, read from LDS in operand
// order.  So a cached word is fetched once per row tile, a query word once per workgroup, and while one
// wavefront of a SIMD writes its tile out the other multiplies.
#include "attention_tile.h"

using namespace comet_attn;

namespace {

// KT: blocks of 64 words that fit the rows' place in LDS.  NT: threads.
template <int RF, int KT, int NT>
__global__ __launch_bounds__(NT) void scores_kernel(ProductParams p) {
    constexpr int R = 16 * RF, W = NT / 64;
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
    const int d = p.d, blocks = (2 * d + 63) / 64;

    // the rows' digits: block kb, digit t, lane group g, row
    for (int i = wave; i < blocks * RF; i += W) {
        const int kb = i / RF, rr = (i % RF) * 16 + r;
        const int row = tile.row[rr];
        u64x2 w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int k = 64 * kb + 8 * j + 2 * g;
            w[j] = u64x2{0, 0};
            if (row >= 0 && k < 2 * d)
                w[j] = *reinterpret_cast<const u64x2*>((k < d ? p.E + k : p.A + (k - d)) + (size_t)row * d);
        }
        v4i f[8];
        to_units(w, f);
#pragma unroll
        for (int t = 0; t < 8; ++t) *reinterpret_cast<v4i*>(rows + ((size_t)((kb * 8 + t) * 4 + g) * R + rr) * 16) = f[t];
    }
    __syncthreads();

    // word offset of the lane's key of a tile (16 keys lie in one page)
    const size_t stride = (size_t)b.n_kv_heads * p.ldp;
    auto locate = [&](int key0) { return (sq.slot(b, key0) + r) * stride + (size_t)kvh * p.ldp; };
    auto load = [&](size_t off, int kb, u64x2 (&w)[8]) {
        const int k0 = 64 * kb;
        if (k0 + 64 <= d || (k0 >= d && k0 + 64 <= 2 * d)) {
            const u64* src = (k0 < d ? p.X + k0 : p.F + (k0 - d)) + off + 2 * g;
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = *reinterpret_cast<const u64x2*>(src + 8 * j);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                int k = k0 + 8 * j + 2 * g;
                k = k < 2 * d ? k : 2 * d - 2;               // (the rows' digits are zero there)
                w[j] = *reinterpret_cast<const u64x2*>((k < d ? p.X + k : p.F + (k - d)) + off);
            }
        }
    };

    int key0 = first + 16 * wave;
    if (key0 >= end) return;
    size_t off = locate(key0);
    u64x2 w[8];
    load(off, 0, w);
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
            if (kb + 1 < blocks) load(off, kb + 1, w);
            else load(off_next, 0, w);
            multiply_block<RF>(acc, f, mine + (size_t)kb * (R * 512));
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
                    c[i][e] = p.C[at[i][e]];
                    m[i][e] = p.M ? p.M[at[i][e]] : 0;
                }
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (live[i][e]) p.Z[at[i][e]] = rescale(p.party, c[i][e] + word_of(acc[i0 + i], e), p.frac) - m[i][e];
        }
    }
}

}  // namespace

int comet_attn::launch_scores(comet_ctx* ctx, const char* what, ProductParams& p) {
    const Batch& b = p.b;
    const int blocks = (2 * p.d + 63) / 64;
    const int64_t n_rows = (int64_t)b.max_q * b.group;
    int R, W;
    void (*kern)(ProductParams);
    if (n_rows > 32 && blocks <= 4) { kern = scores_kernel<4, 4, 512>; R = 64; W = 8; }
    else if (n_rows > 16 && blocks <= 9) { kern = scores_kernel<2, 9, 512>; R = 32; W = 8; }
    else if (blocks <= 4) { kern = scores_kernel<1, 4, 256>; R = 16; W = 4; }
    else if (blocks <= 9) { kern = scores_kernel<1, 9, 512>; R = 16; W = 8; }
    else { kern = scores_kernel<1, 19, 1024>; R = 16; W = 16; }
    p.tiles = (int)((n_rows + R - 1) / R);
    // Enough workgroups to fill the chip several times over (sequences differ in length), each with a tile of keys per
    // wavefront at least.
    const int64_t units = (int64_t)b.n_seq * b.n_kv_heads * p.tiles, wanted = (W == 4 ? 8ll : 2ll) * ctx->num_cu;
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
