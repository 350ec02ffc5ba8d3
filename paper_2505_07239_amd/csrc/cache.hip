// Local steps around attention over a cache of shares: rows opened into the pools, rows read back as operands of a share
// product, position rotation with rescaling and masking.  All of them are bound by HBM bandwidth, or, for the tokens of a
// decoding step, by the launch: 2048 rows of 5120 words written in 71 us (5.9 TB/s; 79 through the caches), 6000 rows of 576 read in
// 20 us (5.5 TB/s), 2048 tokens of 40 heads of 128 rotated in 43 us (5.8 TB/s; 50 one word at a time), one token 2.6 us (3.7 a call).
#include "kv_batch.h"

using comet_attn::rescale;

namespace {

constexpr int GT = 256;
typedef u64 u64x2 __attribute__((ext_vector_type(2)));

template <int VEC> struct Word;
template <> struct Word<1> { typedef u64 type; };
template <> struct Word<2> { typedef u64x2 type; };

// Everything here is read and written once: past the caches.
template <class V>
__device__ __forceinline__ V past(const u64* p, size_t i) { return __builtin_nontemporal_load(reinterpret_cast<const V*>(p) + i); }
template <class V>
__device__ __forceinline__ void put(u64* p, size_t i, V v) { __builtin_nontemporal_store(v, reinterpret_cast<V*>(p) + i); }

// Which part of which row a workgroup's thread has: rows of many vectors are cut into pieces, narrow ones share a workgroup
// (2^log lanes each).
struct RowPart {
    int t, first, step;
    __device__ __forceinline__ RowPart(int pieces, int log) {
        if (log < 8) {
            t = (int)(blockIdx.x << (8 - log)) + ((int)threadIdx.x >> log);
            first = (int)threadIdx.x & ((1 << log) - 1);
            step = 1 << log;
        } else {
            t = (int)(blockIdx.x / (unsigned)pieces);
            first = (int)(blockIdx.x % (unsigned)pieces) * GT + (int)threadIdx.x;
            step = pieces * GT;
        }
    }
};

// One thread per VEC words of a row: F = d_0 + d_1 and X = b + party * F at the token's slot.
template <int VEC>
__global__ __launch_bounds__(GT) void cache_write_kernel(int party, const u64* __restrict__ d0, const u64* __restrict__ d1,
                                                         const u64* __restrict__ b, const int* __restrict__ slots,
                                                         int n_tok, int nvec, u64* __restrict__ f_pool,
                                                         u64* __restrict__ x_pool, int n_slots, int pieces, int log) {
    typedef typename Word<VEC>::type V;
    const RowPart part(pieces, log);
    if (part.t >= n_tok) return;
    const int slot = slots[part.t];
    if (slot < 0 || slot >= n_slots) return;
    const size_t from = (size_t)part.t * nvec, to = (size_t)slot * nvec;
    for (int c = part.first; c < nvec; c += part.step) {
        const V f = past<V>(d0, from + c) + past<V>(d1, from + c), x = past<V>(b, from + c);
        put<V>(f_pool, to + c, f);
        put<V>(x_pool, to + c, party ? x + f : x);
    }
}

template <int VEC>
__global__ __launch_bounds__(GT) void cache_read_kernel(int party, const u64* __restrict__ f_pool,
                                                        const u64* __restrict__ x_pool, const int* __restrict__ slots,
                                                        int n_tok, int nvec, u64* __restrict__ e, u64* __restrict__ a,
                                                        int n_slots, int pieces, int log) {
    typedef typename Word<VEC>::type V;
    const RowPart part(pieces, log);
    if (part.t >= n_tok) return;
    const int slot = slots[part.t];
    if (slot < 0 || slot >= n_slots) return;
    const size_t to = (size_t)part.t * nvec, from = (size_t)slot * nvec;
    for (int c = part.first; c < nvec; c += part.step) {
        const V f = past<V>(f_pool, from + c), x = past<V>(x_pool, from + c);
        put<V>(e, to + c, f);
        put<V>(a, to + c, party ? x - f : x);
    }
}

struct RotateParams {
    int party, n_heads, head_dim, half, interleaved, shift, frac;
    long ldx;
    long n_pos;
    const u64* x;
    const int* pos;
    const u64* cos_t;
    const u64* sin_t;
    const u64* m;
    u64* out;
    int units;             // per token: vectors of pairs and of words that are not rotated
};

// One thread per VEC pairs, or VEC words that are not rotated.
template <int VEC, bool INTERLEAVED>
__global__ __launch_bounds__(GT) void rotate_kernel(RotateParams p, int pieces) {
    typedef typename Word<VEC>::type V;
    const int t = (int)(blockIdx.x / (unsigned)pieces), piece = (int)(blockIdx.x % (unsigned)pieces);
    const int pairs = p.half / VEC, per_head = pairs + (p.head_dim - 2 * p.half) / VEC;
    const u64* const x = p.x + (size_t)t * p.ldx;
    const size_t row = (size_t)t * p.n_heads * p.head_dim;
    const u64* const m = p.m ? p.m + row : nullptr;
    u64* const out = p.out + row;
    long at = p.half ? p.pos[t] : 0;
    if (at < 0 || at >= p.n_pos) at = 0;
    const u64* const cos_t = p.cos_t + (size_t)at * p.half;
    const u64* const sin_t = p.sin_t + (size_t)at * p.half;
    auto scaled = [&](V v, int f) {
        if constexpr (VEC == 1) return rescale(p.party, v, f);
        else return V{rescale(p.party, v.x, f), rescale(p.party, v.y, f)};
    };
    for (int i = piece * GT + threadIdx.x; i < p.units; i += pieces * GT) {
        const int h = i / per_head, j = i - h * per_head;
        const int base = h * p.head_dim;
        if (j < pairs) {
            // the words p and q of VEC pairs, as vectors of consecutive words: (p, p + 1), (q, q + 1) or (p, q), (p', q')
            const int a = base + (INTERLEAVED ? 2 * VEC * j : VEC * j), b = a + (INTERLEAVED ? VEC : p.half);
            const V c = *reinterpret_cast<const V*>(cos_t + VEC * j), s = *reinterpret_cast<const V*>(sin_t + VEC * j);
            V xa = scaled(past<V>(x + a, 0), p.shift), xb = scaled(past<V>(x + b, 0), p.shift);
            if constexpr (INTERLEAVED && VEC == 2) {
                const V ya = xa, yb = xb;
                xa = V{ya.x, yb.x};
                xb = V{ya.y, yb.y};
            }
            V ya = scaled(xa * c - xb * s, p.frac), yb = scaled(xb * c + xa * s, p.frac);
            if constexpr (INTERLEAVED && VEC == 2) {
                const V za = ya, zb = yb;
                ya = V{za.x, zb.x};
                yb = V{za.y, zb.y};
            }
            if (m) {
                ya -= past<V>(m + a, 0);
                yb -= past<V>(m + b, 0);
            }
            put<V>(out + a, 0, ya);
            put<V>(out + b, 0, yb);
        } else {
            const int a = base + 2 * p.half + VEC * (j - pairs);
            V y = scaled(past<V>(x + a, 0), p.shift);
            if (m) y -= past<V>(m + a, 0);
            put<V>(out + a, 0, y);
        }
    }
}

// workgroups that share a row of n units (a launch has fewer than 2^32 threads: 2^24 workgroups)
inline int row_pieces(int64_t n_tok, int64_t n, int per_thread) {
    int64_t g = (n + (int64_t)GT * per_thread - 1) / ((int64_t)GT * per_thread);
    if (g > 64) g = 64;
    if (g * n_tok > COMET_DIM_MAX) g = COMET_DIM_MAX / n_tok;
    return (int)(g < 1 ? 1 : g);
}

// lanes of a row, as a power of two: a whole workgroup (8) for rows of more than 128 vectors
inline int row_log(int64_t n) {
    int log = 3;
    while (log < 8 && (1 << log) < n) ++log;
    return log;
}
inline unsigned row_grid(int64_t n_tok, int pieces, int log) {
    return (unsigned)(log < 8 ? (n_tok + (GT >> log) - 1) >> (8 - log) : n_tok * pieces);
}

int check_rows(comet_ctx* ctx, const char* what, int party, const void* const (&ptrs)[5], const int32_t* slots, int64_t n_tok,
               int64_t width, int64_t n_slots) {
    if (party != 0 && party != 1) return comet_fail(ctx, COMET_EINVAL, "%s: party must be 0 or 1", what);
    if (n_tok < 0 || width < 0 || n_slots < 0) return comet_fail(ctx, COMET_EINVAL, "%s: bad size", what);
    if (n_tok > COMET_DIM_MAX || width > COMET_DIM_MAX || n_slots > 0x7fffffffll)
        return comet_fail(ctx, COMET_ECAP, "%s: n_tok and width must stay below 2^24, n_slots below 2^31", what);
    if (n_tok == 0 || width == 0 || n_slots == 0) return COMET_OK;
    if (!slots) return comet_fail(ctx, COMET_EINVAL, "%s: null pointer", what);
    for (const void* q : ptrs) {
        if (!q) return comet_fail(ctx, COMET_EINVAL, "%s: null pointer", what);
        if (!comet_aligned16(q)) return comet_fail(ctx, COMET_EALIGN, "%s: operands must be 16-byte aligned", what);
    }
    return COMET_OK;
}

}  // namespace

extern "C" {

int comet_cache_write(comet_ctx* ctx, int party, const uint64_t* d_0, const uint64_t* d_1, const uint64_t* b_i,
                      const int32_t* slots, int64_t n_tok, int64_t width, uint64_t* f_pool, uint64_t* x_pool, int64_t n_slots) {
    const char* what = "comet_cache_write";
    COMET_CHECK_CTX(ctx);
    const int rc = check_rows(ctx, what, party, {d_0, d_1, b_i, f_pool, x_pool}, slots, n_tok, width, n_slots);
    if (rc != COMET_OK || n_tok == 0 || width == 0 || n_slots == 0) return rc;
    if (f_pool == x_pool) return comet_fail(ctx, COMET_EINVAL, "%s: the pools must not be one buffer", what);
    comet_device_guard guard(ctx);
    if (!guard.ok) return comet_fail(ctx, COMET_EDEVICE, "%s: cannot select device", what);
    const bool vec = (width & 1) == 0;
    const int nvec = (int)(vec ? width / 2 : width), pieces = row_pieces(n_tok, nvec, 2), log = row_log(nvec);
    const dim3 grid(row_grid(n_tok, pieces, log));
    auto kern = vec ? cache_write_kernel<2> : cache_write_kernel<1>;
    hipLaunchKernelGGL(kern, grid, dim3(GT), 0, ctx->stream, party, (const u64*)d_0, (const u64*)d_1, (const u64*)b_i, slots,
                       (int)n_tok, nvec, (u64*)f_pool, (u64*)x_pool, (int)n_slots, pieces, log);
    COMET_LAUNCH_CHECK(ctx, what);
    return COMET_OK;
}

int comet_cache_read(comet_ctx* ctx, int party, const uint64_t* f_pool, const uint64_t* x_pool, const int32_t* slots,
                     int64_t n_tok, int64_t width, int64_t n_slots, uint64_t* e, uint64_t* a_i) {
    const char* what = "comet_cache_read";
    COMET_CHECK_CTX(ctx);
    const int rc = check_rows(ctx, what, party, {f_pool, x_pool, e, a_i, e}, slots, n_tok, width, n_slots);
    if (rc != COMET_OK || n_tok == 0 || width == 0 || n_slots == 0) return rc;
    if (e == a_i) return comet_fail(ctx, COMET_EINVAL, "%s: e and a_i must not be one buffer", what);
    comet_device_guard guard(ctx);
    if (!guard.ok) return comet_fail(ctx, COMET_EDEVICE, "%s: cannot select device", what);
    const bool vec = (width & 1) == 0;
    const int nvec = (int)(vec ? width / 2 : width), pieces = row_pieces(n_tok, nvec, 2), log = row_log(nvec);
    const dim3 grid(row_grid(n_tok, pieces, log));
    auto kern = vec ? cache_read_kernel<2> : cache_read_kernel<1>;
    hipLaunchKernelGGL(kern, grid, dim3(GT), 0, ctx->stream, party, (const u64*)f_pool, (const u64*)x_pool, slots,
                       (int)n_tok, nvec, (u64*)e, (u64*)a_i, (int)n_slots, pieces, log);
    COMET_LAUNCH_CHECK(ctx, what);
    return COMET_OK;
}

int comet_rotate_share(comet_ctx* ctx, int party, const uint64_t* x_i, int64_t ldx, const int32_t* positions,
                       const uint64_t* cos_t, const uint64_t* sin_t, int64_t n_pos, int64_t n_tok, int n_heads, int head_dim,
                       int rot_dim, int interleaved, int shift, int frac_bits, const uint64_t* m_i, uint64_t* out) {
    const char* what = "comet_rotate_share";
    COMET_CHECK_CTX(ctx);
    if ((party != 0 && party != 1) || shift < 0 || shift > 62 || frac_bits < 0 || frac_bits > 62)
        return comet_fail(ctx, COMET_EINVAL, "%s: party must be 0 or 1, 0 <= shift, frac_bits <= 62", what);
    if (n_tok < 0 || n_heads < 1 || head_dim < 1 || rot_dim < 0 || rot_dim > head_dim || (rot_dim & 1))
        return comet_fail(ctx, COMET_EINVAL, "%s: bad size (rot_dim must be even and at most head_dim)", what);
    const int64_t width = (int64_t)n_heads * head_dim;
    if (n_tok > COMET_DIM_MAX || width > COMET_DIM_MAX || n_pos > 0x7fffffffll)
        return comet_fail(ctx, COMET_ECAP, "%s: n_tok and n_heads * head_dim must stay below 2^24, n_pos below 2^31", what);
    if (ldx < width) return comet_fail(ctx, COMET_EINVAL, "%s: ldx must be at least n_heads * head_dim", what);
    if (n_tok == 0) return COMET_OK;
    if (!x_i || !out || (rot_dim > 0 && (!positions || !cos_t || !sin_t || n_pos < 1)))
        return comet_fail(ctx, COMET_EINVAL, "%s: null pointer or empty table", what);
    if (x_i == out) return comet_fail(ctx, COMET_EINVAL, "%s: out must not alias x_i", what);
    if ((reinterpret_cast<uintptr_t>(x_i) & 7u) != 0 || !comet_aligned16(out) || (m_i && !comet_aligned16(m_i)) ||
        (rot_dim > 0 && (!comet_aligned16(cos_t) || !comet_aligned16(sin_t))))
        return comet_fail(ctx, COMET_EALIGN, "%s: operands must be 16-byte aligned (x_i: 8)", what);
    comet_device_guard guard(ctx);
    if (!guard.ok) return comet_fail(ctx, COMET_EDEVICE, "%s: cannot select device", what);
    RotateParams p;
    p.party = party; p.n_heads = n_heads; p.head_dim = head_dim; p.half = rot_dim / 2; p.interleaved = interleaved != 0;
    p.shift = shift; p.frac = frac_bits; p.ldx = ldx; p.n_pos = n_pos;
    p.x = (const u64*)x_i; p.pos = positions; p.cos_t = (const u64*)cos_t; p.sin_t = (const u64*)sin_t;
    p.m = (const u64*)m_i; p.out = (u64*)out;
    // two words at a time where every vector of a head, of the table and of x_i starts on 16 bytes
    const bool vec = (head_dim & 1) == 0 && (p.half & 1) == 0 && (ldx & 1) == 0 && comet_aligned16(x_i);
    p.units = n_heads * (head_dim - p.half) / (vec ? 2 : 1);
    const int pieces = row_pieces(n_tok, p.units, 1);
    auto kern = vec ? (p.interleaved ? rotate_kernel<2, true> : rotate_kernel<2, false>)
                    : (p.interleaved ? rotate_kernel<1, true> : rotate_kernel<1, false>);
    hipLaunchKernelGGL(kern, dim3((unsigned)(n_tok * pieces)), dim3(GT), 0, ctx->stream, p, pieces);
    COMET_LAUNCH_CHECK(ctx, what);
    return COMET_OK;
}

}  // extern "C"
