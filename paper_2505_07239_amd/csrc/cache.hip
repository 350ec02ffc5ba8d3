// Local steps around attention over a cache of shares: rows opened into the pools, rows read back as operands of a share
// product, position rotation with rescaling and masking.  All of them are bound by HBM bandwidth, or, for the tokens of a
// decoding step, by the launch.
#include "common.h"

namespace {

constexpr int GT = 256;
typedef u64 u64x2 __attribute__((ext_vector_type(2)));

template <int VEC> struct Word;
template <> struct Word<1> { typedef u64 type; };
template <> struct Word<2> { typedef u64x2 type; };

// One thread per VEC words of a row: F = d_0 + d_1 and X = b + party * F at the token's slot.
template <int VEC>
__global__ __launch_bounds__(GT) void cache_write_kernel(int party, const u64* __restrict__ d0, const u64* __restrict__ d1,
                                                         const u64* __restrict__ b, const int* __restrict__ slots,
                                                         int nvec, u64* __restrict__ f_pool, u64* __restrict__ x_pool,
                                                         int n_slots, int pieces) {
    typedef typename Word<VEC>::type V;
    const int t = (int)(blockIdx.x / (unsigned)pieces), piece = (int)(blockIdx.x % (unsigned)pieces);
    const int slot = slots[t];
    if (slot < 0 || slot >= n_slots) return;
    const size_t from = (size_t)t * nvec, to = (size_t)slot * nvec;
    for (int c = piece * GT + threadIdx.x; c < nvec; c += pieces * GT) {
        const V f = reinterpret_cast<const V*>(d0)[from + c] + reinterpret_cast<const V*>(d1)[from + c];
        const V x = reinterpret_cast<const V*>(b)[from + c];
        reinterpret_cast<V*>(f_pool)[to + c] = f;
        reinterpret_cast<V*>(x_pool)[to + c] = party ? x + f : x;
    }
}

template <int VEC>
__global__ __launch_bounds__(GT) void cache_read_kernel(int party, const u64* __restrict__ f_pool,
                                                        const u64* __restrict__ x_pool, const int* __restrict__ slots,
                                                        int nvec, u64* __restrict__ e, u64* __restrict__ a, int n_slots,
                                                        int pieces) {
    typedef typename Word<VEC>::type V;
    const int t = (int)(blockIdx.x / (unsigned)pieces), piece = (int)(blockIdx.x % (unsigned)pieces);
    const int slot = slots[t];
    if (slot < 0 || slot >= n_slots) return;
    const size_t to = (size_t)t * nvec, from = (size_t)slot * nvec;
    for (int c = piece * GT + threadIdx.x; c < nvec; c += pieces * GT) {
        const V f = reinterpret_cast<const V*>(f_pool)[from + c];
        const V x = reinterpret_cast<const V*>(x_pool)[from + c];
        reinterpret_cast<V*>(e)[to + c] = f;
        reinterpret_cast<V*>(a)[to + c] = party ? x - f : x;
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
    int units;             // per token: heads x (pairs + unrotated words)
};

__device__ __forceinline__ u64 rescale(int party, u64 v, int f) {
    return party == 0 ? (u64)((long long)v >> f) : (u64)0 - (u64)((long long)((u64)0 - v) >> f);
}

// One thread per pair, or per word that is not rotated.
__global__ __launch_bounds__(GT) void rotate_kernel(RotateParams p, int pieces) {
    const int t = (int)(blockIdx.x / (unsigned)pieces), piece = (int)(blockIdx.x % (unsigned)pieces);
    const int per_head = p.head_dim - p.half;
    const u64* x = p.x + (size_t)t * p.ldx;
    const size_t row = (size_t)t * p.n_heads * p.head_dim;
    long at = p.half ? p.pos[t] : 0;
    if (at < 0 || at >= p.n_pos) at = 0;
    for (int i = piece * GT + threadIdx.x; i < p.units; i += pieces * GT) {
        const int h = i / per_head, j = i - h * per_head;
        const int base = h * p.head_dim;
        if (j < p.half) {
            const int a = base + (p.interleaved ? 2 * j : j), b = base + (p.interleaved ? 2 * j + 1 : j + p.half);
            const u64 c = p.cos_t[(size_t)at * p.half + j], s = p.sin_t[(size_t)at * p.half + j];
            const u64 xa = rescale(p.party, x[a], p.shift), xb = rescale(p.party, x[b], p.shift);
            u64 ya = rescale(p.party, xa * c - xb * s, p.frac), yb = rescale(p.party, xb * c + xa * s, p.frac);
            if (p.m) { ya -= p.m[row + a]; yb -= p.m[row + b]; }
            p.out[row + a] = ya;
            p.out[row + b] = yb;
        } else {
            const int a = base + j + p.half;
            u64 y = rescale(p.party, x[a], p.shift);
            if (p.m) y -= p.m[row + a];
            p.out[row + a] = y;
        }
    }
}

// workgroups that share a row of n units
inline int row_pieces(int64_t n, int per_thread) {
    int64_t g = (n + (int64_t)GT * per_thread - 1) / ((int64_t)GT * per_thread);
    return (int)(g < 1 ? 1 : g > 64 ? 64 : g);
}

int check_rows(comet_ctx* ctx, const char* what, int party, const void* const (&ptrs)[5], const int32_t* slots, int64_t n_tok,
               int64_t width, int64_t n_slots) {
    if (party != 0 && party != 1) return comet_fail(ctx, COMET_EINVAL, "%s: party must be 0 or 1", what);
    if (n_tok < 0 || width < 0 || n_slots < 0) return comet_fail(ctx, COMET_EINVAL, "%s: bad size", what);
    if (n_tok > COMET_DIM_MAX || width > COMET_DIM_MAX || n_slots > 0x7fffffffll)
        return comet_fail(ctx, COMET_ECAP, "%s: n_tok and width must stay below 2^24, n_slots below 2^31", what);
    if (n_tok == 0 || width == 0) return COMET_OK;
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
    if (rc != COMET_OK || n_tok == 0 || width == 0) return rc;
    comet_device_guard guard(ctx);
    if (!guard.ok) return comet_fail(ctx, COMET_EDEVICE, "%s: cannot select device", what);
    const bool vec = (width & 1) == 0;
    const int nvec = (int)(vec ? width / 2 : width), pieces = row_pieces(nvec, 2);
    const dim3 grid((unsigned)(n_tok * pieces));              // n_tok < 2^24, pieces <= 64
    auto kern = vec ? cache_write_kernel<2> : cache_write_kernel<1>;
    hipLaunchKernelGGL(kern, grid, dim3(GT), 0, ctx->stream, party, (const u64*)d_0, (const u64*)d_1, (const u64*)b_i, slots,
                       nvec, (u64*)f_pool, (u64*)x_pool, (int)n_slots, pieces);
    COMET_LAUNCH_CHECK(ctx, what);
    return COMET_OK;
}

int comet_cache_read(comet_ctx* ctx, int party, const uint64_t* f_pool, const uint64_t* x_pool, const int32_t* slots,
                     int64_t n_tok, int64_t width, int64_t n_slots, uint64_t* e, uint64_t* a_i) {
    const char* what = "comet_cache_read";
    COMET_CHECK_CTX(ctx);
    const int rc = check_rows(ctx, what, party, {f_pool, x_pool, e, a_i, e}, slots, n_tok, width, n_slots);
    if (rc != COMET_OK || n_tok == 0 || width == 0) return rc;
    comet_device_guard guard(ctx);
    if (!guard.ok) return comet_fail(ctx, COMET_EDEVICE, "%s: cannot select device", what);
    const bool vec = (width & 1) == 0;
    const int nvec = (int)(vec ? width / 2 : width), pieces = row_pieces(nvec, 2);
    const dim3 grid((unsigned)(n_tok * pieces));
    auto kern = vec ? cache_read_kernel<2> : cache_read_kernel<1>;
    hipLaunchKernelGGL(kern, grid, dim3(GT), 0, ctx->stream, party, (const u64*)f_pool, (const u64*)x_pool, slots, nvec,
                       (u64*)e, (u64*)a_i, (int)n_slots, pieces);
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
    p.units = n_heads * (head_dim - p.half);
    const int pieces = row_pieces(p.units, 2);
    hipLaunchKernelGGL(rotate_kernel, dim3((unsigned)(n_tok * pieces)), dim3(GT), 0, ctx->stream, p, pieces);
    COMET_LAUNCH_CHECK(ctx, what);
    return COMET_OK;
}

}  // extern "C"
