// Attention over a cache of shares: the entry points of the products (attention_scores.hip, attention_values.hip), and the
// squared weights between them.
#include "attention_tile.h"

using namespace comet_attn;

namespace {

struct WeightParams {
    Batch b;
    int party, frac;
    u64 bias;
    const u64* d0;
    const u64* d1;
    const u64* r;
    const u64* r2;
    const u64* m;
    u64* out;
    u64* sums;
};

// T threads per row, one pass: five words read and one written for each key, the sum kept in registers.  Bound by HBM, so
// what counts is bytes on their way: a thread requests 2 U words of all operands before it uses the first (out may be one of
// them, so the compiler could not look ahead by itself).  16 x 32 rows of up to 8193 keys: 27 us, 5.1 TB/s; 4 prompts of up to 512
// tokens of 32 heads: 91 us, 5.3 TB/s (through the caches 32 and 107).
template <int T>
__global__ __launch_bounds__(T < 256 ? 256 : T) void weights_kernel(WeightParams p, int n_rows) {
    constexpr int NT = T < 256 ? 256 : T, U = 2;
    const Batch& b = p.b;
    const unsigned at = block_number() * (unsigned)(NT / T) + __builtin_amdgcn_readfirstlane(threadIdx.x / T);
    const int lane = (int)threadIdx.x % T;
    const bool inside = at < (unsigned)n_rows;
    const unsigned w = inside ? at / (unsigned)b.n_heads : 0;
    const int h = inside ? (int)(at % (unsigned)b.n_heads) : 0;
    const Place place(b, w);
    const Sequence sq(b, place.s);
    const int j = place.of(b, sq, w);
    const bool live = inside && j >= 0;
    const int v = live ? sq.sees(b, j, h) : 0;
    const size_t row = (size_t)(sq.q0 + (live ? j : 0)) * b.n_heads + h, base = row * b.ld;
    u64 sum = 0;
    for (int key0 = 2 * lane; key0 < v; key0 += 2 * T * U) {
        u64x2 u[U], u1[U], r[U], r2[U], m[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            // (ld is even; beyond what the row sees its last pair again)
            const int key = key0 + 2 * T * i;
            const size_t at = base + (key < v ? key : (v - 1) & ~1);
            u[i] = __builtin_nontemporal_load(reinterpret_cast<const u64x2*>(p.d0 + at));
            u1[i] = p.d1 ? __builtin_nontemporal_load(reinterpret_cast<const u64x2*>(p.d1 + at)) : u64x2{0, 0};
            r[i] = __builtin_nontemporal_load(reinterpret_cast<const u64x2*>(p.r + at));
            r2[i] = __builtin_nontemporal_load(reinterpret_cast<const u64x2*>(p.r2 + at));
            m[i] = p.m ? __builtin_nontemporal_load(reinterpret_cast<const u64x2*>(p.m + at)) : u64x2{0, 0};
        }
        auto square = [&](u64 x, u64 rr, u64 sq2) {
            const u64 bias = x + p.bias;
            return rescale(p.party, sq2 + bias * (p.party ? 2 * rr + bias : 2 * rr), p.frac);
        };
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int key = key0 + 2 * T * i;
            const u64 x = square(u[i].x + u1[i].x, r[i].x, r2[i].x), y = square(u[i].y + u1[i].y, r[i].y, r2[i].y);
            u64* const to = p.out + base + key;
            if (key + 1 < v) {
                sum += x + y;
                __builtin_nontemporal_store(u64x2{x - m[i].x, y - m[i].y}, reinterpret_cast<u64x2*>(to));
            } else if (key < v) {
                sum += x;
                *to = x - m[i].x;
            }
        }
    }
#pragma unroll
    for (int n = 32; n > 0; n /= 2) sum += __shfl_xor(sum, n);
    if constexpr (T > 64) {
        __shared__ u64 part[NT / 64];
        if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = sum;
        __syncthreads();
        sum = 0;
        for (int i = 0; i < T / 64; ++i) sum += part[(threadIdx.x / T) * (T / 64) + i];
    }
    if (live && lane == 0) p.sums[row] = sum;
}

// Checks of a batch; fills the device view.  COMET_OK with n_tok == 0 or n_seq == 0 means: nothing to do.  paged: the call
// looks up pages.
int make_batch(comet_ctx* ctx, const char* what, const comet_kv_batch* in, int64_t n_pages, int64_t ld, bool paged, Batch* b) {
    if (!in) return comet_fail(ctx, COMET_EINVAL, "%s: null batch", what);
    if (in->n_seq < 0 || in->n_tok < 0 || in->n_heads < 1 || in->n_kv_heads < 1 || in->n_heads % in->n_kv_heads != 0 ||
        in->max_q < 0 || in->max_pages < 0 || in->page_size < 16 || in->page_size % 16 != 0 || (in->flags & ~COMET_CAUSAL) != 0)
        return comet_fail(ctx, COMET_EINVAL, "%s: bad batch (n_heads must be a multiple of n_kv_heads, page_size of 16)", what);
    if (ld < 2 || (ld & 1) || n_pages < 0) return comet_fail(ctx, COMET_EINVAL, "%s: ld must be even and at least 2", what);
    if (ld > COMET_DIM_MAX || n_pages > 0x7fffffffll || n_pages * in->page_size > 0x7fffffffll ||
        (int64_t)in->n_tok * in->n_heads > 0x7fffffffll || (int64_t)in->n_seq * in->max_q > COMET_DIM_MAX ||
        (int64_t)in->n_seq * in->n_kv_heads > COMET_DIM_MAX)
        return comet_fail(ctx, COMET_ECAP, "%s: ld, n_seq * max_q and n_seq * n_kv_heads must stay below 2^24, rows and slots below 2^31", what);
    if (in->n_seq > 0 && in->n_tok > 0 && (!in->q_start || !in->kv_len || (paged && in->max_pages > 0 && !in->block_table)))
        return comet_fail(ctx, COMET_EINVAL, "%s: null pointer in the batch", what);
    b->n_seq = in->n_seq; b->n_tok = in->n_tok; b->n_heads = in->n_heads; b->n_kv_heads = in->n_kv_heads;
    b->group = in->n_heads / in->n_kv_heads;
    b->page_size = in->page_size; b->max_pages = in->max_pages; b->n_pages = (int)n_pages;
    b->max_q = in->max_q < in->n_tok ? in->max_q : in->n_tok; b->causal = (in->flags & COMET_CAUSAL) != 0;
    b->by_sequence = Place::by_sequence(*b);
    b->ld = (int)ld;
    const int64_t cap = (int64_t)in->max_pages * in->page_size;
    b->kv_cap = (int)(cap < ld ? cap : ld);
    b->q_start = in->q_start; b->kv_len = in->kv_len; b->block_table = in->block_table; b->head_mask = in->head_mask;
    return COMET_OK;
}

int make_product(comet_ctx* ctx, const char* what, int party, const comet_kv_batch* batch, int d, int ldp, int64_t n_pages,
                 int64_t ld, int frac_bits, const uint64_t* E, const uint64_t* A_i, const uint64_t* f_pool,
                 const uint64_t* x_pool, const uint64_t* C_i, const uint64_t* M_i, uint64_t* Z_i, ProductParams* p) {
    if ((party != 0 && party != 1) || frac_bits < 0 || frac_bits > 62)
        return comet_fail(ctx, COMET_EINVAL, "%s: party must be 0 or 1, 0 <= frac_bits <= 62", what);
    const int rc = make_batch(ctx, what, batch, n_pages, ld, true, &p->b);
    if (rc != COMET_OK) return rc;
    if (d < 1 || (d & 1) || (ldp & 1) || ldp < d) return comet_fail(ctx, COMET_EINVAL, "%s: d and ldp must be even, 1 <= d <= ldp", what);
    if (d > MAX_D || (int64_t)p->b.n_kv_heads * ldp > COMET_DIM_MAX)
        return comet_fail(ctx, COMET_ECAP, "%s: d must be at most %d, a slot's words below 2^24", what, MAX_D);
    if (p->b.n_tok == 0 || p->b.n_seq == 0 || p->b.max_q == 0) return COMET_OK;
    if (n_pages < 1 && p->b.kv_cap > 0) return comet_fail(ctx, COMET_EINVAL, "%s: empty pools", what);
    // (no pool is read where a sequence has no pages)
    const void* ptrs[] = {E, A_i, C_i, Z_i, f_pool, x_pool};
    for (int i = 0; i < (p->b.kv_cap > 0 ? 6 : 4); ++i) {
        const void* const q = ptrs[i];
        if (!q) return comet_fail(ctx, COMET_EINVAL, "%s: null pointer", what);
        if (!comet_aligned16(q)) return comet_fail(ctx, COMET_EALIGN, "%s: operands must be 16-byte aligned", what);
    }
    if (M_i && !comet_aligned16(M_i)) return comet_fail(ctx, COMET_EALIGN, "%s: operands must be 16-byte aligned", what);
    if (Z_i == E || Z_i == A_i || Z_i == f_pool || Z_i == x_pool)
        return comet_fail(ctx, COMET_EINVAL, "%s: Z_i may be C_i or M_i, no other operand", what);
    p->party = party; p->d = d; p->ldp = ldp; p->frac = frac_bits;
    p->E = (const u64*)E; p->A = (const u64*)A_i; p->F = (const u64*)f_pool; p->X = (const u64*)x_pool;
    p->C = (const u64*)C_i; p->M = (const u64*)M_i; p->Z = (u64*)Z_i;
    p->part = nullptr;
    p->far_rows = false;
    p->tiles = p->groups = p->chunks = p->chunk = p->parts = 1;
    return COMET_OK;
}

}  // namespace

size_t comet_attention_workspace_bytes(int op, int64_t m, int64_t k, int64_t n) {
    return op == COMET_OP_VALUES ? values_workspace_bytes(m, k, n) : 0;
}

extern "C" {

int comet_attention_scores(comet_ctx* ctx, int party, const comet_kv_batch* batch, int d, int ldp, int64_t n_pages, int64_t ld,
                           int frac_bits, const uint64_t* E, const uint64_t* A_i, const uint64_t* f_pool, const uint64_t* x_pool,
                           const uint64_t* C_i, const uint64_t* M_i, uint64_t* Z_i, void* ws, size_t ws_bytes) {
    const char* what = "comet_attention_scores";
    COMET_CHECK_CTX(ctx);
    (void)ws; (void)ws_bytes;                                 // (none is needed)
    ProductParams p;
    const int rc = make_product(ctx, what, party, batch, d, ldp, n_pages, ld, frac_bits, E, A_i, f_pool, x_pool, C_i, M_i, Z_i, &p);
    if (rc != COMET_OK) return rc;
    const Batch& b = p.b;
    if (b.n_tok == 0 || b.n_seq == 0 || b.max_q == 0 || b.kv_cap == 0) return COMET_OK;
    comet_device_guard guard(ctx);
    if (!guard.ok) return comet_fail(ctx, COMET_EDEVICE, "%s: cannot select device", what);
    return launch_scores(ctx, what, p);
}

int comet_attention_values(comet_ctx* ctx, int party, const comet_kv_batch* batch, int d, int ldp, int64_t n_pages, int64_t ld,
                           int frac_bits, const uint64_t* E, const uint64_t* A_i, const uint64_t* f_pool, const uint64_t* x_pool,
                           const uint64_t* C_i, const uint64_t* M_i, uint64_t* Z_i, void* ws, size_t ws_bytes) {
    const char* what = "comet_attention_values";
    COMET_CHECK_CTX(ctx);
    ProductParams p;
    const int rc = make_product(ctx, what, party, batch, d, ldp, n_pages, ld, frac_bits, E, A_i, f_pool, x_pool, C_i, M_i, Z_i, &p);
    if (rc != COMET_OK) return rc;
    const Batch& b = p.b;
    if (b.n_tok == 0 || b.n_seq == 0 || b.max_q == 0) return COMET_OK;
    comet_device_guard guard(ctx);
    if (!guard.ok) return comet_fail(ctx, COMET_EDEVICE, "%s: cannot select device", what);
    return launch_values(ctx, what, p, ws, ws_bytes);
}

int comet_attention_weights(comet_ctx* ctx, int party, const comet_kv_batch* batch, int64_t ld, int frac_bits, uint64_t bias,
                            const uint64_t* d_0, const uint64_t* d_1, const uint64_t* r_i, const uint64_t* r2_i,
                            const uint64_t* m_i, uint64_t* out, uint64_t* sums) {
    const char* what = "comet_attention_weights";
    COMET_CHECK_CTX(ctx);
    if ((party != 0 && party != 1) || frac_bits < 0 || frac_bits > 62)
        return comet_fail(ctx, COMET_EINVAL, "%s: party must be 0 or 1, 0 <= frac_bits <= 62", what);
    WeightParams p;
    const int rc = make_batch(ctx, what, batch, 1, ld, false, &p.b);
    if (rc != COMET_OK) return rc;
    const Batch& b = p.b;
    if (b.n_tok == 0 || b.n_seq == 0 || b.max_q == 0) return COMET_OK;
    const void* ptrs[] = {d_0, r_i, r2_i, out, sums};
    for (const void* q : ptrs)
        if (!q) return comet_fail(ctx, COMET_EINVAL, "%s: null pointer", what);
    const void* all[] = {d_0, d_1, r_i, r2_i, m_i, out, sums};
    for (const void* q : all)
        if (q && !comet_aligned16(q)) return comet_fail(ctx, COMET_EALIGN, "%s: operands must be 16-byte aligned", what);
    if (out == sums) return comet_fail(ctx, COMET_EINVAL, "%s: out and sums must not be one buffer", what);
    comet_device_guard guard(ctx);
    if (!guard.ok) return comet_fail(ctx, COMET_EDEVICE, "%s: cannot select device", what);
    p.party = party; p.frac = frac_bits; p.bias = bias;
    p.d0 = (const u64*)d_0; p.d1 = (const u64*)d_1; p.r = (const u64*)r_i; p.r2 = (const u64*)r2_i; p.m = (const u64*)m_i;
    p.out = (u64*)out; p.sums = (u64*)sums;
    const int n_rows = (int)(Place::count(b) * b.n_heads);    // (< 2^31: by_sequence())
    // A wavefront per row where rows are short (prompts: many rows), a whole workgroup of sixteen where they are long and few.
    if (b.kv_cap <= 1024) return launch_all(ctx, what, weights_kernel<64>, ((int64_t)n_rows + 3) / 4, 256, p, n_rows);
    if (b.kv_cap <= 4096) return launch_all(ctx, what, weights_kernel<256>, n_rows, 256, p, n_rows);
    return launch_all(ctx, what, weights_kernel<1024>, n_rows, 1024, p, n_rows);
}

}  // extern "C"
