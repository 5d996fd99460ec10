// C-ABI entry points of the operators between the projections: argument validation, and the frequencies of the
// rotation, which are made on the host.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/w2mm.h"
#include "block_ops.h"

using namespace w2;

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

int check_lora(const char* fn, const w2_lora_t* l, int64_t M, int64_t K, int64_t N)
{
    if (!l) return fail(W2_ERR_INVALID_ARG, "%s: lora is NULL", fn);
    if (M < 0 || K <= 0 || N <= 0) return fail(W2_ERR_INVALID_ARG, "%s: M must not be negative, K and N must be positive", fn);
    if (K % 256) return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: K must be a multiple of 256", fn);
    if (N % 8) return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: N must be a multiple of 8", fn);
    if (K > (int64_t)1 << 24 || N > (int64_t)1 << 24 || M > (int64_t)1 << 24)
        return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: M, K and N are limited to 2^24", fn);
    if (l->n_adapters <= 0) return fail(W2_ERR_INVALID_ARG, "%s: n_adapters must be positive", fn);
    if (l->max_rank <= 0 || l->max_rank % 8 || l->max_rank > 128)
        return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: max_rank must be a multiple of 8 up to 128", fn);
    if (l->gated) {
        if (N % 32) return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: gated parts alternate by 16 columns: N must be a multiple of 32", fn);
        return W2_OK;
    }
    if (l->n_parts < 1 || l->n_parts > 4) return fail(W2_ERR_INVALID_ARG, "%s: n_parts must be 1..4", fn);
    int64_t before = 0;
    for (int p = 0; p < l->n_parts; ++p) {
        if (l->part_end[p] <= before) return fail(W2_ERR_INVALID_ARG, "%s: the ends of the parts must increase", fn);
        if (p + 1 < l->n_parts && l->part_end[p] % 16)
            return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: the ends of the parts must be multiples of 16", fn);
        before = l->part_end[p];
    }
    if (before != N) return fail(W2_ERR_INVALID_ARG, "%s: the last part must end at N", fn);
    return W2_OK;
}

int check_cache(const char* fn, const w2_kv_cache_t* c)
{
    if (!c) return fail(W2_ERR_INVALID_ARG, "%s: cache is NULL", fn);
    if (c->n_pages <= 0 || c->page_size <= 0 || c->n_heads <= 0)
        return fail(W2_ERR_INVALID_ARG, "%s: the cache's n_pages, page_size and n_heads must be positive", fn);
    if (c->head_dim <= 0 || c->head_dim % 8 || c->head_dim > 256)
        return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: head_dim must be a multiple of 8 up to 256", fn);
    if (c->n_pages > 0x7fffffff || c->page_size > 0x7fffffff || c->n_pages * c->page_size > 0x7fffffff)
        return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: the cache is limited to 2^31 - 1 places", fn);
    if (c->n_heads > 1024) return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: n_heads is limited to 1024", fn);
    if (!c->k || !c->v) return fail(W2_ERR_INVALID_ARG, "%s: NULL pointer in the cache", fn);
    if (!aligned16(c->k) || !aligned16(c->v)) return fail(W2_ERR_MISALIGNED, "%s: the cache's k and v must be 16-byte aligned", fn);
    const int64_t st[6] = {c->k_page_stride, c->k_slot_stride, c->k_head_stride, c->v_page_stride, c->v_slot_stride, c->v_head_stride};
    for (int i = 0; i < 6; ++i)
        if (st[i] < 0 || st[i] % 8) return fail(W2_ERR_MISALIGNED, "%s: the cache's strides must be multiples of 8, not negative", fn);
    for (int i = 0; i < 6; ++i)
        if (st[i] > 0x7fffffff) return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: the cache's strides are limited to 2^31 - 1 elements", fn);
    return W2_OK;
}

int check_tree_sizes(const char* fn, int64_t n_requests, int64_t M, int n_q, int n_kv, int D, int64_t max_rows, int64_t max_len,
                     int64_t total_len)
{
    if (n_requests < 0 || M < 0 || max_rows < 0 || max_len < 0 || total_len < 0)
        return fail(W2_ERR_INVALID_ARG, "%s: negative size", fn);
    if (n_q <= 0 || n_kv <= 0) return fail(W2_ERR_INVALID_ARG, "%s: numbers of heads must be positive", fn);
    if (n_q % n_kv) return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: n_q must be a multiple of the cache's n_heads", fn);
    if (n_q > 1024) return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: n_q is limited to 1024", fn);
    if (D <= 0 || D % 8 || D > 256) return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: head_dim must be a multiple of 8 up to 256", fn);
    if (n_requests > 65535 || M > (int64_t)1 << 24 || max_len > 0x7fffffff)
        return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: limited to 65535 requests, 2^24 rows and 2^31 - 1 keys a request", fn);
    return W2_OK;
}

}  // namespace

extern "C" {

int w2_lora_workspace_size(const w2_lora_t* lora, int64_t M, int64_t K, int64_t N, size_t* bytes)
{
    if (!bytes) return fail(W2_ERR_INVALID_ARG, "w2_lora_workspace_size: bytes is NULL");
    const int rc = check_lora("w2_lora_workspace_size", lora, M, K, N);
    if (rc) return rc;
    *bytes = lora_workspace_bytes(lora->gated ? 2 : lora->n_parts, lora->max_rank, lora->n_adapters, M, K, N);
    return W2_OK;
}

int w2_lora_add(const w2_lora_t* lora, int64_t K, int64_t N, const void* X, w2_dtype_t x_dtype, int64_t ldx, int64_t M,
                const int32_t* adapter, const uint16_t* base, int64_t ldb, uint16_t* Y, int64_t ldy, int act,
                void* workspace, size_t workspace_bytes, void* stream)
{
    const char* fn = "w2_lora_add";
    const int rc = check_lora(fn, lora, M, K, N);
    if (rc) return rc;
    if (x_dtype != W2_DT_F32 && x_dtype != W2_DT_BF16) return fail(W2_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, (int)x_dtype);
    if (act < ACT_NONE || act > ACT_SILU_MUL) return fail(W2_ERR_INVALID_ARG, "%s: unknown activation %d", fn, act);
    if (act == ACT_SILU_MUL && N % 32)
        return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: the gated activation pairs 16-column blocks: N must be a multiple of 32", fn);
    if (M == 0) return W2_OK;
    if (!X || !adapter || !Y || !lora->A || !lora->B) return fail(W2_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    if (!aligned16(X) || !aligned16(Y) || !aligned16(base) || !aligned16(lora->A) || !aligned16(lora->B) || !aligned16(workspace))
        return fail(W2_ERR_MISALIGNED, "%s: X, A, B, base, Y and workspace must be 16-byte aligned", fn);
    if (((uintptr_t)adapter & 3) || ((uintptr_t)lora->rank & 3) || ((uintptr_t)lora->scale & 3))
        return fail(W2_ERR_MISALIGNED, "%s: adapter, rank or scale is not aligned to its type", fn);
    const int64_t n_out = act == ACT_SILU_MUL ? N / 2 : N;
    if (ldx < K || ldx % 8) return fail(W2_ERR_MISALIGNED, "%s: ldx must be >= K and a multiple of 8", fn);
    if (base && (ldb < N || ldb % 8)) return fail(W2_ERR_MISALIGNED, "%s: ldb must be >= N and a multiple of 8", fn);
    if (ldy < n_out || ldy % 8) return fail(W2_ERR_MISALIGNED, "%s: ldy must be >= the number of output columns and a multiple of 8", fn);
    if (lora->a_stride < 0 || lora->a_stride % 8 || lora->b_stride < 0 || lora->b_stride % 8)
        return fail(W2_ERR_MISALIGNED, "%s: a_stride and b_stride must be multiples of 8, not negative", fn);
    if (act == ACT_SILU_MUL && base == Y) return fail(W2_ERR_INVALID_ARG, "%s: Y may not be base with the gated activation", fn);
    if (base == Y && ldb != ldy) return fail(W2_ERR_INVALID_ARG, "%s: Y may be base only with the same row stride", fn);
    if ((base && ldb >= (int64_t)1 << 25) || ldy >= (int64_t)1 << 25)
        return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: ldb and ldy are limited to 2^25 - 8", fn);
    LoraArgs a = {};
    a.A = lora->A; a.B = lora->B; a.rank = lora->rank; a.scale = lora->scale;
    a.a_stride = lora->a_stride; a.b_stride = lora->b_stride;
    a.n_adapters = lora->n_adapters; a.R = lora->max_rank; a.gated = lora->gated != 0;
    a.n_parts = a.gated ? 2 : lora->n_parts;
    for (int p = 0; p < 4; ++p) a.end16[p] = a.gated || p >= a.n_parts ? 0x7fffffff : (int)((lora->part_end[p] + 15) / 16);
    a.X = X; a.x_f32 = x_dtype == W2_DT_F32; a.adapter = adapter; a.base = base; a.Y = Y;
    a.K = K; a.N = N; a.M = M; a.ldx = ldx; a.ldb = ldb; a.ldy = ldy; a.act = act;
    const size_t need = lora_part_bytes(a.n_parts, a.R, M);
    if (!workspace || workspace_bytes < need)
        return fail(W2_ERR_BUFFER_TOO_SMALL, "%s: workspace_bytes %zu < %zu", fn, workspace ? workspace_bytes : (size_t)0, need);
    a.T = (float*)workspace;
    return launch_lora(a, workspace_bytes, (hipStream_t)stream);
}

int w2_rope_phases(double base, int rotary_dim, w2_rope_scaling_t scaling, double factor, double original_len, double low,
                   double high, uint64_t* phase)
{
    const char* fn = "w2_rope_phases";
    if (!phase) return fail(W2_ERR_INVALID_ARG, "%s: phase is NULL", fn);
    if (rotary_dim <= 0 || rotary_dim % 4 || rotary_dim > 256)
        return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: rotary_dim must be a multiple of 4 up to 256", fn);
    if (!(base >= 1.0) || !isfinite(base)) return fail(W2_ERR_INVALID_ARG, "%s: base must be finite and at least 1", fn);
    if (scaling < W2_ROPE_NONE || scaling > W2_ROPE_BANDS) return fail(W2_ERR_INVALID_ARG, "%s: unknown scaling %d", fn, (int)scaling);
    if (scaling != W2_ROPE_NONE && (!(factor >= 1.0) || !isfinite(factor)))
        return fail(W2_ERR_INVALID_ARG, "%s: factor must be finite and at least 1", fn);
    if (scaling == W2_ROPE_BANDS && (!(original_len > 0) || !isfinite(original_len) || !(low >= 0) || !(high > low) || !isfinite(high)))
        return fail(W2_ERR_INVALID_ARG, "%s: bands need original_len > 0 and 0 <= low < high", fn);
    if (scaling == W2_ROPE_NTK) base *= pow(factor, (double)rotary_dim / (rotary_dim - 2));
    for (int i = 0; i < rotary_dim / 2; ++i) {
        double turns = pow(base, -2.0 * i / rotary_dim) / (2.0 * M_PI);          // at most 1/2 pi
        if (scaling == W2_ROPE_LINEAR) turns /= factor;
        if (scaling == W2_ROPE_BANDS) {
            const double u = original_len * turns;
            const double keep = fmin(1.0, fmax(0.0, (u - low) / (high - low)));
            turns = turns / factor * (1.0 - keep) + turns * keep;
        }
        phase[i] = (uint64_t)ldexp(turns, 64);
    }
    return W2_OK;
}

int w2_qk_norm_rope(const uint16_t* x, int64_t ldx, int64_t M, int n_q, const uint16_t* q_weight, const uint16_t* k_weight,
                    float eps, const w2_rope_t* rope, const int32_t* positions, uint16_t* q, int64_t ldq,
                    const w2_kv_cache_t* cache, const int64_t* slots, void* stream)
{
    const char* fn = "w2_qk_norm_rope";
    const int rc = check_cache(fn, cache);
    if (rc) return rc;
    if (M < 0 || n_q <= 0) return fail(W2_ERR_INVALID_ARG, "%s: M must not be negative, n_q must be positive", fn);
    if (M > (int64_t)1 << 24 || n_q > 1024) return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: limited to 2^24 rows and 1024 heads", fn);
    if ((q_weight || k_weight) && !(eps >= 0.0f)) return fail(W2_ERR_INVALID_ARG, "%s: eps must not be negative", fn);
    const int D = cache->head_dim;
    if (rope) {
        if (rope->rotary_dim <= 0 || rope->rotary_dim % 4 || rope->rotary_dim > D)
            return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: rotary_dim must be a multiple of 4 up to head_dim", fn);
        if (M > 0 && (!rope->phase || !positions)) return fail(W2_ERR_INVALID_ARG, "%s: NULL pointer", fn);
        if ((uintptr_t)rope->phase & 7) return fail(W2_ERR_MISALIGNED, "%s: phase must be 8-byte aligned", fn);
    }
    if (!slots && M > cache->n_pages * cache->page_size) return fail(W2_ERR_BUFFER_TOO_SMALL, "%s: more rows than places in the cache", fn);
    if (M == 0) return W2_OK;
    if (!x || !q) return fail(W2_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    if (!aligned16(x) || !aligned16(q) || !aligned16(q_weight) || !aligned16(k_weight))
        return fail(W2_ERR_MISALIGNED, "%s: x, q and the weights must be 16-byte aligned", fn);
    if (((uintptr_t)positions & 3) || ((uintptr_t)slots & 7))
        return fail(W2_ERR_MISALIGNED, "%s: positions or slots is not aligned to its type", fn);
    if (ldx < (int64_t)(n_q + 2 * cache->n_heads) * D || ldx % 8)
        return fail(W2_ERR_MISALIGNED, "%s: ldx must be >= the heads' columns and a multiple of 8", fn);
    if (ldq < (int64_t)n_q * D || ldq % 8) return fail(W2_ERR_MISALIGNED, "%s: ldq must be >= n_q * head_dim and a multiple of 8", fn);
    if (q == x && ldq != ldx) return fail(W2_ERR_INVALID_ARG, "%s: q may be x only with the same row stride", fn);
    RopeArgs a = {};
    a.x = x; a.ldx = ldx; a.M = M; a.n_q = n_q; a.n_kv = cache->n_heads; a.D = D;
    a.qw = q_weight; a.kw = k_weight; a.eps = eps;
    a.phase = rope ? rope->phase : nullptr;
    a.rd = rope ? rope->rotary_dim : 0;
    a.interleaved = rope && rope->interleaved;
    a.mscale = rope ? rope->mscale : 1.0f;
    a.positions = positions; a.q = q; a.ldq = ldq; a.cache = *cache;
    a.page = make_divider((uint32_t)cache->page_size);
    a.slots = slots;
    return launch_qk_norm_rope(a, (hipStream_t)stream);
}

int w2_tree_attention_workspace_size(int64_t n_requests, int64_t M, int n_q, int n_heads, int head_dim, int64_t max_rows,
                                     int64_t max_len, int64_t total_len, size_t* bytes)
{
    const char* fn = "w2_tree_attention_workspace_size";
    if (!bytes) return fail(W2_ERR_INVALID_ARG, "%s: bytes is NULL", fn);
    const int rc = check_tree_sizes(fn, n_requests, M, n_q, n_heads, head_dim, max_rows, max_len, total_len);
    if (rc) return rc;
    *bytes = tree_workspace_bytes(n_requests, M, n_q, n_heads, head_dim, max_rows, max_len, total_len);
    return W2_OK;
}

int w2_tree_attention(const uint16_t* q, int64_t ldq, int64_t M, int n_q, const w2_kv_cache_t* cache, const int32_t* page_table,
                      int64_t table_cols, int64_t ld_table, const int32_t* row_start, const int32_t* kv_len, int64_t n_requests,
                      int64_t max_rows, int64_t max_len, int64_t total_len, const uint64_t* mask, int mask_words, float scale,
                      uint16_t* out, int64_t ldo, float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    const char* fn = "w2_tree_attention";
    int rc = check_cache(fn, cache);
    if (rc) return rc;
    const int D = cache->head_dim;
    rc = check_tree_sizes(fn, n_requests, M, n_q, cache->n_heads, D, max_rows, max_len, total_len);
    if (rc) return rc;
    if (mask && (mask_words <= 0 || mask_words > 65536)) return fail(W2_ERR_INVALID_ARG, "%s: mask_words must be 1..65536", fn);
    if (!isfinite(scale)) return fail(W2_ERR_INVALID_ARG, "%s: scale must be finite", fn);
    if (M == 0 || n_requests == 0 || max_rows == 0) return W2_OK;
    if (!q || !out || !row_start || !kv_len) return fail(W2_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    if (table_cols < 0 || ld_table < table_cols) return fail(W2_ERR_INVALID_ARG, "%s: ld_table must be >= table_cols >= 0", fn);
    if (table_cols > 0 && !page_table) return fail(W2_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    if (!aligned16(q) || !aligned16(out) || !aligned16(workspace))
        return fail(W2_ERR_MISALIGNED, "%s: q, out and workspace must be 16-byte aligned", fn);
    if (((uintptr_t)mask & 7) || ((uintptr_t)lse & 3) || ((uintptr_t)page_table & 3) || ((uintptr_t)row_start & 3) || ((uintptr_t)kv_len & 3))
        return fail(W2_ERR_MISALIGNED, "%s: mask, lse or an index array is not aligned to its type", fn);
    if (ldq < (int64_t)n_q * D || ldq % 8 || ldo < (int64_t)n_q * D || ldo % 8)
        return fail(W2_ERR_MISALIGNED, "%s: ldq and ldo must be >= n_q * head_dim and multiples of 8", fn);
    TreeArgs a = {};
    a.q = q; a.ldq = ldq; a.M = M; a.n_q = n_q; a.G = n_q / cache->n_heads; a.D = D;
    a.cache = *cache;
    a.page = make_divider((uint32_t)cache->page_size);
    a.table = page_table; a.table_cols = table_cols; a.ld_table = ld_table;
    a.row_start = row_start; a.kv_len = kv_len; a.n_requests = n_requests;
    a.max_rows = max_rows < M ? max_rows : M;
    a.max_len = max_len; a.total_len = total_len;
    a.mask = mask; a.mask_words = mask_words; a.scale = scale;
    a.out = out; a.ldo = ldo; a.lse = lse;
    a.workspace = workspace; a.workspace_bytes = workspace ? workspace_bytes : 0;
    return launch_tree_attention(a, (hipStream_t)stream);
}

}  // extern "C"
