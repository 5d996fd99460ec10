// C-ABI entry points of the operators of a layer's feed-forward half: argument validation.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/w2mm.h"
#include "ffn_ops.h"

using namespace w2;

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

int check_router(const char* fn, const w2_router_t* r, int64_t M, int64_t K)
{
    if (!r) return fail(W2_ERR_INVALID_ARG, "%s: router is NULL", fn);
    if (M < 0 || K <= 0) return fail(W2_ERR_INVALID_ARG, "%s: M must not be negative, K must be positive", fn);
    if (K % 8 || K > 1 << 20 || M > 1 << 24)
        return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: K must be a multiple of 8 up to 2^20, M at most 2^24", fn);
    if (r->n_experts <= 0 || r->top_k <= 0) return fail(W2_ERR_INVALID_ARG, "%s: n_experts and top_k must be positive", fn);
    if (r->n_experts > 1024 || r->top_k > 64) return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: limited to 1024 experts and top_k 64", fn);
    if (r->score != W2_SCORE_SOFTMAX && r->score != W2_SCORE_SIGMOID)
        return fail(W2_ERR_INVALID_ARG, "%s: unknown score %d", fn, r->score);
    if (r->n_groups < 1 || r->n_groups > 64 || r->n_experts % r->n_groups)
        return fail(W2_ERR_INVALID_ARG, "%s: n_groups must be a divisor of n_experts up to 64", fn);
    if (r->top_groups < 1 || r->top_groups > r->n_groups)
        return fail(W2_ERR_INVALID_ARG, "%s: top_groups must be 1..n_groups", fn);
    if (r->group_top != 1 && r->group_top != 2) return fail(W2_ERR_INVALID_ARG, "%s: group_top must be 1 or 2", fn);
    if (r->top_k > r->n_experts / r->n_groups * r->top_groups)
        return fail(W2_ERR_INVALID_ARG, "%s: top_k is more than the experts of top_groups groups", fn);
    if (!isfinite(r->scale)) return fail(W2_ERR_INVALID_ARG, "%s: scale must be finite", fn);
    return W2_OK;
}

int check_experts(const char* fn, const w2_experts_t* e, int64_t M, int top_k)
{
    if (!e) return fail(W2_ERR_INVALID_ARG, "%s: experts is NULL", fn);
    if (M < 0 || top_k <= 0 || e->n_experts <= 0 || e->hidden <= 0 || e->inter <= 0)
        return fail(W2_ERR_INVALID_ARG, "%s: M must not be negative, top_k, n_experts, hidden and inter must be positive", fn);
    if (e->G != 64 && e->G != 128) return fail(W2_ERR_INVALID_ARG, "%s: G must be 64 or 128", fn);
    if (e->hidden % 256 || e->inter % 256) return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: hidden and inter must be multiples of 256", fn);
    if (e->hidden > 1 << 17 || e->inter > 1 << 17 || e->n_experts > 1024 || top_k > 64)
        return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: hidden and inter are limited to 2^17, n_experts to 1024, top_k to 64", fn);
    if (M > (1 << 24) / top_k) return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: M * top_k is limited to 2^24", fn);
    return W2_OK;
}

}  // namespace

extern "C" {

int w2_residual_norm(const w2_norm_t* norm, const void* residual, w2_dtype_t r_dtype, int64_t ldr, const uint16_t* y, int64_t ldy,
                     int64_t M, int64_t N, void* residual_out, int64_t ldro, uint16_t* x, int64_t ldx, int8_t* xq, float* sx,
                     void* stream)
{
    const char* fn = "w2_residual_norm";
    if (!norm) return fail(W2_ERR_INVALID_ARG, "%s: norm is NULL", fn);
    if (M < 0 || N <= 0) return fail(W2_ERR_INVALID_ARG, "%s: M must not be negative, N must be positive", fn);
    if (N % 8 || N > 65536 || M > 0x7fffffff)
        return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: N must be a multiple of 8 up to 65536, M below 2^31", fn);
    if (r_dtype != W2_DT_F32 && r_dtype != W2_DT_BF16) return fail(W2_ERR_INVALID_ARG, "%s: unknown dtype %d", fn, (int)r_dtype);
    if (!(norm->eps >= 0.0f) || !isfinite(norm->residual_scale) || !isfinite(norm->block_scale) || !isfinite(norm->weight_offset))
        return fail(W2_ERR_INVALID_ARG, "%s: eps must not be negative, scales and offset must be finite", fn);
    if ((xq == nullptr) != (sx == nullptr)) return fail(W2_ERR_INVALID_ARG, "%s: xq and sx come together", fn);
    if (xq && N % 16) return fail(W2_ERR_UNSUPPORTED_SHAPE, "%s: N must be a multiple of 16 for xq", fn);
    if (M == 0) return W2_OK;
    if (!residual && !y) return fail(W2_ERR_INVALID_ARG, "%s: neither residual nor y", fn);
    if (!residual_out && !x && !xq) return fail(W2_ERR_INVALID_ARG, "%s: nothing is wanted", fn);
    if (!aligned16(residual) || !aligned16(y) || !aligned16(residual_out) || !aligned16(x) || !aligned16(xq) ||
        !aligned16(norm->weight) || !aligned16(norm->post_weight) || !aligned16(norm->gate))
        return fail(W2_ERR_MISALIGNED, "%s: rows, weights and gate must be 16-byte aligned", fn);
    if ((uintptr_t)sx & 3) return fail(W2_ERR_MISALIGNED, "%s: sx is not aligned to its type", fn);
    if ((residual && (ldr < N || ldr % 8)) || (y && (ldy < N || ldy % 8)) || (residual_out && (ldro < N || ldro % 8)) ||
        (x && (ldx < N || ldx % 8)))
        return fail(W2_ERR_MISALIGNED, "%s: row strides must be >= N and multiples of 8", fn);
    if (norm->gate && norm->ld_gate && (norm->ld_gate < N || norm->ld_gate % 8))
        return fail(W2_ERR_MISALIGNED, "%s: ld_gate must be 0, or >= N and a multiple of 8", fn);
    if (residual && residual_out == residual && ldro != ldr)
        return fail(W2_ERR_INVALID_ARG, "%s: residual_out may be residual only with the same row stride", fn);
    if (y && x == y && ldx != ldy) return fail(W2_ERR_INVALID_ARG, "%s: x may be y only with the same row stride", fn);
    NormArgs a = {};
    a.p = *norm;
    a.residual = residual; a.r_bf16 = r_dtype == W2_DT_BF16; a.y = y;
    a.ldr = ldr; a.ldy = ldy; a.ldro = ldro; a.ldx = ldx; a.M = M; a.N = N;
    a.residual_out = residual_out; a.x = x; a.xq = xq; a.sx = sx;
    return launch_residual_norm(a, (hipStream_t)stream);
}

int w2_moe_route_workspace_size(const w2_router_t* router, int64_t M, int64_t K, size_t* bytes)
{
    if (!bytes) return fail(W2_ERR_INVALID_ARG, "w2_moe_route_workspace_size: bytes is NULL");
    const int rc = check_router("w2_moe_route_workspace_size", router, M, K);
    if (rc) return rc;
    *bytes = route_workspace_bytes(router->n_experts, M, K);
    return W2_OK;
}

int w2_moe_route(const w2_router_t* router, const uint16_t* x, int64_t ldx, int64_t M, int64_t K, int32_t* ids, float* weights,
                 float* logits, void* workspace, size_t workspace_bytes, void* stream)
{
    const char* fn = "w2_moe_route";
    const int rc = check_router(fn, router, M, K);
    if (rc) return rc;
    if (M == 0) return W2_OK;
    if (!x || !ids || !weights || !router->weight) return fail(W2_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    if (!aligned16(x) || !aligned16(router->weight) || !aligned16(workspace))
        return fail(W2_ERR_MISALIGNED, "%s: x, weight and workspace must be 16-byte aligned", fn);
    if (((uintptr_t)ids & 3) || ((uintptr_t)weights & 3) || ((uintptr_t)logits & 3) || ((uintptr_t)router->choice_bias & 3))
        return fail(W2_ERR_MISALIGNED, "%s: ids, weights, logits or choice_bias is not aligned to its type", fn);
    if (ldx < K || ldx % 8 || router->ldw < K || router->ldw % 8)
        return fail(W2_ERR_MISALIGNED, "%s: ldx and ldw must be >= K and multiples of 8", fn);
    const size_t need = route_workspace_bytes(router->n_experts, M, K);
    if (!workspace || workspace_bytes < need)
        return fail(W2_ERR_BUFFER_TOO_SMALL, "%s: workspace_bytes %zu < %zu", fn, workspace ? workspace_bytes : (size_t)0, need);
    RouteArgs a = {};
    a.r = *router; a.x = x; a.ldx = ldx; a.M = M; a.K = K;
    a.ids = ids; a.weights = weights; a.logits = logits; a.workspace = workspace;
    return launch_moe_route(a, (hipStream_t)stream);
}

int w2_moe_experts_workspace_size(const w2_experts_t* experts, int64_t M, int top_k, size_t* bytes)
{
    if (!bytes) return fail(W2_ERR_INVALID_ARG, "w2_moe_experts_workspace_size: bytes is NULL");
    const int rc = check_experts("w2_moe_experts_workspace_size", experts, M, top_k);
    if (rc) return rc;
    *bytes = experts_workspace_bytes(*experts, M, top_k);
    return W2_OK;
}

int w2_moe_experts(const w2_experts_t* experts, const uint16_t* x, int64_t ldx, int64_t M, const int32_t* ids, const float* weights,
                   int top_k, const uint16_t* base, int64_t ldb, uint16_t* Y, int64_t ldy, void* workspace, size_t workspace_bytes,
                   void* stream)
{
    const char* fn = "w2_moe_experts";
    const int rc = check_experts(fn, experts, M, top_k);
    if (rc) return rc;
    if (M == 0) return W2_OK;
    if (!x || !ids || !weights || !Y || !experts->gate_up || !experts->down) return fail(W2_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    if (!aligned16(x) || !aligned16(base) || !aligned16(Y) || !aligned16(experts->gate_up) || !aligned16(experts->down) ||
        !aligned16(workspace))
        return fail(W2_ERR_MISALIGNED, "%s: x, base, Y, the blobs and workspace must be 16-byte aligned", fn);
    if (((uintptr_t)ids & 3) || ((uintptr_t)weights & 3)) return fail(W2_ERR_MISALIGNED, "%s: ids or weights is not aligned to its type", fn);
    if (ldx < experts->hidden || ldx % 8 || ldy < experts->hidden || ldy % 8 || (base && (ldb < experts->hidden || ldb % 8)))
        return fail(W2_ERR_MISALIGNED, "%s: ldx, ldb and ldy must be >= hidden and multiples of 8", fn);
    if (Y == x) return fail(W2_ERR_INVALID_ARG, "%s: Y may not be x", fn);
    if (base == Y && ldb != ldy) return fail(W2_ERR_INVALID_ARG, "%s: Y may be base only with the same row stride", fn);
    ExpertsArgs a = {};
    a.e = *experts;
    a.up = make_layout(experts->hidden, 2 * experts->inter, experts->G);
    a.down = make_layout(experts->inter, experts->hidden, experts->G);
    if (experts->gate_up_stride % 16 || experts->down_stride % 16)
        return fail(W2_ERR_MISALIGNED, "%s: the strides of the blobs must be multiples of 16", fn);
    if (experts->n_experts > 1 &&
        (experts->gate_up_stride < (int64_t)a.up.total_bytes || experts->down_stride < (int64_t)a.down.total_bytes))
        return fail(W2_ERR_BUFFER_TOO_SMALL, "%s: the strides of the blobs are below the blobs' sizes", fn);
    a.x = x; a.ldx = ldx; a.M = M; a.ids = ids; a.weights = weights; a.top_k = top_k;
    a.base = base; a.ldb = ldb; a.Y = Y; a.ldy = ldy;
    const size_t need = experts_workspace_bytes(*experts, M, top_k);
    if (!workspace || workspace_bytes < need)
        return fail(W2_ERR_BUFFER_TOO_SMALL, "%s: workspace_bytes %zu < %zu", fn, workspace ? workspace_bytes : (size_t)0, need);
    a.workspace = workspace;
    return launch_moe_experts(a, (hipStream_t)stream);
}

}  // extern "C"
