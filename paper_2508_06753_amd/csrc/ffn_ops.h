// Arguments of the operators of a layer's feed-forward half (residual_norm.hip, moe_route.hip, moe_experts.hip), checked by
// ffn_api.hip before anything is launched.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "w2_internal.h"

namespace w2 {

struct NormArgs {
    w2_norm_t p;
    const void* residual;
    int r_bf16;
    const uint16_t* y;
    int64_t ldr, ldy, ldro, ldx, M, N;
    void* residual_out;
    uint16_t* x;
    int8_t* xq;
    float* sx;
};
int launch_residual_norm(const NormArgs& a, hipStream_t stream);

struct RouteArgs {
    w2_router_t r;
    const uint16_t* x;
    int64_t ldx, M, K;
    int32_t* ids;
    float *weights, *logits;
    void* workspace;
};
size_t route_workspace_bytes(int n_experts, int64_t M, int64_t K);
int launch_moe_route(const RouteArgs& a, hipStream_t stream);

struct ExpertsArgs {
    w2_experts_t e;
    Layout up, down;                    // of one expert's blobs
    const uint16_t* x;
    int64_t ldx, M, ldb, ldy;
    const int32_t* ids;
    const float* weights;
    int top_k;
    const uint16_t* base;
    uint16_t* Y;
    void* workspace;
};
size_t experts_workspace_bytes(const w2_experts_t& e, int64_t M, int top_k);
int launch_moe_experts(const ExpertsArgs& a, hipStream_t stream);

}  // namespace w2
