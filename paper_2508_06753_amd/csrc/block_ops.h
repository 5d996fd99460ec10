// Arguments of the operators between the projections (lora.hip, qk_norm_rope.hip, tree_attention.hip), checked by
// block_api.hip before anything is launched.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "w2_internal.h"

namespace w2 {

// two floats to bf16, round to nearest even
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    typedef float v2f __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f){lo, hi}, v2bf));
}

// n / d for 0 <= n < 2^31 by a multiply and a shift.  With s = ceil(log2 d) and m = ceil(2^(31+s) / d), the error
// e = m d - 2^(31+s) is below d <= 2^s, so n e < 2^(31+s) and the quotient, n m / 2^(31+s), is exact.
struct Divider {
    uint32_t m;
    int s;
};
inline Divider make_divider(uint32_t d)
{
    int s = 0;
    while (((uint64_t)1 << s) < d) ++s;
    return {(uint32_t)((((uint64_t)1 << (31 + s)) + d - 1) / d), s};
}
__device__ __forceinline__ uint32_t divide(uint32_t n, const Divider& v) { return __umulhi(2 * n, v.m) >> v.s; }

struct LoraArgs {
    const uint16_t *A, *B;
    const int32_t* rank;
    const float* scale;
    int64_t a_stride, b_stride;
    int n_adapters, R, n_parts, gated;
    int end16[4];                       // the parts' ends in blocks of 16 columns
    const void* X;
    int x_f32;
    const int32_t* adapter;
    const uint16_t* base;
    uint16_t* Y;
    int64_t K, N, M, ldx, ldb, ldy;
    int act;
    float* T;                           // the workspace: [K ranges][M][parts * R]
};
size_t lora_workspace_bytes(int n_parts, int R, int n_adapters, int64_t M, int64_t K, int64_t N);
size_t lora_part_bytes(int n_parts, int R, int64_t M);      // of T for one part of K
int launch_lora(const LoraArgs& a, size_t room, hipStream_t stream);       // room: bytes at a.T, at least one part's

struct RopeArgs {
    const uint16_t* x;
    int64_t ldx, M;
    int n_q, n_kv, D;
    const uint16_t *qw, *kw;
    float eps;
    const uint64_t* phase;
    int rd, interleaved;
    float mscale;
    const int32_t* positions;
    uint16_t* q;
    int64_t ldq;
    w2_kv_cache_t cache;
    Divider page;
    const int64_t* slots;
};
int launch_qk_norm_rope(const RopeArgs& a, hipStream_t stream);

struct TreeArgs {
    const uint16_t* q;
    int64_t ldq, M;
    int n_q, G, D;                      // G query heads share a cache head
    w2_kv_cache_t cache;
    Divider page;
    const int32_t* table;
    int64_t table_cols, ld_table;
    const int32_t *row_start, *kv_len;
    int64_t n_requests, max_rows, max_len, total_len;
    const uint64_t* mask;
    int mask_words;
    float scale;
    uint16_t* out;
    int64_t ldo;
    float* lse;
    void* workspace;
    size_t workspace_bytes;
};
size_t tree_workspace_bytes(int64_t n_requests, int64_t M, int n_q, int n_kv, int D, int64_t max_rows, int64_t max_len,
                            int64_t total_len);
int launch_tree_attention(const TreeArgs& a, hipStream_t stream);

}  // namespace w2
