// Attention of each request's drafted tokens over its pages of the cache.
#include <hip/hip_runtime.h>
#include <math.h>

#include "block_ops.h"

namespace w2 {

size_t tree_workspace_bytes(int64_t, int64_t, int, int, int, int64_t, int64_t, int64_t) { return 0; }

__device__ __forceinline__ bool tree_sees(const TreeArgs& a, int64_t row, int64_t i, int64_t j)
{
    if (j < 0) return true;
    if (!a.mask) return j <= i;
    return j < 64 * (int64_t)a.mask_words && (a.mask[row * a.mask_words + (j >> 6)] >> (j & 63) & 1);
}

// One wave per (row of a request, query head).
__global__ void __launch_bounds__(64) tree_attention_kernel(TreeArgs a)
{
    const int lane = threadIdx.x, h = blockIdx.x;
    const int64_t r = blockIdx.y, i = blockIdx.z;
    const int64_t first = a.row_start[r], last = min((int64_t)a.row_start[r + 1], a.M);
    const int64_t row = first + i;
    if (first < 0 || row >= last) return;
    const int64_t len = min(min((int64_t)a.kv_len[r], a.max_len), a.table_cols * a.cache.page_size);
    const int64_t context = len - (last - first);
    const int hk = h / a.G;
    float q[4] = {}, o[4] = {}, top = -INFINITY, sum = 0.0f;
    for (int t = 0; t < 4; ++t)
        if (lane + 64 * t < a.D) q[t] = bf16_f32(a.q[row * a.ldq + (int64_t)h * a.D + lane + 64 * t]);
    for (int64_t c = 0; c < len; ++c) {
        if (!tree_sees(a, row, i, c - context)) continue;
        const uint32_t at = divide((uint32_t)c, a.page);
        const int32_t page = a.table[r * a.ld_table + at];
        if (page < 0 || page >= a.cache.n_pages) continue;
        const int64_t place = c - (int64_t)at * a.cache.page_size;
        const uint16_t* k = a.cache.k + page * a.cache.k_page_stride + place * a.cache.k_slot_stride + hk * a.cache.k_head_stride;
        const uint16_t* v = a.cache.v + page * a.cache.v_page_stride + place * a.cache.v_slot_stride + hk * a.cache.v_head_stride;
        float s = 0.0f;
        for (int t = 0; t < 4; ++t)
            if (lane + 64 * t < a.D) s = fmaf(q[t], bf16_f32(k[lane + 64 * t]), s);
        for (int off = 32; off; off >>= 1) s += __shfl_xor(s, off);
        s *= a.scale;
        const float up = fmaxf(top, s);
        const float keep = top == -INFINITY ? 0.0f : expf(top - up), p = expf(s - up);
        sum = sum * keep + p;
        for (int t = 0; t < 4; ++t)
            if (lane + 64 * t < a.D) o[t] = o[t] * keep + p * bf16_f32(v[lane + 64 * t]);
        top = up;
    }
    for (int t = 0; t < 4; ++t)
        if (lane + 64 * t < a.D) a.out[row * a.ldo + (int64_t)h * a.D + lane + 64 * t] = f32_bf16(sum > 0.0f ? o[t] / sum : 0.0f);
    if (a.lse && lane == 0) a.lse[row * a.n_q + h] = sum > 0.0f ? top + logf(sum) : -INFINITY;
}

int launch_tree_attention(const TreeArgs& a, hipStream_t stream)
{
    hipLaunchKernelGGL(tree_attention_kernel, dim3(a.n_q, (unsigned)a.n_requests, (unsigned)a.max_rows), dim3(64), 0, stream, a);
    return check_launch("w2_tree_attention");
}

}  // namespace w2
