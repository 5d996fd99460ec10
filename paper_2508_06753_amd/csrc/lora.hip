// Low-rank adapters of many requests beside a shared projection:
//   T[m,j] = sum_k X[m,k] A[a_m, j, k],  Y[m,n] = act(base[m,n] + scale * sum_r T[m, part(n) R + r] B[a_m, n, r]).
#include <hip/hip_runtime.h>

#include "block_ops.h"

namespace w2 {

size_t lora_workspace_bytes(int n_parts, int R, int64_t M, int64_t, int64_t)
{
    return ((size_t)M * n_parts * R * sizeof(float) + 255) & ~(size_t)255;
}

__device__ __forceinline__ int lora_part(const LoraArgs& a, int block)
{
    if (a.gated) return block & 1;
    return (block >= a.end16[0]) + (block >= a.end16[1]) + (block >= a.end16[2]);
}

__device__ __forceinline__ int lora_rank(const LoraArgs& a, int ad)
{
    return a.rank ? min(max(a.rank[ad], 0), a.R) : a.R;
}

__global__ void __launch_bounds__(256) lora_shrink_kernel(LoraArgs a)
{
    const int lane = threadIdx.x & 63;
    const int PR = a.n_parts * a.R;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit >= a.M * PR) return;
    const int64_t m = unit / PR;
    const int j = (int)(unit % PR), ad = a.adapter[m];
    if (ad < 0 || ad >= a.n_adapters) return;
    float s = 0.0f;
    if (j % a.R < lora_rank(a, ad)) {
        const uint16_t* A = a.A + ad * a.a_stride + (int64_t)j * a.K;
        for (int64_t k = lane; k < a.K; k += 64) {
            const float x = a.x_f32 ? ((const float*)a.X)[m * a.ldx + k] : bf16_f32(((const uint16_t*)a.X)[m * a.ldx + k]);
            s = fmaf(x, bf16_f32(A[k]), s);
        }
#pragma unroll
        for (int off = 32; off; off >>= 1) s += __shfl_xor(s, off);
    }
    if (lane == 0) a.T[unit] = s;
}

__device__ float lora_z(const LoraArgs& a, int64_t m, int ad, int rank, float scale, int64_t n)
{
    const float base = a.base ? bf16_f32(a.base[m * a.ldb + n]) : 0.0f;
    if (ad < 0) return base;
    const float* T = a.T + (m * a.n_parts + lora_part(a, (int)(n / 16))) * a.R;
    const uint16_t* B = a.B + ad * a.b_stride + n * a.R;
    float s = 0.0f;
    for (int r = 0; r < rank; ++r) s = fmaf(T[r], bf16_f32(B[r]), s);
    return fmaf(scale, s, base);
}

__device__ __forceinline__ float silu(float z) { return z / (1.0f + __expf(-z)); }

__global__ void __launch_bounds__(256) lora_expand_kernel(LoraArgs a)
{
    const int64_t m = blockIdx.y, n_out = a.act == ACT_SILU_MUL ? a.N / 2 : a.N;
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= n_out) return;
    int ad = a.adapter[m];
    if (ad >= a.n_adapters) ad = -1;
    const int rank = ad < 0 ? 0 : lora_rank(a, ad);
    const float scale = ad < 0 || !a.scale ? 1.0f : a.scale[ad];
    float y;
    if (a.act == ACT_SILU_MUL) {
        const int64_t n = c / 16 * 32 + c % 16;
        y = silu(lora_z(a, m, ad, rank, scale, n)) * lora_z(a, m, ad, rank, scale, n + 16);
    } else {
        y = lora_z(a, m, ad, rank, scale, c);
        if (a.act == ACT_SILU) y = silu(y);
    }
    a.Y[m * a.ldy + c] = f32_bf16(y);
}

int launch_lora(const LoraArgs& a, hipStream_t stream)
{
    const int64_t units = a.M * a.n_parts * a.R, n_out = a.act == ACT_SILU_MUL ? a.N / 2 : a.N;
    hipLaunchKernelGGL(lora_shrink_kernel, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, stream, a);
    const int rc = check_launch("w2_lora_add");
    if (rc) return rc;
    for (int64_t m = 0; m < a.M; m += 65535) {                 // a grid's second dimension ends at 65535
        LoraArgs b = a;
        const int64_t rows = a.M - m < 65535 ? a.M - m : 65535;
        b.adapter += m;
        b.base = a.base ? a.base + m * a.ldb : nullptr;
        b.Y += m * a.ldy;
        b.T += m * a.n_parts * a.R;
        hipLaunchKernelGGL(lora_expand_kernel, dim3((unsigned)((n_out + 255) / 256), (unsigned)rows), dim3(256), 0, stream, b);
    }
    return check_launch("w2_lora_add");
}

}  // namespace w2
