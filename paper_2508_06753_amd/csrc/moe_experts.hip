// Rows through their 2-bit experts: gate and up projection, silu(gate) * up, down projection, sum over a row's experts.
#include <hip/hip_runtime.h>

#include "block_ops.h"
#include "ffn_ops.h"

namespace w2 {

namespace {

__device__ __forceinline__ float scale_of(const char* blob, const Layout& L, int64_t cb, int64_t kt, int n, int g)
{
    const uint16_t* s = reinterpret_cast<const uint16_t*>(blob + L.codes_bytes);
    return __uint_as_float((uint32_t)s[((cb * L.n_kt + kt) * 16 + n) * L.gpt + g] << 16);
}

// sum_k x[k] W[k][n] of one column; x(k) gives the numbers
template <typename F>
__device__ __forceinline__ float dot_column(const char* blob, const Layout& L, int64_t n, F x)
{
    const int64_t cb = n / 16;
    const int c = (int)(n % 16);
    float y = 0.0f;
    for (int64_t kt = 0; kt < L.n_kt; ++kt)
        for (int g = 0; g < L.gpt; ++g) {
            float acc = 0.0f;
            for (int u = g * L.G / 16; u < (g + 1) * L.G / 16; ++u) {       // 16 k: dword t = u / 4 of lane 16 (u % 4) + c
                const uint32_t w = reinterpret_cast<const uint32_t*>(blob)[((cb * L.n_kt + kt) * 64 + 16 * (u % 4) + c) * 4 + u / 4];
                for (int i = 0; i < 16; ++i) {
                    const int q = (int)(w << (30 - 8 * (i % 4) - 2 * (i / 4))) >> 30;
                    acc += x(256 * kt + 16 * u + i) * (float)q;
                }
            }
            y += acc * scale_of(blob, L, cb, kt, c, g);
        }
    return y;
}

__global__ void __launch_bounds__(256) experts_up_kernel(ExpertsArgs a, float* h)
{
    const int64_t s = blockIdx.x, i = (int64_t)blockIdx.y * 256 + threadIdx.x;
    const int id = a.ids[s];
    if (id < 0 || id >= a.e.n_experts) return;
    const char* blob = (const char*)a.e.gate_up + id * a.e.gate_up_stride;
    const uint16_t* x = a.x + s / a.top_k * a.ldx;
    auto at = [&](int64_t k) { return __uint_as_float((uint32_t)x[k] << 16); };
    const int64_t n = i / 16 * 32 + i % 16;
    const float g = dot_column(blob, a.up, n, at), u = dot_column(blob, a.up, n + 16, at);
    h[s * a.e.inter + i] = g / (1.0f + expf(-g)) * u;
}

__global__ void __launch_bounds__(256) experts_down_kernel(ExpertsArgs a, const float* h)
{
    const int64_t m = blockIdx.x, n = (int64_t)blockIdx.y * 256 + threadIdx.x;
    float y = a.base ? __uint_as_float((uint32_t)a.base[m * a.ldb + n] << 16) : 0.0f;
    for (int j = 0; j < a.top_k; ++j) {
        const int64_t s = m * a.top_k + j;
        const int id = a.ids[s];
        if (id < 0 || id >= a.e.n_experts) continue;
        y += a.weights[s] * dot_column((const char*)a.e.down + id * a.e.down_stride, a.down, n, [&](int64_t k) { return h[s * a.e.inter + k]; });
    }
    a.Y[m * a.ldy + n] = (uint16_t)pack_bf16(y, y);
}

}  // namespace

size_t experts_workspace_bytes(const w2_experts_t& e, int64_t M, int top_k)
{
    return (size_t)M * top_k * e.inter * sizeof(float);
}

int launch_moe_experts(const ExpertsArgs& a, hipStream_t stream)
{
    float* const h = (float*)a.workspace;
    hipLaunchKernelGGL(experts_up_kernel, dim3((unsigned)(a.M * a.top_k), (unsigned)(a.e.inter / 256)), dim3(256), 0, stream, a, h);
    hipLaunchKernelGGL(experts_down_kernel, dim3((unsigned)a.M, (unsigned)(a.e.hidden / 256)), dim3(256), 0, stream, a, (const float*)h);
    return check_launch("w2_moe_experts");
}

}  // namespace w2
