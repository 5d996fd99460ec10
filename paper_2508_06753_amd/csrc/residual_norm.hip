// What stands between two blocks, in one pass over the rows: norm of a block's output, gate, residual scale, the sum, norm
// before the next block, and if asked for the next projection's int8 rows (8191 rows of 5120: 8 us more, w2_quantize_rows behind it 22).
//
// A workgroup takes a row and keeps it in registers (NV vectors of 8 numbers a thread), so that each number is read once and
// written once however many sums the row needs: mean(y^2) where the block's output is normed, mean(r'^2), the abs-max of x
// where it is quantised.  A sum is reduced by moves inside the waves and one trip through local memory.  Sums and what is between the
// roundings of r' (none in 32 bits) and x are in fp32; mean(r'^2) takes r' before its rounding.
//
// Bound: many rows by memory (8191 rows of 5120, residual in 32 bits: 503 MB in 95 us, 5.3 TB/s, above the 4.75 of a large copy), few by the launch
// (1 row of 4096: 6.3 us by the host's clock; 77 rows of 5120 with gate 6.9).  Threads a row: 512 for up to 64 rows, whose trips to
// memory are then one, 256 for more, so that several rows share a CU; not more than 4 vectors a thread where 1024 threads allow it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "block_ops.h"
#include "ffn_ops.h"

namespace w2 {

namespace {

__device__ __forceinline__ float wave_sum(float v)           // the same in every lane
{
    v += dpp_move_f32<0xB1>(v);                              // quad_perm [1,0,3,2]
    v += dpp_move_f32<0x4E>(v);                              // quad_perm [2,3,0,1]
    v += dpp_move_f32<0x141>(v);                             // row_half_mirror
    v += dpp_move_f32<0x140>(v);                             // row_mirror
    const int b = __float_as_int(v);
    const float r0 = __int_as_float(__builtin_amdgcn_readlane(b, 0)), r1 = __int_as_float(__builtin_amdgcn_readlane(b, 16));
    const float r2 = __int_as_float(__builtin_amdgcn_readlane(b, 32)), r3 = __int_as_float(__builtin_amdgcn_readlane(b, 48));
    return (r0 + r1) + (r2 + r3);
}

__device__ __forceinline__ float bf16_at(const uint4& v, int i)
{
    const uint32_t w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
}

template <int NV, bool RBF>
__global__ void __launch_bounds__(1024) residual_norm_kernel(NormArgs a, int64_t m0, float inv_n)
{
    __shared__ float s_red[3][16];
    const int64_t m = m0 + blockIdx.x;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, n_waves = blockDim.x >> 6;
    const int step = blockDim.x * 8;
    const int N = (int)a.N;

    // Everything the row needs is asked for before the first sum waits; of more than 4 vectors a thread only y, the others where they are
    // used: together they would be up to 192 registers of the 128 that 1024 threads have (141 were spilled, and the row
    // went to memory and back: 1000 gated rows of 65536, residual in 32 bits, 332 us; now 187, 4.9 TB/s).
    constexpr bool EARLY = NV <= 4;
    constexpr int NE = EARLY ? NV : 1;
    uint4 y[NV], g[NE], w[NE], pw[NE], r0[NE], r1[NE];
    const uint4 zero = make_uint4(0, 0, 0, 0);
    auto load_others = [&](int e, int n) {
        g[e] = pw[e] = r0[e] = r1[e] = zero;
        if (n < N) {
            if (a.residual) {
                if constexpr (RBF) r0[e] = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(a.residual) + m * a.ldr + n);
                else {
                    const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const float*>(a.residual) + m * a.ldr + n);
                    r0[e] = p[0];
                    r1[e] = p[1];
                }
            }
            if (a.p.gate) g[e] = *reinterpret_cast<const uint4*>(a.p.gate + m * a.p.ld_gate + n);
            if (a.p.post_weight) pw[e] = *reinterpret_cast<const uint4*>(a.p.post_weight + n);
        }
    };
    auto load_weight = [&](int e, int n) {
        w[e] = zero;
        if (n < N && a.p.weight) w[e] = *reinterpret_cast<const uint4*>(a.p.weight + n);
    };
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int n = tid * 8 + v * step;
        y[v] = zero;
        if (n < N && a.y) y[v] = *reinterpret_cast<const uint4*>(a.y + m * a.ldy + n);
        if constexpr (EARLY) {
            load_others(v, n);
            load_weight(v, n);
        }
    }
    auto total = [&](float s, int slot) -> float {
        s = wave_sum(s);
        if (n_waves == 1) return s;
        if (lane == 0) s_red[slot][wave] = s;
        __syncthreads();
        return wave_sum(lane < n_waves ? s_red[slot][lane] : 0.0f);
    };

    float post = 1.0f;
    if (a.p.post_norm && a.y) {         // (none: zero, with eps = 0 too)
        float s = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(bf16_at(y[v], i), bf16_at(y[v], i), s);
        post = 1.0f / sqrtf(total(s, 0) * inv_n + a.p.eps);
    }
    float r[NV][8], s = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int n = tid * 8 + v * step, e = EARLY ? v : 0;
        if constexpr (!EARLY) load_others(e, n);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float b = bf16_at(y[v], i);
            if (a.p.post_norm) b = a.p.post_weight ? b * post * (bf16_at(pw[e], i) + a.p.weight_offset) : b * post;
            if (a.p.gate) b *= bf16_at(g[e], i);
            float old;
            if constexpr (RBF) old = bf16_at(r0[e], i);
            else old = __uint_as_float(i < 4 ? (&r0[e].x)[i & 3] : (&r1[e].x)[i & 3]);
            r[v][i] = fmaf(a.p.residual_scale, old, a.p.block_scale * b);
            s = fmaf(r[v][i], r[v][i], s);
        }
        if (a.residual_out && n < N) {
            if constexpr (RBF) {
                *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(a.residual_out) + m * a.ldro + n) =
                    make_uint4(pack_bf16(r[v][0], r[v][1]), pack_bf16(r[v][2], r[v][3]), pack_bf16(r[v][4], r[v][5]), pack_bf16(r[v][6], r[v][7]));
            } else {
                float4* p = reinterpret_cast<float4*>(reinterpret_cast<float*>(a.residual_out) + m * a.ldro + n);
                p[0] = make_float4(r[v][0], r[v][1], r[v][2], r[v][3]);
                p[1] = make_float4(r[v][4], r[v][5], r[v][6], r[v][7]);
            }
        }
    }
    if (!a.x && !a.xq) return;
    const float f = 1.0f / sqrtf(total(s, 1) * inv_n + a.p.eps);
    uint4 out[NV];
    float amax = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        float t[8];
        const int n = tid * 8 + v * step, e = EARLY ? v : 0;
        if constexpr (!EARLY) load_weight(e, n);
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = a.p.weight ? r[v][i] * f * (bf16_at(w[e], i) + a.p.weight_offset) : r[v][i] * f;
        out[v] = make_uint4(pack_bf16(t[0], t[1]), pack_bf16(t[2], t[3]), pack_bf16(t[4], t[5]), pack_bf16(t[6], t[7]));
        if (n < N) {
            if (a.x) *reinterpret_cast<uint4*>(a.x + m * a.ldx + n) = out[v];
#pragma unroll
            for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(bf16_at(out[v], i)));
        }
    }
    if (!a.xq) return;
    amax = wave_max_f32(amax);
    if (n_waves > 1) {
        if (lane == 0) s_red[2][wave] = amax;
        __syncthreads();
        amax = wave_max_f32(lane < n_waves ? s_red[2][lane] : 0.0f);
    }
    const float inv = amax > 0.0f ? __fdiv_rn(127.0f, amax) : 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int n = tid * 8 + v * step;
        if (n >= N) continue;
        uint32_t q[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) b[i] = quantised_bits(bf16_at(out[v], 4 * h + i), inv);
            q[h] = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u) | __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
        }
        *reinterpret_cast<uint2*>(a.xq + m * N + n) = make_uint2(q[0], q[1]);
    }
    if (tid == 0) a.sx[m] = amax > 0.0f ? __fdiv_rn(amax, 127.0f) : 0.0f;
}

// a launch has fewer than 2^32 threads
constexpr int64_t ROWS_A_LAUNCH = (int64_t)1 << 20;

}  // namespace

int launch_residual_norm(const NormArgs& a, hipStream_t stream)
{
    const int64_t vecs = a.N / 8;
    int threads = a.M <= 64 ? 512 : 256;
    while (threads < 1024 && vecs > (int64_t)4 * threads) threads <<= 1;
    while (threads > 64 && threads / 2 >= vecs) threads >>= 1;
    const int64_t nv = (vecs + threads - 1) / threads;
    const float inv_n = (float)(1.0 / (double)a.N);
    auto go = [&](auto nv_c) {
        constexpr int NV = decltype(nv_c)::value;
        for (int64_t m0 = 0; m0 < a.M; m0 += ROWS_A_LAUNCH) {
            const dim3 grid((unsigned)std::min(ROWS_A_LAUNCH, a.M - m0));
            if (a.r_bf16) hipLaunchKernelGGL((residual_norm_kernel<NV, true>), grid, dim3(threads), 0, stream, a, m0, inv_n);
            else hipLaunchKernelGGL((residual_norm_kernel<NV, false>), grid, dim3(threads), 0, stream, a, m0, inv_n);
        }
        return check_launch("w2_residual_norm");
    };
    if (nv <= 1) return go(std::integral_constant<int, 1>{});
    if (nv <= 2) return go(std::integral_constant<int, 2>{});
    if (nv <= 3) return go(std::integral_constant<int, 3>{});
    if (nv <= 4) return go(std::integral_constant<int, 4>{});
    return go(std::integral_constant<int, 8>{});
}

}  // namespace w2
