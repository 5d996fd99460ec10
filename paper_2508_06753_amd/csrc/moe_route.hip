// Which experts each row goes to: scores of the router's product, then the choice.
//
// The order of two scores decides which weights a row meets, so scores are computed in 64 bits: with sums in 32 bits about one row in
// ten thousand would pick another expert than exact arithmetic does.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ffn_ops.h"

namespace w2 {

namespace {

constexpr int ROWS = 8;

// One wave: one expert, ROWS rows.
__global__ void __launch_bounds__(256) route_logits_kernel(RouteArgs a, double* logits)
{
    const int lane = threadIdx.x & 63, e = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t m0 = (int64_t)blockIdx.y * ROWS;
    if (e >= a.r.n_experts) return;
    double acc[ROWS] = {};
    for (int64_t k = lane * 8; k < a.K; k += 512) {
        const uint4 w4 = *reinterpret_cast<const uint4*>(a.r.weight + e * a.r.ldw + k);
        const uint32_t wd[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (m0 + r >= a.M) break;
            const uint4 x4 = *reinterpret_cast<const uint4*>(a.x + (m0 + r) * a.ldx + k);
            const uint32_t xd[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                acc[r] = fma((double)__uint_as_float(xd[i] << 16), (double)__uint_as_float(wd[i] << 16), acc[r]);
                acc[r] = fma((double)__uint_as_float(xd[i] & 0xffff0000u), (double)__uint_as_float(wd[i] & 0xffff0000u), acc[r]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        for (int off = 32; off; off >>= 1) acc[r] += __shfl_xor(acc[r], off);
        if (lane == 0 && m0 + r < a.M) logits[(m0 + r) * a.r.n_experts + e] = acc[r];
    }
}

// A number as an unsigned integer of the same order, NaN below all; 0: not to be chosen
__device__ __forceinline__ uint64_t sortable(double c)
{
    if (c != c) return 1;
    if (c == 0) c = 0;                                       // -0 and 0 are equal
    const int64_t b = __double_as_longlong(c);
    return (uint64_t)(b < 0 ? ~b : b | (int64_t)1 << 63);
}

// One wave: one row.  Expert e in lane e / PER.
template <int PER>
__global__ void __launch_bounds__(64) route_select_kernel(RouteArgs a, const double* logits)
{
    __shared__ uint64_t s_key[1024];
    __shared__ double s_val[1024];
    const int lane = threadIdx.x, E = a.r.n_experts;
    const int64_t m = blockIdx.x;
    double l[PER], p[PER];
    uint64_t key[PER];
    double top = -INFINITY;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int e = lane * PER + j;
        l[j] = e < E ? logits[m * E + e] : 0.0;
        if (e < E) top = fmax(top, l[j]);
        if (a.logits && e < E) a.logits[m * E + e] = (float)l[j];
    }
    for (int off = 32; off; off >>= 1) top = fmax(top, __shfl_xor(top, off));
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const bool is = lane * PER + j < E;
        p[j] = a.r.score == W2_SCORE_SOFTMAX ? exp(l[j] - top) : 1.0 / (1.0 + exp(-l[j]));
        if (is) sum += p[j];
    }
    if (a.r.score == W2_SCORE_SOFTMAX) {
        for (int off = 32; off; off >>= 1) sum += __shfl_xor(sum, off);
#pragma unroll
        for (int j = 0; j < PER; ++j) p[j] /= sum;
    }
    // without a bias and without sums over groups the scores' own order decides: it does not run out of digits
    const bool by_logit = !a.r.choice_bias && (a.r.n_groups == 1 || a.r.group_top == 1);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int e = lane * PER + j;
        const double c = by_logit ? l[j] : a.r.choice_bias && e < E ? p[j] + (double)a.r.choice_bias[e] : p[j];
        key[j] = e < E ? sortable(c) : 0;
        s_key[e] = key[j];
        s_val[e] = c;
    }
    if (a.r.n_groups > 1) {
        __syncthreads();
        const int size = E / a.r.n_groups;
        // lane g: the score of group g
        uint64_t score = 0;
        if (lane < a.r.n_groups) {
            double first = -INFINITY, second = -INFINITY;
            for (int i = 0; i < size; ++i) {
                const double c = s_val[lane * size + i];
                if (c > first) { second = first; first = c; }
                else if (c > second) second = c;
            }
            score = sortable(a.r.group_top == 2 && size > 1 ? first + second : first);
        }
        int better = 0;
        for (int g = 0; g < a.r.n_groups; ++g) {
            const uint64_t other = __shfl(score, g);
            better += other > score || (other == score && g < lane);
        }
        const uint64_t open = __ballot(lane < a.r.n_groups && better < a.r.top_groups);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int e = lane * PER + j;
            if (e < E && !(open >> (e / size) & 1)) key[j] = 0;
        }
    }
    int my_id = 0;
    double my_p = 0.0;
    for (int i = 0; i < a.r.top_k; ++i) {
        uint64_t best = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) best = max(best, key[j]);
        uint64_t all = best;
        for (int off = 32; off; off >>= 1) all = max(all, (uint64_t)__shfl_xor((unsigned long long)all, off));
        const int winner = __ffsll(__ballot(best == all)) - 1;
        int id = 0;
        double pv = 0.0;
#pragma unroll
        for (int j = PER - 1; j >= 0; --j)
            if (key[j] == all) { id = lane * PER + j; pv = p[j]; }
        id = __shfl(id, winner);
        pv = __shfl(pv, winner);
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (lane * PER + j == id) key[j] = 0;
        if (lane == i) { my_id = id; my_p = pv; }
    }
    double total = lane < a.r.top_k ? my_p : 0.0;
    for (int off = 32; off; off >>= 1) total += __shfl_xor(total, off);
    if (lane < a.r.top_k) {
        a.ids[m * a.r.top_k + lane] = my_id;
        a.weights[m * a.r.top_k + lane] = (float)((a.r.renormalise ? my_p / total : my_p) * (double)a.r.scale);
    }
}

}  // namespace

size_t route_workspace_bytes(int n_experts, int64_t M, int64_t)
{
    return (size_t)M * n_experts * sizeof(double);
}

int launch_moe_route(const RouteArgs& a, hipStream_t stream)
{
    double* const logits = (double*)a.workspace;
    const int E = a.r.n_experts;
    RouteArgs b = a;
    for (int64_t m0 = 0; m0 < a.M; m0 += (int64_t)ROWS * 65535) {          // grid y is limited to 65535
        b.M = std::min(a.M - m0, (int64_t)ROWS * 65535);
        b.x = a.x + m0 * a.ldx;
        hipLaunchKernelGGL(route_logits_kernel, dim3((E + 3) / 4, (unsigned)((b.M + ROWS - 1) / ROWS)), dim3(256), 0, stream, b, logits + m0 * E);
    }
    auto select = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)a.M), dim3(64), 0, stream, a, (const double*)logits); };
    if (E <= 64) select(route_select_kernel<1>);
    else if (E <= 128) select(route_select_kernel<2>);
    else if (E <= 256) select(route_select_kernel<4>);
    else if (E <= 512) select(route_select_kernel<8>);
    else select(route_select_kernel<16>);
    return check_launch("w2_moe_route");
}

}  // namespace w2
