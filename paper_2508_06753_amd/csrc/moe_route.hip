// Which experts each row goes to: scores of the router's product, then the choice.
//
// The order of two scores decides which weights a row meets, so scores are computed in 64 bits: with sums in 32 bits about one row in
// ten thousand would pick another expert than exact arithmetic does.  A product of two bf16 numbers has 16 bits, so sums of
// 2^20 of them in 64 are as good as exact.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ffn_ops.h"

namespace w2 {

namespace {

typedef double v4d __attribute__((ext_vector_type(4)));

constexpr int WAVES = 8;

// Bound: many rows by the products (4095 rows, 4096 x 64: 2.1 GFLOP, 31 us at the 64-bit rate of the card, 41 + 5 for the choice (43 with one block of K under way instead of four); with bf16 products and
// sums in 32 bits it would be the 7 us that x takes from memory, but see above); few by latency (1 row, 128 experts of 4096: 8.9 us for both launches;
// 11.3 with vector instructions).  T = 2 (each number read meets twice as many) from 192 workgroups on.
//
// A workgroup: 16 T rows by 16 T experts, one of the parts of K, eight waves that share it out.  The matrix instruction is the one for
// 64-bit numbers (16 x 16 x 4); a lane asks for 8 numbers of a row in a row of memory, and step i multiplies the i-th of
// them: which of K's numbers those are is the same on both sides.  Sums of the waves meet in their order.
template <int T>
__global__ void __launch_bounds__(WAVES * 64) route_logits_kernel(RouteArgs a, double* part, int parts)
{
    __shared__ double s_sum[WAVES][T * T][256];
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, q = lane >> 4, wave = tid >> 6;
    const int E = a.r.n_experts;
    const int64_t m0 = (int64_t)blockIdx.x * (16 * T);
    const int e0 = blockIdx.y * (16 * T);
    const int blocks = (int)((a.K + 31) / 32), ranges = parts * WAVES, range = blockIdx.z * WAVES + wave;
    const int begin = (int)((int64_t)blocks * range / ranges), end = (int)((int64_t)blocks * (range + 1) / ranges);
    const uint16_t *x[T], *w[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {       // (rows and experts that are not there: the last one again)
        x[t] = a.x + min(m0 + t * 16 + col, a.M - 1) * a.ldx + q * 8;
        w[t] = a.r.weight + (int64_t)min(e0 + t * 16 + col, E - 1) * a.r.ldw + q * 8;
    }
    v4d acc[T][T] = {};
    auto at = [](const uint4& v, int i) -> double {
        const uint32_t d = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
        return (double)__uint_as_float(i & 1 ? d & 0xffff0000u : d << 16);
    };
    auto multiply = [&](const uint4 (&xs)[T], const uint4 (&ws)[T]) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int r = 0; r < T; ++r)
#pragma unroll
                for (int c = 0; c < T; ++c) acc[r][c] = __builtin_amdgcn_mfma_f64_16x16x4f64(at(xs[r], i), at(ws[c], i), acc[r][c], 0, 0, 0);
    };
    auto load = [&](int b, uint4 (&to_x)[T], uint4 (&to_w)[T]) {
#pragma unroll
        for (int t = 0; t < T; ++t) {
            to_x[t] = *reinterpret_cast<const uint4*>(x[t] + (int64_t)b * 32);
            to_w[t] = *reinterpret_cast<const uint4*>(w[t] + (int64_t)b * 32);
        }
    };
    auto load_rest = [&](int b, uint4 (&to_x)[T], uint4 (&to_w)[T]) {            // K % 8 == 0: eight numbers or none
#pragma unroll
        for (int t = 0; t < T; ++t) to_x[t] = to_w[t] = make_uint4(0, 0, 0, 0);
        if (b * 32 + q * 8 < a.K) load(b, to_x, to_w);
    };
    if constexpr (T == 1) {             // a few blocks a wave: one ahead, and little code to fetch
        uint4 xs[T], ws[T], xn[T], wn[T];
        if (begin < end) load_rest(begin, xn, wn);
        for (int b = begin; b < end; ++b) {
            xs[0] = xn[0];
            ws[0] = wn[0];
            if (b + 1 < end) load_rest(b + 1, xn, wn);
            multiply(xs, ws);
        }
    } else {                            // all of K: whole blocks, four under way (past the last one that one again), then what is left
        constexpr int AHEAD = 4;
        const int whole = min(end, (int)(a.K / 32));
        uint4 xs[AHEAD][T], ws[AHEAD][T];
        if (begin < whole) {
#pragma unroll
            for (int d = 0; d < AHEAD; ++d) {
                load(min(begin + d, whole - 1), xs[d], ws[d]);
                __builtin_amdgcn_sched_barrier(0);
            }
            int b = begin;
            for (; b + AHEAD <= whole; b += AHEAD) {
#pragma unroll
                for (int d = 0; d < AHEAD; ++d) {
                    multiply(xs[d], ws[d]);
                    __builtin_amdgcn_sched_barrier(0);
                    load(min(b + d + AHEAD, whole - 1), xs[d], ws[d]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
#pragma unroll
            for (int d = 0; d < AHEAD - 1; ++d)
                if (b + d < whole) multiply(xs[d], ws[d]);
        }
        if (whole < end) {
            load_rest(whole, xs[0], ws[0]);
            multiply(xs[0], ws[0]);
        }
    }
    // number i of a lane: row 4 i + q, column col
#pragma unroll
    for (int r = 0; r < T; ++r)
#pragma unroll
        for (int c = 0; c < T; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) s_sum[wave][r * T + c][(4 * i + q) * 16 + col] = acc[r][c][i];
    __syncthreads();
    for (int o = tid; o < T * T * 256; o += WAVES * 64) {
        const int t = o / 256, in = o % 256;
        const int64_t m = m0 + t / T * 16 + in / 16;
        const int e = e0 + t % T * 16 + in % 16;
        double s = s_sum[0][t][in];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) s += s_sum[v][t][in];
        if (m < a.M && e < E) part[((int64_t)blockIdx.z * a.M + m) * E + e] = s;
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

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v)           // the same in every lane
{
    auto move = [](uint32_t x, auto ctrl) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xf, 0xf, true); };
    v = max(v, move(v, std::integral_constant<int, 0xB1>{}));
    v = max(v, move(v, std::integral_constant<int, 0x4E>{}));
    v = max(v, move(v, std::integral_constant<int, 0x141>{}));
    v = max(v, move(v, std::integral_constant<int, 0x140>{}));
    const uint32_t r0 = __builtin_amdgcn_readlane(v, 0), r1 = __builtin_amdgcn_readlane(v, 16);
    const uint32_t r2 = __builtin_amdgcn_readlane(v, 32), r3 = __builtin_amdgcn_readlane(v, 48);
    return max(max(r0, r1), max(r2, r3));
}

template <int CTRL>
__device__ __forceinline__ double move(double v)
{
    const int64_t b = __double_as_longlong(v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, CTRL, 0xf, 0xf, true), hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, 0xf, 0xf, true);
    return __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}

__device__ __forceinline__ double lane_of(double v, int lane)          // (lane: the same in every lane)
{
    const int64_t b = __double_as_longlong(v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)b, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(b >> 32), lane);
    return __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}

// op over the lanes of a wave, the same in every lane: moves inside rows of 16, then the four rows' in their order
template <typename F>
__device__ __forceinline__ double over_wave(double v, F op)
{
    v = op(v, move<0xB1>(v));
    v = op(v, move<0x4E>(v));
    v = op(v, move<0x141>(v));
    v = op(v, move<0x140>(v));
    return op(op(lane_of(v, 0), lane_of(v, 16)), op(lane_of(v, 32), lane_of(v, 48)));
}

__device__ __forceinline__ double wave_max(double v)
{
    return over_wave(v, [](double a, double b) { return fmax(a, b); });
}

__device__ __forceinline__ double wave_total(double v)
{
    return over_wave(v, [](double a, double b) { return a + b; });
}

// One wave: one row, expert e in lane e / PER; four rows a workgroup.  The largest key of the wave is found by its upper
// 32 bits, moves that ride on the comparison, and by the lower ones where two lanes share those: a round of the choice is 150 cycles
// (53 rows, 8 of 256 experts in groups: 7 us for the scores and 8 here; 29.9 together with vector sums and a butterfly of 64-bit shuffles).
template <int PER, bool GROUPS>
__global__ void __launch_bounds__(256) route_select_kernel(RouteArgs a, const double* part, int parts)
{
    extern __shared__ double s_all[];                        // GROUPS: [4][64 * PER]
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, E = a.r.n_experts;
    const int64_t m = (int64_t)blockIdx.x * 4 + wave;
    if (m >= a.M) return;
    double l[PER], p[PER];
    uint64_t key[PER];
    double top = -INFINITY;
#pragma unroll
    for (int j = 0; j < PER; ++j) l[j] = 0.0;
    constexpr int AT_ONCE = PER <= 4 ? 8 : 16 / PER;         // parts whose sums are under way together
    for (int s0 = 0; s0 < parts; s0 += AT_ONCE) {
        double v[AT_ONCE][PER];
#pragma unroll
        for (int s = 0; s < AT_ONCE; ++s)
#pragma unroll
            for (int j = 0; j < PER; ++j)
                v[s][j] = s0 + s < parts && lane * PER + j < E ? part[((int64_t)(s0 + s) * a.M + m) * E + lane * PER + j] : 0.0;
#pragma unroll
        for (int s = 0; s < AT_ONCE; ++s)
#pragma unroll
            for (int j = 0; j < PER; ++j) l[j] += v[s][j];
    }
#pragma unroll
    for (int j = 0; j < PER; ++j)
        if (lane * PER + j < E) {
            top = fmax(top, l[j]);
            if (a.logits) a.logits[m * E + lane * PER + j] = (float)l[j];
        }
    if (a.r.score == W2_SCORE_SOFTMAX) {
        top = wave_max(top);
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            p[j] = lane * PER + j < E ? exp(l[j] - top) : 0.0;
            sum += p[j];
        }
        sum = wave_total(sum);
#pragma unroll
        for (int j = 0; j < PER; ++j) p[j] /= sum;
    } else {
#pragma unroll
        for (int j = 0; j < PER; ++j) p[j] = 1.0 / (1.0 + exp(-l[j]));
    }
    // without a bias the scores' own order decides, which does not run out of digits; a sum over a group is one of p
    const bool by_logit = !a.r.choice_bias, group_by_logit = by_logit && a.r.group_top == 1;
    double* const s_val = s_all + wave * (64 * PER);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int e = lane * PER + j;
        double c = by_logit ? l[j] : p[j];
        if (a.r.choice_bias && e < E) c += (double)a.r.choice_bias[e];
        key[j] = e < E ? sortable(c) : 0;
        if constexpr (GROUPS) {
            if (by_logit && !group_by_logit) c = p[j];
            s_val[e] = c == c ? c : -INFINITY;
        }
    }
    if constexpr (GROUPS) {
        // (a wave's own part of local memory, in order: no barrier)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int size = E / a.r.n_groups;
        int lanes = 1;                                       // of a group, a power of two
        while (2 * lanes * a.r.n_groups <= 64) lanes *= 2;
        const int g = lane / lanes;
        double first = -INFINITY, second = -INFINITY;
        if (g < a.r.n_groups)
            for (int i = lane % lanes; i < size; i += lanes) {
                const double c = s_val[g * size + i];
                second = fmax(second, fmin(first, c));
                first = fmax(first, c);
            }
        for (int off = 1; off < lanes; off <<= 1) {
            const double f = __shfl_xor(first, off), s = __shfl_xor(second, off);
            second = fmax(fmin(first, f), fmax(second, s));
            first = fmax(first, f);
        }
        const uint64_t score = sortable(a.r.group_top == 2 && size > 1 ? first + second : first);
        int better = 0;
        for (int o = 0; o < a.r.n_groups; ++o) {
            const uint64_t other = (uint64_t)__double_as_longlong(lane_of(__longlong_as_double((int64_t)score), o * lanes));
            better += other > score || (other == score && o < g);
        }
        const uint64_t open = __ballot(lane % lanes == 0 && g < a.r.n_groups && better < a.r.top_groups);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int e = lane * PER + j;
            if (e < E && !(open >> (e / size * lanes) & 1)) key[j] = 0;
        }
    }
    int my_id = 0;
    double my_p = 0.0;
    for (int i = 0; i < a.r.top_k; ++i) {
        uint64_t best = 0;
        int id = 0;
        double pv = 0.0;
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (key[j] > best || j == 0) {
                best = key[j];
                id = lane * PER + j;
                pv = p[j];
            }
        uint64_t winners = __ballot((uint32_t)(best >> 32) == wave_max_u32((uint32_t)(best >> 32)));
        if (winners & (winners - 1)) {                       // (the lane's own upper half again where it lost: 0 below all keys)
            const uint32_t low = winners >> lane & 1 ? (uint32_t)best : 0;
            winners &= __ballot(low == wave_max_u32(low));
        }
        const int winner = __ffsll((unsigned long long)winners) - 1;
        id = __builtin_amdgcn_readlane(id, winner);
        const int64_t pb = __double_as_longlong(pv);
        const uint32_t p0 = __builtin_amdgcn_readlane((int)pb, winner), p1 = __builtin_amdgcn_readlane((int)(pb >> 32), winner);
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (lane * PER + j == id) key[j] = 0;
        if (lane == i) {
            my_id = id;
            my_p = __longlong_as_double((int64_t)((uint64_t)p1 << 32 | p0));
        }
    }
    double total = a.r.renormalise ? wave_total(lane < a.r.top_k ? my_p : 0.0) : 1.0;
    if (total < 0x1p-900) {
        // All the chosen ones' p are next to nothing: quotients of their exponentials beside the largest one's.  (A sigmoid is exp(l) there to
        // 2^-900 of itself; above, a p that lost digits is below 2^-100 of the sum.)
        double my_l = 0.0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const double v = __shfl(l[j], my_id / PER);
            if (my_id % PER == j) my_l = v;
        }
        const double largest = wave_max(lane < a.r.top_k ? my_l : -INFINITY);
        my_p = exp(my_l - largest);
        total = wave_total(lane < a.r.top_k ? my_p : 0.0);
    }
    if (lane < a.r.top_k) {
        a.ids[m * a.r.top_k + lane] = my_id;
        a.weights[m * a.r.top_k + lane] = (float)(my_p / total * (double)a.r.scale);
    }
}

struct Shape {
    int t, parts;
};

// Parts of K across workgroups until there are two to a CU
Shape shape(int E, int64_t M, int64_t K)
{
    Shape s;
    const int64_t wide = ((M + 31) / 32) * ((E + 31) / 32), narrow = ((M + 15) / 16) * ((E + 15) / 16);
    s.t = wide >= 192 ? 2 : 1;
    s.parts = s.t == 2 ? 1 : (int)std::min<int64_t>(std::min<int64_t>(8, std::max<int64_t>(1, 512 / narrow)), std::max<int64_t>(1, K / 256));
    return s;
}

}  // namespace

// (no less for more rows: parts * M * n_experts is at most 512 * 256 sums where there are parts)
size_t route_workspace_bytes(int n_experts, int64_t M, int64_t)
{
    return (size_t)std::min<int64_t>(8 * M, M + (512 * 256 + n_experts - 1) / n_experts) * n_experts * sizeof(double);
}

int launch_moe_route(const RouteArgs& a, hipStream_t stream)
{
    double* const part = (double*)a.workspace;
    const int E = a.r.n_experts;
    const Shape s = shape(E, a.M, a.K);
    auto logits = [&](auto kern, int t) {
        hipLaunchKernelGGL(kern, dim3((unsigned)((a.M + 16 * t - 1) / (16 * t)), (unsigned)((E + 16 * t - 1) / (16 * t)), (unsigned)s.parts), dim3(WAVES * 64), 0,
                           stream, a, part, s.parts);
    };
    if (s.t == 2) logits(route_logits_kernel<2>, 2);
    else logits(route_logits_kernel<1>, 1);
    auto select = [&](auto per) {
        constexpr int PER = decltype(per)::value;
        const dim3 grid((unsigned)((a.M + 3) / 4));
        if (a.r.n_groups > 1) hipLaunchKernelGGL((route_select_kernel<PER, true>), grid, dim3(256), 4 * 64 * PER * sizeof(double), stream, a, (const double*)part, s.parts);
        else hipLaunchKernelGGL((route_select_kernel<PER, false>), grid, dim3(256), 0, stream, a, (const double*)part, s.parts);
    };
    if (E <= 64) select(std::integral_constant<int, 1>{});
    else if (E <= 128) select(std::integral_constant<int, 2>{});
    else if (E <= 256) select(std::integral_constant<int, 4>{});
    else if (E <= 512) select(std::integral_constant<int, 8>{});
    else select(std::integral_constant<int, 16>{});
    return check_launch("w2_moe_route");
}

}  // namespace w2
