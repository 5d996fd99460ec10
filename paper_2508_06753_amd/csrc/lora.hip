// Low-rank adapters of many requests beside a shared projection:
//   T[m,j] = sum_k X[m,k] A[a_m, j, k]      Y[m,n] = act(base[m,n] + scale * sum_r T[m, part(n) R + r] B[a_m, n, r]).
//
// Rows are taken in windows of 64, one a lane, and a window is sorted by adapter with ballots: the rows of one adapter (a
// tile, 1 to 64 of them) meet its factors together, whatever order the rows come in, and nothing has to be planned before
// the call.  An adapter's factors are read once a window.  Two launches: lora_shrink_kernel writes T, fp32, in `ks` parts
// of K; lora_expand_kernel adds them in order and finishes Y.  Matrix instructions 16x16x32 with the factors' rows on one
// side and the tile's rows on the other; numbers in 32 bits (T, and X if it is fp32) go in as two bf16 parts, 16 bits of
// mantissa, in two instructions.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "block_ops.h"

namespace w2 {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

constexpr int WINDOW = 64;

__device__ __forceinline__ v4f mfma(const v4i& a, const v4i& b, const v4f& c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    typedef float v2f __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f){lo, hi}, v2bf));
}

// eight floats as two bf16 parts whose sum has 16 bits of them
__device__ __forceinline__ void split_bf16(const float (&f)[8], v4i& hi, v4i& lo)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t h = pack_bf16(f[2 * e], f[2 * e + 1]);
        hi[e] = (int)h;
        lo[e] = (int)pack_bf16(f[2 * e] - __uint_as_float(h << 16), f[2 * e + 1] - __uint_as_float(h & 0xffff0000u));
    }
}

__device__ __forceinline__ int part_of(const LoraArgs& a, int block)
{
    if (a.gated) return block & 1;
    return (block >= a.end16[0]) + (block >= a.end16[1]) + (block >= a.end16[2]);
}

// One adapter's rows of a window.
struct Tile {
    int adapter;                         // -1: rows without one
    int rank, count, row;                // row: the window's row that is the lane-th of the tile
    float scale;
};

// The u-th adapter of the window (in the order of their first rows) that starts at row m0; false: there are not so many.
__device__ __forceinline__ bool find_tile(const LoraArgs& a, int64_t m0, int u, bool with_none, Tile& t)
{
    const int lane = threadIdx.x & 63;
    const bool there = m0 + lane < a.M;
    int ad = there ? a.adapter[m0 + lane] : -1;
    if (ad < 0 || ad >= a.n_adapters) ad = -1;
    uint64_t left = __ballot(there && (with_none || ad >= 0)), mine = 0;
    int which = -1;
    for (int v = 0; left; ++v) {
        which = __builtin_amdgcn_readlane(ad, __builtin_ctzll(left));
        mine = __ballot(there && ad == which);
        if (v == u) break;
        left &= ~mine;
    }
    if (!left) return false;
    t.adapter = which;
    t.count = __builtin_popcountll(mine);
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    const int at = mine >> lane & 1 ? __builtin_popcountll(mine & below) : t.count + __builtin_popcountll(~mine & below);
    t.row = __builtin_amdgcn_ds_permute(at * 4, lane);
    t.rank = which < 0 ? 0 : a.rank ? min(max(a.rank[which], 0), a.R) : a.R;
    t.scale = which < 0 || !a.scale ? 1.0f : a.scale[which];
    return true;
}

// ---------------------------------------------------------------------------------------------- T = X A^T
// A workgroup: one adapter's rows of a window, J * 16 rows of A, one of the ks ranges of K, cut again over its four waves.
// NR: row tiles of 16 that are multiplied together.
template <bool F32, int J, int NR>
__device__ __forceinline__ void shrink(const LoraArgs& a, const Tile& t, int64_t m0, int j0, int kb, int ke, v4f* part, float* T)
{
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int PR = a.n_parts * a.R;
    const uint16_t* ap[J];
#pragma unroll
    for (int j = 0; j < J; ++j) ap[j] = a.A + t.adapter * a.a_stride + (int64_t)min(j0 + 16 * j + l16, PR - 1) * a.K + 8 * q;
    const char* xp[NR];
    bool live[NR];
    int64_t row[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        live[n] = 16 * n + l16 < t.count;
        row[n] = m0 + __shfl(t.row, 16 * n + l16);
        xp[n] = (const char*)a.X + (row[n] * a.ldx + 8 * q) * (F32 ? 4 : 2);
    }
    v4f acc[J][NR];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int n = 0; n < NR; ++n) acc[j][n] = (v4f){0.f, 0.f, 0.f, 0.f};
    // U steps of 32: all loads first, then the products
    auto span = [&](int k, auto uc) {
        constexpr int U = decltype(uc)::value;
        v4i av[J][U], xv[NR][U * (F32 ? 2 : 1)];
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int u = 0; u < U; ++u) av[j][u] = *reinterpret_cast<const v4i*>(ap[j] + k + 32 * u);
#pragma unroll
        for (int n = 0; n < NR; ++n) {
#pragma unroll
            for (int u = 0; u < U * (F32 ? 2 : 1); ++u) xv[n][u] = (v4i){0, 0, 0, 0};
            if (live[n])                                     // (rows that are not there cost no memory traffic)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if constexpr (F32) {
                        xv[n][2 * u] = *reinterpret_cast<const v4i*>(xp[n] + (int64_t)(k + 32 * u) * 4);
                        xv[n][2 * u + 1] = *reinterpret_cast<const v4i*>(xp[n] + (int64_t)(k + 32 * u) * 4 + 16);
                    } else {
                        xv[n][u] = *reinterpret_cast<const v4i*>(xp[n] + (int64_t)(k + 32 * u) * 2);
                    }
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                if constexpr (F32) {
                    float f[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] = __int_as_float(xv[n][2 * u + e / 4][e % 4]);
                    v4i hi, lo;
                    split_bf16(f, hi, lo);
#pragma unroll
                    for (int j = 0; j < J; ++j) acc[j][n] = mfma(av[j][u], lo, mfma(av[j][u], hi, acc[j][n]));
                } else {
#pragma unroll
                    for (int j = 0; j < J; ++j) acc[j][n] = mfma(av[j][u], xv[n][u], acc[j][n]);
                }
            }
    };
    constexpr int U = J * NR >= 8 ? 2 : 4;
    int k = kb;
    for (; k + 32 * U <= ke; k += 32 * U) span(k, std::integral_constant<int, U>{});
    for (; k < ke; k += 32) span(k, std::integral_constant<int, 1>{});
    // the four waves' sums, in order; lane: row l16 of tile n, T's columns j0 + 16 j + 4 q ..+ 3
    __syncthreads();
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int n = 0; n < NR; ++n) part[((j * NR + n) * 4 + wave) * 64 + lane] = acc[j][n];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            if (((j * NR + n) & 3) != wave) continue;
            const v4f* p = part + (j * NR + n) * 4 * 64 + lane;
            const v4f s = p[0] + p[64] + p[128] + p[192];
            const int col = j0 + 16 * j + 4 * q;
            if (live[n] && col < PR) *reinterpret_cast<v4f*>(T + row[n] * PR + col) = s;
        }
}

template <bool F32, int J>
__global__ void __launch_bounds__(256) lora_shrink_kernel(LoraArgs a, int slots, int groups, int ks)
{
    extern __shared__ __align__(16) char smem[];
    // (slot, group of A's rows, range of K) of a window side by side
    uint32_t id = blockIdx.x;
    const int kr = id % ks;
    id /= ks;
    const int g = id % groups;
    id /= groups;
    const int slot = id % slots;
    const int64_t m0 = (int64_t)(id / slots) * WINDOW;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t steps = a.K / 32;
    const int kb = (int)(steps * (kr * 4 + wave) / (ks * 4)) * 32, ke = (int)(steps * (kr * 4 + wave + 1) / (ks * 4)) * 32;
    float* const T = a.T + (int64_t)kr * a.M * a.n_parts * a.R;
    const int j0 = g * J * 16;
    Tile t;
    for (int u = slot; find_tile(a, m0, u, false, t); u += slots) {
        // (nothing to do where every one of these rows of A is past the adapter's rank)
        bool any = false;
        for (int j = j0; j < min(j0 + J * 16, a.n_parts * a.R); j += 8) any |= j % a.R < t.rank;
        if (!any) continue;
        if (t.count <= 16) shrink<F32, J, 1>(a, t, m0, j0, kb, ke, (v4f*)smem, T);
        else if (t.count <= 32) shrink<F32, J, 2>(a, t, m0, j0, kb, ke, (v4f*)smem, T);
        else shrink<F32, J, 4>(a, t, m0, j0, kb, ke, (v4f*)smem, T);
    }
}

// ---------------------------------------------------------------------------------------------- Y
__device__ __forceinline__ float silu(float z) { return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }

// A workgroup: one adapter's rows of a window, `steps` times 64 columns a wave.  A wave's four matrix tiles take its 64
// columns in an order that leaves 16 (with the gated activation: 8 gate and the 8 up) columns of one row in a lane.
// S: steps of 32 ranks.
template <int S, bool PAIRED>
__global__ void __launch_bounds__(256) lora_expand_kernel(LoraArgs a, int slots, int groups, int steps, int ks, int row_tiles)
{
    extern __shared__ __align__(16) char smem[];             // T: [part][row tile][step][hi, lo][64 lanes] 16 bytes
    v4i* const ts = reinterpret_cast<v4i*>(smem);
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    uint32_t id = blockIdx.x;
    const int g = id % groups;
    id /= groups;
    const int slot = id % slots;
    const int64_t m0 = (int64_t)(id / slots) * WINDOW;
    const int PR = a.n_parts * a.R;
    const int64_t n_first = ((int64_t)g * steps * waves + wave) * 64;
    // the column (of the wave's 64) that row l16 of matrix tile t stands for
    auto column = [&](int t) {
        const int p = l16 >> 2, i = l16 & 3;
        return PAIRED ? 32 * (p >> 1) + 8 * (p & 1) + 4 * (t & 1) + i + 16 * (t >> 1) : 16 * p + 4 * t + i;
    };

    Tile t;
    for (int u = slot; find_tile(a, m0, u, true, t); u += slots) {
        const int tiles = (t.count + 15) / 16, live_steps = (t.rank + 31) / 32;
        if (t.rank == 0 && a.act == ACT_NONE && a.base == a.Y) continue;      // rows that stay where they are
        __syncthreads();                                     // (the tile before is done with local memory)
        for (int e = threadIdx.x; e < a.n_parts * tiles * live_steps * 64; e += blockDim.x) {
            const int s = e / 64 % live_steps, n = e / 64 / live_steps % tiles, p = e / 64 / live_steps / tiles;
            const int pos = 16 * n + l16, r = 32 * s + 8 * q;
            const int64_t row = m0 + __shfl(t.row, pos);
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = 0.0f;
            if (pos < t.count && r < t.rank) {
                const float* src = a.T + row * PR + p * a.R + r;
                for (int c = 0; c < ks; ++c, src += a.M * PR) {
                    const float4 x = *reinterpret_cast<const float4*>(src), y = *reinterpret_cast<const float4*>(src + 4);
                    f[0] += x.x; f[1] += x.y; f[2] += x.z; f[3] += x.w;
                    f[4] += y.x; f[5] += y.y; f[6] += y.z; f[7] += y.w;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = r + i < t.rank ? f[i] * t.scale : 0.0f;
            v4i hi, lo;
            split_bf16(f, hi, lo);
            v4i* dst = ts + ((p * row_tiles + n) * S + s) * 128 + lane;
            dst[0] = hi;
            dst[64] = lo;
        }
        __syncthreads();
        for (int step = 0; step < steps; ++step) {
            const int64_t n0 = n_first + (int64_t)step * waves * 64;
            if (n0 >= a.N) break;
            // operands: column(t)'s ranks 32 s + 8 q ..+ 7, nothing past the adapter's rank
            v4i bv[4][S];
            int part[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) part[h] = part_of(a, (int)((n0 + column(2 * h)) >> 4));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t n = n0 + column(i);
                const uint16_t* src = a.B + (int64_t)max(t.adapter, 0) * a.b_stride + n * a.R + 8 * q;
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    const int left = t.rank - 32 * s - 8 * q;
                    bv[i][s] = (v4i){0, 0, 0, 0};
                    if (left > 0 && n < a.N) bv[i][s] = *reinterpret_cast<const v4i*>(src + 32 * s);
                    if (t.rank & 7)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            bv[i][s][e] &= (int)((left > 2 * e ? 0xffffu : 0u) | (left > 2 * e + 1 ? 0xffff0000u : 0u));
                }
            }
            for (int n = 0; n < tiles; ++n) {
                const int64_t row = m0 + __shfl(t.row, 16 * n + l16);
                const bool live = 16 * n + l16 < t.count;
                // this lane's columns: 16 in a row, or 8 gate columns and the up columns 16 further
                const int64_t c0 = n0 + (PAIRED ? 32 * (q >> 1) + 8 * (q & 1) : 16 * q), c1 = c0 + (PAIRED ? 16 : 8);
                v4i b0 = {0, 0, 0, 0}, b1 = {0, 0, 0, 0};
                if (live && a.base) {
                    const uint16_t* src = a.base + row * a.ldb;
                    if (c0 < a.N) b0 = *reinterpret_cast<const v4i*>(src + c0);
                    if (c1 < a.N) b1 = *reinterpret_cast<const v4i*>(src + c1);
                }
                v4f acc[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i] = (v4f){0.f, 0.f, 0.f, 0.f};
                for (int p = 0; p < a.n_parts && t.rank > 0; ++p) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint64_t in = __ballot(part[h] == p);
                        if (!in) continue;
                        const bool some = in != ~(uint64_t)0, mine = part[h] == p;
#pragma unroll
                        for (int s = 0; s < S; ++s) {
                            if (s >= live_steps) break;
                            const v4i* src = ts + ((p * row_tiles + n) * S + s) * 128 + lane;
                            const v4i hi = src[0], lo = src[64];
#pragma unroll
                            for (int i = 2 * h; i < 2 * h + 2; ++i) {
                                v4i b = bv[i][s];
                                if (some && !mine) b = (v4i){0, 0, 0, 0};
                                acc[i] = mfma(b, hi, acc[i]);
                                acc[i] = mfma(b, lo, acc[i]);
                            }
                        }
                    }
                }
                if (!live) continue;
                float z[16];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t x = (uint32_t)b0[e / 2], y = (uint32_t)b1[e / 2];
                    z[e] = __uint_as_float(e & 1 ? x & 0xffff0000u : x << 16) + acc[e / 4][e % 4];
                    z[8 + e] = __uint_as_float(e & 1 ? y & 0xffff0000u : y << 16) + acc[2 + e / 4][e % 4];
                }
                v4i y0, y1;
                if constexpr (PAIRED) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        y0[e] = (int)pack_bf16(silu(z[2 * e]) * z[8 + 2 * e], silu(z[2 * e + 1]) * z[9 + 2 * e]);
                    if (c0 < a.N) *reinterpret_cast<v4i*>(a.Y + row * a.ldy + n0 / 2 + 8 * q) = y0;
                } else {
                    if (a.act == ACT_SILU)
#pragma unroll
                        for (int e = 0; e < 16; ++e) z[e] = silu(z[e]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        y0[e] = (int)pack_bf16(z[2 * e], z[2 * e + 1]);
                        y1[e] = (int)pack_bf16(z[8 + 2 * e], z[9 + 2 * e]);
                    }
                    if (c0 < a.N) *reinterpret_cast<v4i*>(a.Y + row * a.ldy + c0) = y0;
                    if (c1 < a.N) *reinterpret_cast<v4i*>(a.Y + row * a.ldy + c1) = y1;
                }
            }
        }
    }
}

struct Plan {
    int64_t windows;
    int slots;           // workgroups that share a window's adapters
    int J, groups, ks;   // shrink: 16-row tiles of A a workgroup, how many such, ranges of K
    int steps, columns;  // expand: steps of 256 columns a workgroup, how many such
};

Plan make_plan(int n_parts, int R, int n_adapters, int64_t M, int64_t K, int64_t N)
{
    Plan p;
    p.windows = (M + WINDOW - 1) / WINDOW;
    const int tiles = (n_parts * R + 15) / 16;
    p.J = p.windows > 4 ? 4 : 1;
    p.groups = (tiles + p.J - 1) / p.J;
    // as many slots as a window can have adapters while that is a few thousand workgroups
    int64_t slots = std::min<int64_t>(std::min<int64_t>(M, WINDOW), n_adapters);
    p.slots = (int)std::max<int64_t>(1, std::min<int64_t>(slots, 4096 / p.windows));
    // K cut until there are about two workgroups on every CU, a wave's share 64 or more
    const int64_t busy = std::min<int64_t>(M, p.windows - 1 + slots) * p.groups;
    p.ks = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(512 / std::max<int64_t>(busy, 1), 16), K / 256));
    const int64_t blocks = (N + 255) / 256;
    p.steps = (int)std::max<int64_t>(1, std::min<int64_t>(blocks, blocks * p.windows / 2048));
    p.columns = (int)((blocks + p.steps - 1) / p.steps);
    return p;
}

template <bool F32, int J>
int launch_shrink(const LoraArgs& a, const Plan& p, hipStream_t stream)
{
    const int row_tiles = a.M <= 16 ? 1 : a.M <= 32 ? 2 : 4, lds = J * row_tiles * 4096;
    if (int rc = ensure_dynamic_lds((const void*)lora_shrink_kernel<F32, J>, lds, "w2_lora_add")) return rc;
    const int64_t blocks = p.windows * p.slots * p.groups * p.ks;
    hipLaunchKernelGGL((lora_shrink_kernel<F32, J>), dim3((unsigned)blocks), dim3(256), lds, stream, a, p.slots, p.groups, p.ks);
    return check_launch("w2_lora_add");
}

template <int S, bool PAIRED>
int launch_expand(const LoraArgs& a, const Plan& p, hipStream_t stream)
{
    const int row_tiles = (int)std::min<int64_t>(4, (a.M + 15) / 16), lds = a.n_parts * row_tiles * S * 2048;
    if (int rc = ensure_dynamic_lds((const void*)lora_expand_kernel<S, PAIRED>, lds, "w2_lora_add")) return rc;
    // (one slot more: the rows without an adapter)
    const int slots = (int)std::min<int64_t>(std::min<int64_t>(a.M, WINDOW), p.slots + 1);
    const int64_t blocks = p.windows * slots * p.columns;
    hipLaunchKernelGGL((lora_expand_kernel<S, PAIRED>), dim3((unsigned)blocks), dim3(256), lds, stream, a, slots, p.columns, p.steps, p.ks, row_tiles);
    return check_launch("w2_lora_add");
}

}  // namespace

size_t lora_workspace_bytes(int n_parts, int R, int n_adapters, int64_t M, int64_t K, int64_t N)
{
    if (M == 0) return 0;
    return ((size_t)make_plan(n_parts, R, n_adapters, M, K, N).ks * M * n_parts * R * sizeof(float) + 255) & ~(size_t)255;
}

int launch_lora(const LoraArgs& a, hipStream_t stream)
{
    const Plan p = make_plan(a.n_parts, a.R, a.n_adapters, a.M, a.K, a.N);
    int rc;
    if (a.x_f32) rc = p.J == 1 ? launch_shrink<true, 1>(a, p, stream) : launch_shrink<true, 4>(a, p, stream);
    else rc = p.J == 1 ? launch_shrink<false, 1>(a, p, stream) : launch_shrink<false, 4>(a, p, stream);
    if (rc) return rc;
    const int S = (a.R + 31) / 32;
    if (a.act == ACT_SILU_MUL)
        return S == 1 ? launch_expand<1, true>(a, p, stream) : S == 2 ? launch_expand<2, true>(a, p, stream) : launch_expand<4, true>(a, p, stream);
    return S == 1 ? launch_expand<1, false>(a, p, stream) : S == 2 ? launch_expand<2, false>(a, p, stream) : launch_expand<4, false>(a, p, stream);
}

}  // namespace w2
