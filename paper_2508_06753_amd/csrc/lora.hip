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
#ifndef LW
#define LW 512
#endif
#ifndef JJ
#define JJ 2
#endif
#ifndef ST
#define ST 2048
#endif
#ifndef OC
#define OC 1
#endif

__device__ __forceinline__ v4f mfma(const v4i& a, const v4i& b, const v4f& c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
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
    int count, row;                      // row: the window's row that is the lane-th of the tile
};

// A window's rows by adapter: the lane's row's, -1 for none; rows past the last one: -2.
__device__ __forceinline__ int window_adapters(const LoraArgs& a, int64_t m0)
{
    const int64_t m = m0 + (threadIdx.x & 63);
    if (m >= a.M) return -2;
    const int ad = a.adapter[m];
    return ad < 0 || ad >= a.n_adapters ? -1 : ad;
}

__device__ __forceinline__ Tile make_tile(int which, uint64_t mine)
{
    const int lane = threadIdx.x & 63;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    Tile t;
    t.adapter = which;
    t.count = __builtin_popcountll(mine);
    const int at = mine >> lane & 1 ? __builtin_popcountll(mine & below) : t.count + __builtin_popcountll(~mine & below);
    t.row = __builtin_amdgcn_ds_permute(at * 4, lane);
    return t;
}

// Calls f(tile) for the tiles of a window that are this workgroup's.  As many slots as rows: the tile whose first row is the
// slot-th (no search: a small batch waits for one load).  Else the slot-th, (slot + slots)-th ... adapter in the order of
// their first rows.
template <typename F>
__device__ __forceinline__ void for_tiles(const LoraArgs& a, int64_t m0, int slot, int slots, bool with_none, F f)
{
    const int ad = window_adapters(a, m0);
    if (slots >= WINDOW || slots >= a.M) {
        const int which = __builtin_amdgcn_readlane(ad, slot);
        const uint64_t mine = __builtin_amdgcn_ballot_w64(ad == which);
        if (which >= (with_none ? -1 : 0) && __builtin_ctzll(mine) == slot) f(make_tile(which, mine));
        return;
    }
    uint64_t left = __builtin_amdgcn_ballot_w64(ad >= (with_none ? -1 : 0));
    for (int u = 0; left; ++u) {
        const int which = __builtin_amdgcn_readlane(ad, __builtin_ctzll(left));
        const uint64_t mine = __builtin_amdgcn_ballot_w64(ad == which);
        left &= ~mine;
        if (u == slot) {
            f(make_tile(which, mine));
            slot += slots;
        }
    }
}

__device__ __forceinline__ int rank_of(const LoraArgs& a, int which)
{
    if (which < 0) return 0;
    return a.rank ? min(max(a.rank[which], 0), a.R) : a.R;
}

// ---------------------------------------------------------------------------------------------- T = X A^T
// A workgroup: one adapter's rows of a window, J * 16 rows of A, one of the ks ranges of K, cut again over its four waves.
// NR: row tiles of 16 that are multiplied together.
template <bool F32, int J, int NR>
__device__ __forceinline__ void shrink(const LoraArgs& a, const Tile& t, int64_t m0, int j0, int row0, int kb, int ke, uint32_t turn, v4f* part, float* T)
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
        live[n] = row0 + 16 * n + l16 < t.count;
        row[n] = m0 + __shfl(t.row, (row0 + 16 * n + l16) & 63);
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
    // Rows of X and A often lie a multiple of 4 KiB apart, so that what an instruction asks for is one channel of the cache's.
    // Each wave starts somewhere else in its range, or the whole machine would go from channel to channel together.
    constexpr int U = J * NR >= 8 ? 2 : 4;
    const int spans = (ke - kb) / (32 * U);
    int at = spans ? (int)(turn % (uint32_t)spans) : 0;
    for (int i = 0; i < spans; ++i) {
        span(kb + 32 * U * at, std::integral_constant<int, U>{});
        at = at + 1 < spans ? at + 1 : 0;
    }
    for (int k = kb + 32 * U * spans; k < ke; k += 32) span(k, std::integral_constant<int, 1>{});
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
    const uint32_t turn = (uint32_t)(m0 / WINDOW) * 3 + (uint32_t)(g * 5 + slot * 7 + wave);
    const int j0 = g * J * 16;
    for_tiles(a, m0, slot, slots, false, [&](const Tile& t) {
        // (nothing to do where every one of these rows of A is past the adapter's rank)
        const int rank = rank_of(a, t.adapter);
        bool any = false;
        for (int j = j0; j < min(j0 + J * 16, a.n_parts * a.R); j += 8) any |= j % a.R < rank;
        if (!any) return;
        // few rows an adapter: one row tile at a time, in few registers; else up to four together
        if constexpr (J == 1)
            for (int row0 = 0; row0 < t.count; row0 += 16) shrink<F32, J, 1>(a, t, m0, j0, row0, kb, ke, turn, (v4f*)smem, T);
        else if (t.count <= 16) shrink<F32, J, 1>(a, t, m0, j0, 0, kb, ke, turn, (v4f*)smem, T);
        else shrink<F32, J, 4>(a, t, m0, j0, 0, kb, ke, turn, (v4f*)smem, T);
    });
}

// ---------------------------------------------------------------------------------------------- Y
__device__ __forceinline__ float silu(float z) { return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }

// A workgroup: one adapter's rows of a window, `steps` times 64 columns a wave.  A wave's four matrix tiles take its 64
// columns in an order that leaves 16 (with the gated activation: 8 gate and the 8 up) columns of one row in a lane.
// S: steps of 32 ranks.
template <int S, bool PAIRED>
__global__ void __launch_bounds__(256, OC) lora_expand_kernel(LoraArgs a, int slots, int groups, int steps, int ks, int row_tiles)
{
    extern __shared__ __align__(16) char smem[];             // T: [part][row tile][step][hi, lo][64 lanes] 16 bytes
    v4i* const ts = reinterpret_cast<v4i*>(smem);
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    // workgroups eight apart run on one die: it takes every eighth group of columns and, for one group after the other, all
    // windows, so that the columns of B stay in its cache
    const uint32_t units = (uint32_t)((a.M + WINDOW - 1) / WINDOW) * slots, turn = blockIdx.x >> 3;
    const uint32_t g = (turn / units << 3) + (blockIdx.x & 7), unit = turn % units;
    if (g >= (uint32_t)groups) return;
    const int slot = unit % slots;
    const int64_t m0 = (int64_t)(unit / slots) * WINDOW;
    const int PR = a.n_parts * a.R;
    const int64_t n_first = ((int64_t)g * steps * waves + wave) * 64;
    // the column (of the wave's 64) that row l16 of matrix tile t stands for
    auto column = [&](int t) {
        const int p = l16 >> 2, i = l16 & 3;
        return PAIRED ? 32 * (p >> 1) + 8 * (p & 1) + 4 * (t & 1) + i + 16 * (t >> 1) : 16 * p + 4 * t + i;
    };

    for_tiles(a, m0, slot, slots, true, [&](const Tile& t) {
        const int tiles = (t.count + 15) / 16;
        // operands: column(i)'s ranks 32 s + 8 q ..+ 7
        v4i bv[4][S];
        auto load_b = [&](int64_t n0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t n = n0 + column(i);
                const uint16_t* src = a.B + (int64_t)t.adapter * a.b_stride + n * a.R + 8 * q;
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    bv[i][s] = (v4i){0, 0, 0, 0};
                    if (t.adapter >= 0 && 32 * s + 8 * q < a.R && n < a.N) bv[i][s] = *reinterpret_cast<const v4i*>(src + 32 * s);
                }
            }
        };
        // this lane's columns: 16 in a row, or 8 gate columns and the up columns 16 further; where they lie in the rows of row
        // tile n, from the window's first row on (strides are below 2^25: 32 bits)
        const int c0 = PAIRED ? 32 * (q >> 1) + 8 * (q & 1) : 16 * q, c1 = c0 + (PAIRED ? 16 : 8);
        uint32_t from[4], to[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const uint32_t row = __shfl(t.row, 16 * n + l16);
            from[n] = (row * (uint32_t)a.ldb + c0) * 2;
            to[n] = (row * (uint32_t)a.ldy + (PAIRED ? 8 * q : c0)) * 2;
        }
        const char* const base = (const char*)(a.base + m0 * a.ldb);
        char* const Y = (char*)(a.Y + m0 * a.ldy);
        v4i b0, b1;
        auto load_base = [&](int64_t n0, uint32_t off, int n) {
            b0 = b1 = (v4i){0, 0, 0, 0};
            if (16 * n + l16 < t.count && a.base) {
                const char* src = base + n0 * 2 + off;
                if (n0 + c0 < a.N) b0 = *reinterpret_cast<const v4i*>(src);
                if (n0 + c1 < a.N) b1 = *reinterpret_cast<const v4i*>(src + (c1 - c0) * 2);
            }
        };
        // everything that the first columns need is asked for at once
        load_b(n_first);
        load_base(n_first, from[0], 0);
        const int rank = rank_of(a, t.adapter);
        const float scale = t.adapter < 0 || !a.scale ? 1.0f : a.scale[t.adapter];
        if (rank == 0 && a.act == ACT_NONE && a.base == a.Y) return;         // rows that stay where they are
        __syncthreads();                                     // (the tile before is done with local memory)
        for (int e = threadIdx.x; e < a.n_parts * tiles * S * 64; e += blockDim.x) {
            const int s = e / 64 % S, n = e / 64 / S % tiles, p = e / 64 / S / tiles;
            const int pos = 16 * n + l16, r = 32 * s + 8 * q;
            const int64_t row = m0 + __shfl(t.row, pos);
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = 0.0f;
            if (pos < t.count && r < rank) {
                const float* src = a.T + row * PR + p * a.R + r;
                int c = 0;
                for (; c + 4 <= ks; c += 4) {
                    float4 x[4], y[4];
#pragma unroll
                    for (int g = 0; g < 4; ++g, src += a.M * PR) {
                        x[g] = *reinterpret_cast<const float4*>(src);
                        y[g] = *reinterpret_cast<const float4*>(src + 4);
                    }
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        f[0] += x[g].x; f[1] += x[g].y; f[2] += x[g].z; f[3] += x[g].w;
                        f[4] += y[g].x; f[5] += y[g].y; f[6] += y[g].z; f[7] += y[g].w;
                    }
                }
                for (; c < ks; ++c, src += a.M * PR) {
                    const float4 x = *reinterpret_cast<const float4*>(src), y = *reinterpret_cast<const float4*>(src + 4);
                    f[0] += x.x; f[1] += x.y; f[2] += x.z; f[3] += x.w;
                    f[4] += y.x; f[5] += y.y; f[6] += y.z; f[7] += y.w;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = r + i < rank ? f[i] * scale : 0.0f;
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
            if (step) {
                load_b(n0);
                load_base(n0, from[0], 0);
            }
            // the parts of the wave's columns: as a rule the same for every column of a matrix tile
            int part[2], first[2];
            bool plain = true;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                part[h] = part_of(a, (int)((n0 + column(2 * h)) >> 4));
                first[h] = __builtin_amdgcn_readfirstlane(part[h]);
                plain &= __builtin_amdgcn_ballot_w64(part[h] == first[h] || n0 + column(2 * h) >= a.N) == ~(uint64_t)0;
            }
            if (rank < a.R)                                  // what lies past the adapter's rank may be anything
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int s = 0; s < S; ++s)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int left = rank - 32 * s - 8 * q;
                            bv[i][s][e] &= (int)((left > 2 * e ? 0xffffu : 0u) | (left > 2 * e + 1 ? 0xffff0000u : 0u));
                        }
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                if (n >= tiles) break;
                // the sums start from base
                v4f acc[4];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t x = (uint32_t)b0[e / 2], y = (uint32_t)b1[e / 2];
                    acc[e / 4][e % 4] = __uint_as_float(e & 1 ? x & 0xffff0000u : x << 16);
                    acc[2 + e / 4][e % 4] = __uint_as_float(e & 1 ? y & 0xffff0000u : y << 16);
                }
                if (n + 1 < 4 && n + 1 < tiles) load_base(n0, from[(n + 1) & 3], n + 1);
                if (rank > 0 && plain) {
                    v4i tv[2][S][2];
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int s = 0; s < S; ++s) {
                            const v4i* src = ts + ((first[h] * row_tiles + n) * S + s) * 128 + lane;
                            tv[h][s][0] = src[0];
                            tv[h][s][1] = src[64];
                        }
#pragma unroll
                    for (int s = 0; s < S; ++s)
#pragma unroll
                        for (int l = 0; l < 2; ++l)
#pragma unroll
                            for (int i = 0; i < 4; ++i) acc[i] = mfma(bv[i][s], tv[i >> 1][s][l], acc[i]);
                } else if (rank > 0) {
                    for (int p = 0; p < a.n_parts; ++p)
#pragma unroll
                        for (int s = 0; s < S; ++s) {
                            const v4i* src = ts + ((p * row_tiles + n) * S + s) * 128 + lane;
                            const v4i hi = src[0], lo = src[64];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const v4i b = part[i >> 1] == p ? bv[i][s] : (v4i){0, 0, 0, 0};
                                acc[i] = mfma(b, lo, mfma(b, hi, acc[i]));
                            }
                        }
                }
                if (16 * n + l16 >= t.count) continue;
                char* const dst = Y + (PAIRED ? n0 : 2 * n0) + to[n];
                v4i y0, y1;
                if constexpr (PAIRED) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = e >> 1, c = (2 * e) & 3;
                        y0[e] = (int)pack_bf16(silu(acc[i][c]) * acc[2 + i][c], silu(acc[i][c + 1]) * acc[2 + i][c + 1]);
                    }
                    if (n0 + c0 < a.N) *reinterpret_cast<v4i*>(dst) = y0;
                } else {
                    if (a.act == ACT_SILU)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int c = 0; c < 4; ++c) acc[i][c] = silu(acc[i][c]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = e >> 1, c = (2 * e) & 3;
                        y0[e] = (int)pack_bf16(acc[i][c], acc[i][c + 1]);
                        y1[e] = (int)pack_bf16(acc[2 + i][c], acc[2 + i][c + 1]);
                    }
                    if (n0 + c0 < a.N) *reinterpret_cast<v4i*>(dst) = y0;
                    if (n0 + c1 < a.N) *reinterpret_cast<v4i*>(dst + 16) = y1;
                }
            }
        }
    });
}

struct Plan {
    int64_t windows;
    int J, groups, ks, slots;            // shrink: 16-row tiles of A a workgroup, how many such, ranges of K; workgroups that share a window's adapters
    int steps, columns, eslots;          // expand: steps of 256 columns a workgroup, how many such; as above
};

// Slots: as many as a window has rows while that is a small grid (no search, see for_tiles), else enough to fill the machine.
int slots_for(int64_t M, int64_t windows, int64_t others, int64_t adapters)
{
    const int64_t rows = std::min<int64_t>(M, WINDOW);
    if (windows <= 4) return (int)rows;
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(rows - 1, adapters), 1024 / (windows * others)));
}

Plan make_plan(int n_parts, int R, int n_adapters, int64_t M, int64_t K, int64_t N)
{
    Plan p;
    p.windows = (M + WINDOW - 1) / WINDOW;
    const int tiles = (n_parts * R + 15) / 16;
    p.J = p.windows > 4 ? JJ : 1;
    p.groups = (tiles + p.J - 1) / p.J;
    // K cut until there are eight workgroups on every CU, which wait for memory; one where there are many rows: every part of T
    // is written and read again.  A wave's share is 64 numbers or more.
    const int64_t busy = std::min<int64_t>(M, p.windows - 1 + n_adapters) * p.groups, want = p.windows > 4 ? LW : 2048;
    p.ks = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want / std::max<int64_t>(busy, 1), 16), K / 256));
    p.slots = slots_for(M, p.windows, p.groups * p.ks, n_adapters);
    const int64_t blocks = (N + 255) / 256;
    p.steps = (int)std::max<int64_t>(1, std::min<int64_t>(blocks, blocks * p.windows / ST));
    p.columns = (int)((blocks + p.steps - 1) / p.steps);
    p.eslots = slots_for(M, p.windows, p.columns, (int64_t)n_adapters + 1);
    return p;
}

template <bool F32, int J>
int launch_shrink(const LoraArgs& a, const Plan& p, hipStream_t stream)
{
    const int row_tiles = J == 1 || a.M <= 16 ? 1 : 4, lds = J * row_tiles * 4096;
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
    const int64_t blocks = p.windows * p.eslots * ((p.columns + 7) / 8 * 8);
    hipLaunchKernelGGL((lora_expand_kernel<S, PAIRED>), dim3((unsigned)blocks), dim3(256), lds, stream, a, p.eslots, p.columns, p.steps, p.ks, row_tiles);
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
    if (a.x_f32) rc = p.J == 1 ? launch_shrink<true, 1>(a, p, stream) : launch_shrink<true, JJ>(a, p, stream);
    else rc = p.J == 1 ? launch_shrink<false, 1>(a, p, stream) : launch_shrink<false, JJ>(a, p, stream);
    if (rc) return rc;
    const int S = (a.R + 31) / 32;
    if (a.act == ACT_SILU_MUL)
        return S == 1 ? launch_expand<1, true>(a, p, stream) : S == 2 ? launch_expand<2, true>(a, p, stream) : launch_expand<4, true>(a, p, stream);
    return S == 1 ? launch_expand<1, false>(a, p, stream) : S == 2 ? launch_expand<2, false>(a, p, stream) : launch_expand<4, false>(a, p, stream);
}

}  // namespace w2
