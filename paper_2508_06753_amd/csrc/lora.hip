// Low-rank adapters of many requests beside a shared projection:
//   T[m,j] = sum_k X[m,k] A[a_m, j, k]      Y[m,n] = act(base[m,n] + scale * sum_r T[m, part(n) R + r] B[a_m, n, r]).
//
// Rows are taken in windows of 64, one a lane, and a window is sorted by adapter with ballots: the rows of one adapter (a
// tile, 1 to 64 of them) meet its factors together, whatever order the rows come in, and nothing has to be planned before
// the call.  An adapter's factors are read once a window.  Two launches: lora_shrink_kernel writes T, fp32, in `ks` parts
// of K; lora_expand_kernel adds them in order and finishes Y.  Matrix instructions 16x16x32 with the factors' rows on one
// side and the tile's rows on the other; numbers in 32 bits (T, and X if it is fp32) go in as two bf16 parts, 16 bits of
// mantissa, in two instructions: the outputs' rounding to 8 hides it.
//
// Bound (kernels alone, in a trace): few rows, by two launches and the trips to memory in each, one behind the other (whose
// adapter, its factors; T, the stores): one row, K = 4096, 16 ranks, N = 6144: 4.0 + 5.5 us; 61 rows of 48 adapters, 37 MB: 12.3 +
// 10.9 us; 37 fp32 rows, K = 14336: 8.3 + 6.2, the first in 216 workgroups of four trips a wave.  Many rows, by base and Y: 4000
// rows, K = 4096, 64 ranks, 28672 gated columns, 344 MB: 26 + 109 us, 3.2 TB/s in the second launch (a large copy: 4.75); there two
// waves a SIMD (four row tiles of base and the factors in registers) load, multiply and store in turns.  Base by way of local
// memory: 121 us; the next columns' base asked for before this one's products: no faster with all stores behind it, slower among
// them.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "block_ops.h"
#include "w2_small_common.h"

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

// 16 bytes a lane from wherever the lane says to local memory, lane after lane from dst on
__device__ __forceinline__ void load_lds16(const void* src, char* dst)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}

constexpr float MOST_BF16 = 0x1.fep127f;

// Eight floats as two bf16 parts whose sum has 16 bits of them.  FAR: numbers that are infinite, or round to infinity in bf16, are
// among them: the first part stays finite, so that both have the number's sign, and the second is cut, so that the sum of a finite
// number's is finite.
template <bool FAR>
__device__ __forceinline__ void split_bf16(const float (&f)[8], v4i& hi, v4i& lo)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a = f[2 * e], b = f[2 * e + 1];
        if (FAR) {
            a = __builtin_amdgcn_fmed3f(a, -MOST_BF16, MOST_BF16);
            b = __builtin_amdgcn_fmed3f(b, -MOST_BF16, MOST_BF16);
        }
        const uint32_t h = pack_bf16(a, b);
        a = f[2 * e] - __uint_as_float(h << 16);
        b = f[2 * e + 1] - __uint_as_float(h & 0xffff0000u);
        if (FAR) {
            if (fabsf(f[2 * e]) > MOST_BF16) a = __uint_as_float(__float_as_uint(a) & 0xffff0000u);
            if (fabsf(f[2 * e + 1]) > MOST_BF16) b = __uint_as_float(__float_as_uint(b) & 0xffff0000u);
        }
        hi[e] = (int)h;
        lo[e] = (int)pack_bf16(a, b);
    }
}

__device__ __forceinline__ int part_of(const LoraArgs& a, int block)
{
    if (a.gated) return block & 1;
    return (block >= a.end16[0]) + (block >= a.end16[1]) + (block >= a.end16[2]);
}

// of a row; top: the largest number that was split (not FAR)
template <bool FAR>
__device__ __forceinline__ void split_row(const v4i& x0, const v4i& x1, v4i& hi, v4i& lo, float& top)
{
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __int_as_float(e < 4 ? x0[e & 3] : x1[e & 3]);
    if (!FAR)
#pragma unroll
        for (int e = 0; e < 8; e += 2) top = fmaxf(top, fmaxf(fabsf(f[e]), fabsf(f[e + 1])));
    split_bf16<FAR>(f, hi, lo);
}
__device__ __forceinline__ bool is_far(float top) { return __builtin_expect(__builtin_amdgcn_ballot_w64(top > MOST_BF16) != 0, 0); }

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

// ---------------------------------------------------------------------------------------------- T = X A^T, few rows
// A workgroup: one adapter's rows of a window, 16 rows of A, one of the ks ranges of K, cut again over its four waves.
template <bool F32>
__global__ void __launch_bounds__(256) lora_shrink_kernel(LoraArgs a, int slots, int groups, int ks)
{
    __shared__ v4f part[4 * 64];
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // (slot, group of A's rows, range of K) of a window side by side
    uint32_t id = blockIdx.x;
    const int kr = id % ks;
    id /= ks;
    const int j0 = id % groups * 16;
    id /= groups;
    const int slot = id % slots;
    const int64_t m0 = (int64_t)(id / slots) * WINDOW;
    const int64_t steps = a.K / 32;
    const int kb = (int)(steps * (kr * 4 + wave) / (ks * 4)) * 32, ke = (int)(steps * (kr * 4 + wave + 1) / (ks * 4)) * 32;
    const int PR = a.n_parts * a.R;
    float* const T = a.T + (int64_t)kr * a.M * PR;
    for_tiles(a, m0, slot, slots, false, [&](const Tile& t) {
        // (nothing to do where every one of these rows of A is past the adapter's rank)
        const int rank = rank_of(a, t.adapter);
        if (j0 % a.R >= rank && (j0 + 8 >= PR || (j0 + 8) % a.R >= rank)) return;
        const uint16_t* const ap = a.A + t.adapter * a.a_stride + (int64_t)min(j0 + l16, PR - 1) * a.K + 8 * q;
        for (int row0 = 0; row0 < t.count; row0 += 16) {
            const bool live = row0 + l16 < t.count;
            const int64_t row = m0 + __shfl(t.row, (row0 + l16) & 63);
            const char* const xp = (const char*)a.X + (row * a.ldx + 8 * q) * (F32 ? 4 : 2);
            v4f acc;
            float top = 0.0f;
            // U steps of 32: all loads first, then the products
            auto span = [&](int k, auto uc, auto far) {
                constexpr int U = decltype(uc)::value;
                v4i av[U], xv[U * (F32 ? 2 : 1)];
#pragma unroll
                for (int u = 0; u < U; ++u) av[u] = *reinterpret_cast<const v4i*>(ap + k + 32 * u);
#pragma unroll
                for (int u = 0; u < U * (F32 ? 2 : 1); ++u) xv[u] = (v4i){0, 0, 0, 0};
                if (live)                                    // (rows that are not there cost no memory traffic)
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        if constexpr (F32) {
                            xv[2 * u] = *reinterpret_cast<const v4i*>(xp + (int64_t)(k + 32 * u) * 4);
                            xv[2 * u + 1] = *reinterpret_cast<const v4i*>(xp + (int64_t)(k + 32 * u) * 4 + 16);
                        } else {
                            xv[u] = *reinterpret_cast<const v4i*>(xp + (int64_t)(k + 32 * u) * 2);
                        }
                    }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if constexpr (F32) {
                        v4i hi, lo;
                        split_row<decltype(far)::value>(xv[2 * u], xv[2 * u + 1], hi, lo, top);
                        acc = mfma(av[u], lo, mfma(av[u], hi, acc));
                    } else {
                        acc = mfma(av[u], xv[u], acc);
                    }
                }
            };
            auto sum = [&](auto far) {
                acc = (v4f){0.f, 0.f, 0.f, 0.f};
                int k = kb;
                for (; k + 128 <= ke; k += 128) span(k, std::integral_constant<int, 4>{}, far);
                for (; k + 64 <= ke; k += 64) span(k, std::integral_constant<int, 2>{}, far);
                if (k < ke) span(k, std::integral_constant<int, 1>{}, far);
            };
            sum(std::false_type{});
            if (F32 && is_far(top)) sum(std::true_type{});
            // the four waves' sums, in order; lane: row l16 of the row tile, T's columns j0 + 4 q ..+ 3
            __syncthreads();
            part[wave * 64 + lane] = acc;
            __syncthreads();
            if (wave == 0 && live && j0 + 4 * q < PR)
                *reinterpret_cast<v4f*>(T + row * PR + j0 + 4 * q) = part[lane] + part[64 + lane] + part[128 + lane] + part[192 + lane];
        }
    });
}

// ---------------------------------------------------------------------------------------------- T = X A^T, many rows
// A workgroup: one adapter's rows of a window (up to 64), 16 J rows of A, one of the ks ranges of K, in stages of 64 k through a
// ring in local memory.  A wave multiplies 16 rows.  Whole 128-byte pieces of rows an instruction: rows of X and A often lie
// a multiple of 8 KiB apart, in one set of the vector cache, and operands that are loaded from there directly, half a line
// of 16 rows each, evict one another (4000 rows, K = 4096, 128 ranks: 90 us in one range of K against 30).
// J = 4 where there are more than 32 rows of A: X is read half as often (2948 rows of 4096, fp32, 192 ranks: 64 -> 49 us; 3747,
// bf16, 48 ranks: 26 -> 16).
template <bool F32> constexpr int STAGES = F32 ? 3 : 4;       // (two workgroups on a CU, or more)
template <bool F32, int J> constexpr int shrink_stage() { return 64 * (F32 ? 256 : 128) + 16 * J * 128; }

template <bool F32, int J>
__global__ void __launch_bounds__(256) lora_shrink_tile_kernel(LoraArgs a, int slots, int groups, int ks)
{
    constexpr int XB = F32 ? 256 : 128, XL = F32 ? 4 : 2, AL = J / 2;        // bytes of a row's stage; loads of X and of A a wave and stage
    constexpr int STAGE = shrink_stage<F32, J>(), A_AT = 64 * XB, N = STAGES<F32>;
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t id = blockIdx.x;
    const int kr = id % ks;
    id /= ks;
    const int j0 = id % groups * 16 * J;
    id /= groups;
    // (the windows' first adapters one after the other: as a rule there are no others, and every die has its share of work)
    const uint32_t windows = (uint32_t)((a.M + WINDOW - 1) / WINDOW);
    const int slot = id / windows;
    const int64_t m0 = (int64_t)(id % windows) * WINDOW;
    const int kb = (int)(a.K / 64 * kr / ks), n_st = (int)(a.K / 64 * (kr + 1) / ks) - kb;
    const int PR = a.n_parts * a.R;
    float* const T = a.T + (int64_t)kr * a.M * PR;
    // 16-byte pieces are stored XORed: 16 rows at one piece lie in 16 different places of the 256 bytes delivered at once
    auto swz = [](int row) { return F32 ? row & 15 : (row >> 1) & 7; };
    auto swz_a = [](int row) { return (row >> 1) & 7; };

    for_tiles(a, m0, slot, slots, false, [&](const Tile& t) {
        const int rank = rank_of(a, t.adapter);
        bool any = false;
        for (int j = j0; j < min(j0 + 16 * J, PR); j += 8) any |= j % a.R < rank;
        if (!any) return;
        const char* xsrc[XL];
#pragma unroll
        for (int j = 0; j < XL; ++j) {
            const int at = (wave * XL + j) * 64 + lane, row = at / (XB / 16), piece = at % (XB / 16) ^ swz(row);
            const int64_t from = m0 + __shfl(t.row, row < t.count ? row : 0);        // (rows that are not there: the first one again)
            xsrc[j] = (const char*)a.X + from * a.ldx * (F32 ? 4 : 2) + (int64_t)kb * XB + piece * 16;
        }
        const char* asrc[AL];
#pragma unroll
        for (int j = 0; j < AL; ++j) {
            const int row = (wave * AL + j) * 8 + lane / 8;
            asrc[j] = (const char*)(a.A + t.adapter * a.a_stride + (int64_t)min(j0 + row, PR - 1) * a.K) + (int64_t)kb * 128 + (lane % 8 ^ swz_a(row)) * 16;
        }
        auto fetch = [&](int st) {
            char* const dst = smem + st % N * STAGE;
#pragma unroll
            for (int j = 0; j < XL; ++j) load_lds16(xsrc[j] + (int64_t)st * XB, dst + (wave * XL + j) * 1024);
#pragma unroll
            for (int j = 0; j < AL; ++j) load_lds16(asrc[j] + (int64_t)st * 128, dst + A_AT + (wave * AL + j) * 1024);
        };
        __syncthreads();                                     // (the tile before is done with local memory)
#pragma unroll
        for (int st = 0; st < N - 1; ++st)
            if (st < n_st) fetch(st);
        v4f acc[J];
#pragma unroll
        for (int j = 0; j < J; ++j) acc[j] = (v4f){0.f, 0.f, 0.f, 0.f};
        const int xrow = wave * 16 + l16;
        float top = 0.0f;
        for (int st = 0; st < n_st; ++st) {
            // this stage is there; up to N - 2 behind it are under way (at the end: none)
            if (st + N - 2 < n_st) wait_loads<(N - 2) * (XL + AL)>();
            else wait_loads<0>();
            bare_barrier();                                  // every wave's part of it, and no wave reads the stage before any more
            if (st + N - 1 < n_st) fetch(st + N - 1);
            const char* const xb = smem + st % N * STAGE + xrow * XB;
            const char* const ab = smem + st % N * STAGE + A_AT;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int p = 4 * s + q;
                v4i av[J];
#pragma unroll
                for (int j = 0; j < J; ++j) av[j] = *reinterpret_cast<const v4i*>(ab + (16 * j + l16) * 128 + ((p ^ swz_a(16 * j + l16)) << 4));
                if constexpr (F32) {
                    const v4i x0 = *reinterpret_cast<const v4i*>(xb + ((2 * p ^ swz(xrow)) << 4));
                    const v4i x1 = *reinterpret_cast<const v4i*>(xb + (((2 * p + 1) ^ swz(xrow)) << 4));
                    v4i hi, lo;
                    split_row<false>(x0, x1, hi, lo, top);
#pragma unroll
                    for (int j = 0; j < J; ++j) acc[j] = mfma(av[j], lo, mfma(av[j], hi, acc[j]));
                } else {
                    const v4i xv = *reinterpret_cast<const v4i*>(xb + ((p ^ swz(xrow)) << 4));
#pragma unroll
                    for (int j = 0; j < J; ++j) acc[j] = mfma(av[j], xv, acc[j]);
                }
            }
        }
        if (F32 && is_far(top)) {                            // once more, straight from memory
            const float* const x = (const float*)a.X + (m0 + __shfl(t.row, xrow < t.count ? xrow : 0)) * a.ldx + 8 * q;
            const uint16_t* const A = a.A + t.adapter * a.a_stride + 8 * q;
#pragma unroll
            for (int j = 0; j < J; ++j) acc[j] = (v4f){0.f, 0.f, 0.f, 0.f};
            for (int k = kb * 64; k < (kb + n_st) * 64; k += 32) {
                v4i hi, lo;
                split_row<true>(*reinterpret_cast<const v4i*>(x + k), *reinterpret_cast<const v4i*>(x + k + 4), hi, lo, top);
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const v4i av = *reinterpret_cast<const v4i*>(A + (int64_t)min(j0 + 16 * j + l16, PR - 1) * a.K + k);
                    acc[j] = mfma(av, lo, mfma(av, hi, acc[j]));
                }
            }
        }
        if (xrow < t.count) {
            const int64_t row = m0 + __shfl(t.row, xrow);
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (j0 + 16 * j + 4 * q < PR) *reinterpret_cast<v4f*>(T + row * PR + j0 + 16 * j + 4 * q) = acc[j];
        }
    });
}

// ---------------------------------------------------------------------------------------------- Y
__device__ __forceinline__ float silu(float z) { return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }

// A workgroup: one adapter's rows of a window, `steps` times 64 columns a wave.  A wave's four matrix tiles take its 64
// columns in an order that leaves 16 (with the gated activation: 8 gate and the 8 up) columns of one row in a lane.
// S: steps of 32 ranks.
// NT: row tiles whose rows of base are asked for together: all four of a window, or one, in half the registers, where
// adapters have few rows.
template <int S, bool PAIRED, int NT>
__global__ void __launch_bounds__(256, NT == 1 ? (S == 1 ? 4 : S == 2 ? 3 : 2) : S == 1 ? 3 : 2) lora_expand_kernel(LoraArgs a, int slots, int groups, int steps, int ks, int row_tiles)
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
    const uint32_t windows = (uint32_t)((a.M + WINDOW - 1) / WINDOW);        // (their first adapters one after the other)
    const int slot = unit / windows;
    const int64_t m0 = (int64_t)(unit % windows) * WINDOW;
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
        auto row_offset = [&](int n, int64_t ld) { return __shfl(t.row, (16 * n + l16) & 63) * (uint32_t)ld * 2; };
        uint32_t from[NT], to[NT];
        if constexpr (NT == 4)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                from[n] = row_offset(n, a.ldb) + 2 * c0;
                to[n] = row_offset(n, a.ldy) + 2 * (PAIRED ? 8 * q : c0);
            }
        const char* const base = (const char*)(a.base + m0 * a.ldb);
        char* const Y = (char*)(a.Y + m0 * a.ldy);
        v4i b0[NT], b1[NT];
        auto load_base = [&](int64_t n0, int first) {
            const char* const src = base + n0 * 2;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const uint32_t off = NT == 4 ? from[n] : row_offset(first + n, a.ldb) + 2 * c0;
                b0[n] = b1[n] = (v4i){0, 0, 0, 0};
                if (16 * (first + n) + l16 < t.count && a.base) {
                    if (n0 + c0 < a.N) b0[n] = *reinterpret_cast<const v4i*>(src + off);
                    if (n0 + c1 < a.N) b1[n] = *reinterpret_cast<const v4i*>(src + off + (c1 - c0) * 2);
                }
            }
        };
        // everything that the first columns need is asked for at once
        load_b(n_first);
        load_base(n_first, 0);
        const int rank = rank_of(a, t.adapter);
        const float scale = t.adapter < 0 || !a.scale ? 1.0f : a.scale[t.adapter];
        if (rank == 0 && a.act == ACT_NONE && a.base == a.Y) return;         // rows that stay where they are
        __syncthreads();                                     // (the tile before is done with local memory)
        // T of the tile's rows, scaled, as operands.  Items of 64 lanes: (part, row tile, step of ranks).
        const int items = a.n_parts * tiles * S;
        auto place = [&](int e, int& p, int& n, int& s) { s = e % S; n = e / S % tiles; p = e / S / tiles; };
        auto source = [&](int e) {                           // nullptr: zeros
            int p, n, s;
            place(e, p, n, s);
            const int pos = 16 * n + l16, r = 32 * s + 8 * q;
            const int64_t row = m0 + __shfl(t.row, pos & 63);
            return e < items && pos < t.count && r < rank ? a.T + row * PR + p * a.R + r : nullptr;
        };
        auto put = [&](int e, float (&f)[8]) {
            int p, n, s;
            place(e, p, n, s);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = 32 * s + 8 * q + i < rank ? f[i] * scale : 0.0f;
            v4i hi, lo;
            float top = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(f[i]));
            if (is_far(top)) split_bf16<true>(f, hi, lo);
            else split_bf16<false>(f, hi, lo);
            v4i* dst = ts + ((p * row_tiles + n) * S + s) * 128 + lane;
            dst[0] = hi;
            dst[64] = lo;
        };
        if (NT == 4 && ks == 1) {                            // four items' loads together
            for (int e0 = wave; e0 < items; e0 += 4 * waves) {
                float f[4][8];
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float* src = source(e0 + g * waves);
                    const v4f x = src ? *reinterpret_cast<const v4f*>(src) : (v4f){0.f, 0.f, 0.f, 0.f};
                    const v4f y = src ? *reinterpret_cast<const v4f*>(src + 4) : (v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[g][i] = i < 4 ? x[i & 3] : y[i & 3];
                }
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    if (e0 + g * waves < items) put(e0 + g * waves, f[g]);
            }
        } else {                                             // several parts' loads together
            constexpr int PB = NT == 1 ? 4 : 8;
            for (int e = wave; e < items; e += waves) {
                const float* src = source(e);
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = 0.0f;
                if (src)
                    for (int c = 0; c < ks; c += PB, src += PB * a.M * PR) {
                        v4f x[PB], y[PB];
#pragma unroll
                        for (int g = 0; g < PB; ++g) {
                            x[g] = y[g] = (v4f){0.f, 0.f, 0.f, 0.f};
                            if (c + g < ks) {
                                x[g] = *reinterpret_cast<const v4f*>(src + g * a.M * PR);
                                y[g] = *reinterpret_cast<const v4f*>(src + g * a.M * PR + 4);
                            }
                        }
#pragma unroll
                        for (int g = 0; g < PB; ++g)
#pragma unroll
                            for (int i = 0; i < 8; ++i) f[i] += i < 4 ? x[g][i & 3] : y[g][i & 3];
                    }
                put(e, f);
            }
        }
        __syncthreads();
        for (int step = 0; step < steps; ++step) {
            const int64_t n0 = n_first + (int64_t)step * waves * 64;
            if (n0 >= a.N) break;
            if (step) {
                load_b(n0);
                load_base(n0, 0);
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
            for (int group = 0; group < tiles; group += NT)
#pragma unroll
            for (int k = 0; k < NT; ++k) {
                const int n = group + k;
                if (n >= tiles) break;
                if (NT == 1 && n) load_base(n0, n);
                // the sums start from base
                v4f acc[4];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t x = (uint32_t)b0[k][e / 2], y = (uint32_t)b1[k][e / 2];
                    acc[e / 4][e % 4] = __uint_as_float(e & 1 ? x & 0xffff0000u : x << 16);
                    acc[2 + e / 4][e % 4] = __uint_as_float(e & 1 ? y & 0xffff0000u : y << 16);
                }
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
                    // (every part's sums for every column, and a lane keeps its columns' own: zeros in place of B would meet an infinite T)
                    const int own[2] = {part_of(a, (int)((n0 + c0) >> 4)), part_of(a, (int)((n0 + c1) >> 4))};
                    for (int p = 0; p < a.n_parts; ++p)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            v4f sum = acc[i];
#pragma unroll
                            for (int s = 0; s < S; ++s) {
                                const v4i* src = ts + ((p * row_tiles + n) * S + s) * 128 + lane;
                                sum = mfma(bv[i][s], src[64], mfma(bv[i][s], src[0], sum));
                            }
                            acc[i] = own[i >> 1] == p ? sum : acc[i];
                        }
                }
                char* const dst = Y + (PAIRED ? n0 : 2 * n0) + (NT == 4 ? to[k] : row_offset(n, a.ldy) + 2 * (PAIRED ? 8 * q : c0));
                const bool live = 16 * n + l16 < t.count;
                v4i y0, y1;
                if constexpr (PAIRED) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = e >> 1, c = (2 * e) & 3;
                        y0[e] = (int)pack_bf16(silu(acc[i][c]) * acc[2 + i][c], silu(acc[i][c + 1]) * acc[2 + i][c + 1]);
                    }
                    if (live && n0 + c0 < a.N) *reinterpret_cast<v4i*>(dst) = y0;
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
                    if (live && n0 + c0 < a.N) *reinterpret_cast<v4i*>(dst) = y0;
                    if (live && n0 + c1 < a.N) *reinterpret_cast<v4i*>(dst + 16) = y1;
                }
            }
        }
    });
}

struct Plan {
    int64_t windows;
    int many, j, groups, ks, slots;      // shrink: the kernel for many rows; groups of A's rows, ranges of K; workgroups that share a window's adapters
    int steps, columns, eslots;          // expand: steps of 256 columns a workgroup, how many such; as above
};

// Slots: a window's workgroups for its adapters.  Few windows: one for each row where adapters are about as many (no search, see
// for_tiles), else one for each adapter; many: as fill the machine.
int slots_for(int64_t M, int64_t windows, int64_t others, int64_t adapters)
{
    const int64_t rows = std::min<int64_t>(M, WINDOW);
    if (windows <= 4) return (int)(2 * adapters >= rows ? rows : adapters);
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(rows - 1, adapters), 1024 / (windows * others)));
}

Plan make_plan(int n_parts, int R, int n_adapters, int64_t M, int64_t K, int64_t N)
{
    Plan p;
    p.windows = (M + WINDOW - 1) / WINDOW;
    p.many = p.windows > 4 || (M > 32 && M > 32 * (int64_t)n_adapters);
    p.j = !p.many ? 1 : n_parts * R > 32 ? 4 : 2;
    p.groups = (n_parts * R + 16 * p.j - 1) / (16 * p.j);
    // K cut until there are eight workgroups on every CU, which wait for memory, or of the larger ones for many rows one and a
    // half, or one where they take 64 rows of A.  At most eight parts, four of a wide T: every part is written, and read again
    // by every group of columns (us, both launches, one row, K = 4096, 64 ranks, 16 parts: 12.5, 8: 11.0; 9 rows of 5 adapters
    // of 128: 22 and 20; 574 rows, 128 ranks, gated 34816 columns, 5 parts: 89, 4: 83; 218 fp32 rows of 384 ranks, 8 parts: 38,
    // 4: 35).  That is of K = 4096 and 5120; 37 rows of nine adapters and K = 14336 come to 216 workgroups, and eight parts have
    // not been compared with more there.  A wave's share is 128 numbers or more, which are one trip to memory.
    const int64_t busy = std::min<int64_t>(M, p.windows - 1 + n_adapters) * p.groups, want = p.j == 4 ? 256 : p.many ? 384 : 2048;
    p.ks = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want / std::max<int64_t>(busy, 1), p.j == 4 ? 4 : 8), K / 512));
    p.slots = slots_for(M, p.windows, p.groups * p.ks, n_adapters);
    // Columns of a workgroup: it reads T once for all of them, but the workgroups of a die (every eighth group of columns; room
    // for so many at once) should fill whole rounds: the number of rounds times the steps of one, and what it does before its
    // first step, about half a step and the reading of T (bytes against those of a step, 49152 of base and Y: gated columns with
    // their activation; others have 65536, and are planned alike).  4000 rows, 28672 gated columns,
    // us with 1, 3, 5, 7, 13 steps: 152, 123, 117, 110, 152; 933 rows, 34816, with 1, 2, 3: 66, 63, 51.
    const int64_t blocks = (N + 255) / 256, most = p.many ? std::min<int64_t>(blocks, 16) : 1, room = 32 * (R <= 32 ? 3 : 2);
    const double start = 0.5 + (double)(n_parts * R * p.ks) * 256 / (49152 + 512 * R);
    double least = 1e30;
    for (int64_t s = 1; s <= most; ++s) {
        const int64_t columns = (blocks + s - 1) / s, slots = slots_for(M, p.windows, columns, (int64_t)n_adapters + 1);
        const double cost = (double)(((columns + 7) / 8 * p.windows * slots + room - 1) / room) * (s + start);
        if (cost < least) least = cost, p.steps = (int)s, p.columns = (int)columns, p.eslots = (int)slots;
    }
    return p;
}

template <bool F32>
int launch_shrink(const LoraArgs& a, const Plan& p, hipStream_t stream)
{
    const int lds = p.j == 4 ? STAGES<F32> * shrink_stage<F32, 4>() : p.j == 2 ? STAGES<F32> * shrink_stage<F32, 2>() : 0;
    const auto kern = p.j == 4 ? lora_shrink_tile_kernel<F32, 4> : p.j == 2 ? lora_shrink_tile_kernel<F32, 2> : lora_shrink_kernel<F32>;
    if (int rc = ensure_dynamic_lds((const void*)kern, lds, "w2_lora_add")) return rc;
    const int64_t blocks = p.windows * p.slots * p.groups * p.ks;
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(256), lds, stream, a, p.slots, p.groups, p.ks);
    return check_launch("w2_lora_add");
}

template <int S, bool PAIRED>
int launch_expand(const LoraArgs& a, const Plan& p, hipStream_t stream)
{
    const int row_tiles = (int)std::min<int64_t>(4, (a.M + 15) / 16), lds = a.n_parts * row_tiles * S * 2048;
    auto kern = a.M > 16 && p.many ? lora_expand_kernel<S, PAIRED, 4> : lora_expand_kernel<S, PAIRED, 1>;
    if (int rc = ensure_dynamic_lds((const void*)kern, lds, "w2_lora_add")) return rc;
    const int64_t blocks = p.windows * p.eslots * ((p.columns + 7) / 8 * 8);
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(256), lds, stream, a, p.eslots, p.columns, p.steps, p.ks, row_tiles);
    return check_launch("w2_lora_add");
}

}  // namespace

size_t lora_part_bytes(int n_parts, int R, int64_t M) { return (size_t)M * n_parts * R * sizeof(float); }

size_t lora_workspace_bytes(int n_parts, int R, int n_adapters, int64_t M, int64_t K, int64_t N)
{
    if (M == 0) return 0;
    return (make_plan(n_parts, R, n_adapters, M, K, N).ks * lora_part_bytes(n_parts, R, M) + 255) & ~(size_t)255;
}

int launch_lora(const LoraArgs& a, size_t room, hipStream_t stream)
{
    Plan p = make_plan(a.n_parts, a.R, a.n_adapters, a.M, a.K, a.N);
    // (as many parts of K as the workspace holds: fewer rows may want more room)
    p.ks = (int)std::min<size_t>(p.ks, room / lora_part_bytes(a.n_parts, a.R, a.M));
    if (const int rc = a.x_f32 ? launch_shrink<true>(a, p, stream) : launch_shrink<false>(a, p, stream)) return rc;
    const int S = (a.R + 31) / 32;
    if (a.act == ACT_SILU_MUL)
        return S == 1 ? launch_expand<1, true>(a, p, stream) : S == 2 ? launch_expand<2, true>(a, p, stream) : launch_expand<4, true>(a, p, stream);
    return S == 1 ? launch_expand<1, false>(a, p, stream) : S == 2 ? launch_expand<2, false>(a, p, stream) : launch_expand<4, false>(a, p, stream);
}

}  // namespace w2
