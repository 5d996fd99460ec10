// Rows through their 2-bit experts: gate and up projection, silu(gate) * up, down projection, sum over a row's experts.
//
// The matrix instruction is the one for eight-bit rows and four-bit columns (16 x 16 x 128, E4M3 x E2M1, a power of two for every 32 k of
// a row): a 2-bit weight -2, -1, 0, 1 IS a four-bit number (-1, -0.5, 0, 0.5 with the column's power of two at 2), seven
// instructions turn 16 of them out of a packed dword, and a row's numbers are the sum of two eight-bit ones: E4M3 has four
// significant bits and bf16 eight, so hi = round(x), lo = round(x - hi) is exact wherever lo's exponent reaches, which is down
// to 2^-14 of the largest of the 32 numbers that share a power of two (off by 2^-22 of it below).  h, which is computed in fp32, is rounded to
// such a pair, by 2^-9 of itself at most: half of what a bf16 h would lose, and no third product.  Against bf16 instructions
// that is a third of the vector work per weight, and the products of hi and of lo together take no longer than one bf16
// product (4300 TFLOP/s for eight bits by four, measured; half that for the pair).  Its sums are not quite those of 32 bits: of 8
// neighbouring products, bits 13 places below the largest one's exponent are cut off (measured), at most 7 * 2^-13 of the sum of magnitudes.
//
// Three ways through, by how many choices there are (moe_plan.h): up to 64 in two launches; few rows an expert, bound by the weights' way from
// memory; many, bound by products.  The last two begin with a launch that sorts the choices and converts x, and end with one that sums.
//
// Rows in memory ("xs", "hs"): for every 256 k [2 halves of 128 k][hi, lo][8 units][16 bytes], a unit being 16 k in the order in which
// the up-convert leaves the weights' nibbles, 0 8 1 9 2 10 3 11 4 12 5 13 6 14 7 15; exponents [4 g][2 halves] bytes beside
// them, g = the units g and g + 4 of a half, which is one lane group's 32 k of the instruction.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "block_ops.h"
#include "ffn_ops.h"
#include "moe_plan.h"
#include "w2_small_common.h"

namespace w2 {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

struct Tile {                           // rows of one expert: places first .. first + rows - 1 of the sorted order; rows = 0: none
    int expert, first, rows, unused;
};

// ---------------------------------------------------------------- rows in two eight-bit parts

// The exponent (biased) that 32 numbers share, from the largest one's exponent field: the largest lands in 2^7 .. 2^8.  lo's is 5 lower.
__device__ __forceinline__ int shared_exponent(int field) { return max(field - 7, 5); }

// Two numbers, scaled: low halves of hi and lo
__device__ __forceinline__ void split2(float a, float b, float f, uint32_t& hi, uint32_t& lo)
{
    a *= f;
    b *= f;
    // an infinity has no place in E4M3, and the conversion may take it for the largest number
    a = fabsf(a) < INFINITY ? a : NAN;
    b = fabsf(b) < INFINITY ? b : NAN;
    const int h = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    typedef float v2f __attribute__((ext_vector_type(2)));
    const v2f back = __builtin_amdgcn_cvt_pk_f32_fp8(h, false);
    const int l = __builtin_amdgcn_cvt_pk_fp8_f32((a - back[0]) * 32.0f, (b - back[1]) * 32.0f, 0, false);
    hi = (uint32_t)h & 0xffffu;
    lo = (uint32_t)l & 0xffffu;
}

// 2^(127 - e) for a biased exponent e of 5 .. 248
__device__ __forceinline__ float scale_down(int e) { return __int_as_float((254 - e) << 23); }

// 32 numbers that share an exponent, the b-th ones of a row x: numbers 16 g .. and 64 + 16 g .. of 128
__device__ __forceinline__ void split_block(const uint16_t* x, int b, char* row, char* exps)
{
    const int kt = b / 8, half = (b & 7) >> 2, g = b & 3;
    const uint16_t* const src = x + kt * 256 + half * 128 + g * 16;
    uint32_t d[2][8], top = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const uint4 p = *reinterpret_cast<const uint4*>(src + u * 64), q = *reinterpret_cast<const uint4*>(src + u * 64 + 8);
        const uint32_t w[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            d[u][j] = w[j];
            top = max(top, max(w[j] & 0x7fffu, w[j] >> 16 & 0x7fffu));
        }
    }
    const int e = shared_exponent((int)(top >> 7));
    const float f = scale_down(e);
    char* const dst = row + kt * 512 + half * 256 + g * 16;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        uint32_t hi[8], lo[8];
#pragma unroll
        for (int n = 0; n < 8; ++n) {                        // numbers n and n + 8 of the unit are neighbours
            const uint32_t lw = d[u][n / 2], hw = d[u][4 + n / 2];
            const float p = __uint_as_float(n & 1 ? lw & 0xffff0000u : lw << 16), q = __uint_as_float(n & 1 ? hw & 0xffff0000u : hw << 16);
            split2(p, q, f, hi[n], lo[n]);
        }
        *reinterpret_cast<uint4*>(dst + u * 64) = make_uint4(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16, hi[4] | hi[5] << 16, hi[6] | hi[7] << 16);
        *reinterpret_cast<uint4*>(dst + u * 64 + 128) = make_uint4(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16, lo[4] | lo[5] << 16, lo[6] | lo[7] << 16);
    }
    exps[kt * 8 + g * 2 + half] = (char)e;
}

// The lanes of a wave that hold the same number below 2^bits, of those that are live
__device__ __forceinline__ uint64_t same_lanes(int id, bool live, int bits)
{
    uint64_t same = __ballot(live);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot(live && id >> b & 1);
        same &= id >> b & 1 ? set : ~set;
    }
    return same;
}

// ---------------------------------------------------------------- before the products: who goes where, and x in two parts

// Workgroup 0 sorts the choices by expert; the others convert x, a thread 32 numbers.  A choice's place among its expert's is
// whichever it gets from a counter in local memory: what a row gives does not depend on the rows beside it, nor on where it stands.
// Bound by latency (384 choices: 4.6 us), with many choices by the counters: 16384 take 14 to 16 us with 16 loads a thread at a time, 2 more with 4 (2 are enough
// up to 2048 choices, and less code).
__global__ void __launch_bounds__(1024) moe_prepare_kernel(ExpertsArgs a, int* total_tiles, Tile* tiles, int64_t max_tiles, int rows_log2, Divider by_top_k,
                                                           int* tile_rows, int* place, char* xs, char* xe)
{
    __shared__ int s_next[1024], s_first[1024], s_tile[1024], s_sum[2][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int E = a.e.n_experts;
    if (blockIdx.x > 0) {
        const int64_t blocks = a.e.hidden / 32, i = (int64_t)(blockIdx.x - 1) * 1024 + tid;
        if (i >= a.M * blocks) return;
        const int64_t m = i / blocks, b = i - m * blocks;
        split_block(a.x + m * a.ldx, (int)b, xs + m * moe::row_bytes(a.e.hidden), xe + m * moe::exp_bytes(a.e.hidden));
        return;
    }
    const int A = (int)(a.M * a.top_k), rows = 1 << rows_log2;
    s_next[tid] = 0;
    __syncthreads();
    auto sort = [&](auto at_once_c) {
        constexpr int AT_ONCE = decltype(at_once_c)::value;  // loads of 1024 choices under way together; the first ones stay in registers
        int kept[AT_ONCE], id[AT_ONCE];
        auto ask = [&](int i0, int (&to)[AT_ONCE]) {
#pragma unroll
            for (int b = 0; b < AT_ONCE; ++b) to[b] = i0 + b * 1024 < A ? a.ids[i0 + b * 1024] : -1;
        };
        auto count_them = [&](const int (&of)[AT_ONCE]) {
#pragma unroll
            for (int b = 0; b < AT_ONCE; ++b)
                if ((unsigned)of[b] < (unsigned)E) atomicAdd(&s_next[of[b]], 1);
        };
        ask(tid, kept);
        count_them(kept);
        for (int i0 = tid + 1024 * AT_ONCE; i0 < A; i0 += 1024 * AT_ONCE) {
            ask(i0, id);
            count_them(id);
        }
        __syncthreads();
        // thread e: expert e's rows, and where they and its tiles begin
        const int count = s_next[tid], n_tiles = (count + rows - 1) >> rows_log2;
        int first = count, tile = n_tiles;                   // inclusive sums over the experts
        for (int off = 1; off < 64; off <<= 1) {
            const int p = __shfl_up(first, off), q = __shfl_up(tile, off);
            if (lane >= off) { first += p; tile += q; }
        }
        if (lane == 63) { s_sum[0][wave] = first; s_sum[1][wave] = tile; }
        __syncthreads();
        int all_tiles = 0;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) { first += s_sum[0][w]; tile += s_sum[1][w]; }
            all_tiles += s_sum[1][w];
        }
        first -= count;
        tile -= n_tiles;
        if (tid == 0) *total_tiles = all_tiles;
        for (int t = 0; t < n_tiles; ++t) tiles[tile + t] = Tile{tid, first + t * rows, min(rows, count - t * rows), 0};
        for (int64_t t = all_tiles + tid; t < max_tiles; t += 1024) tiles[t] = Tile{0, 0, 0, 0};
        s_first[tid] = first;
        s_tile[tid] = tile;
        s_next[tid] = 0;
        __syncthreads();
        auto place_them = [&](int i0, const int (&of)[AT_ONCE]) {
            int n[AT_ONCE];
#pragma unroll
            for (int b = 0; b < AT_ONCE; ++b) n[b] = (unsigned)of[b] < (unsigned)E ? atomicAdd(&s_next[of[b]], 1) : 0;
#pragma unroll
            for (int b = 0; b < AT_ONCE; ++b) {
                const int i = i0 + b * 1024;
                const bool live = (unsigned)of[b] < (unsigned)E;
                if (live) tile_rows[(s_tile[of[b]] << rows_log2) + n[b]] = (int)divide((uint32_t)i, by_top_k);
                if (i < A) place[i] = live ? s_first[of[b]] + n[b] : -1;
            }
        };
        place_them(tid, kept);
        for (int i0 = tid + 1024 * AT_ONCE; i0 < A; i0 += 1024 * AT_ONCE) {
            ask(i0, id);
            place_them(i0, id);
        }
    };
    if (A <= 2048) sort(std::integral_constant<int, 2>{});
    else sort(std::integral_constant<int, 16>{});
}

// ---------------------------------------------------------------- the products

// 16 weights of a dword -> 16 four-bit numbers of the values q / 2: [0] the fields 0 and 2 of each byte, [1] 1 and 3.  q in two's complement
// (b1 b0): sign b1, magnitude b0 | (b1 & ~b0) << 1.
__device__ __forceinline__ void to_fp4(uint32_t w, int& lo, int& hi)
{
    const uint32_t mag = __builtin_amdgcn_bitop3_b32(w, w << 1, 0xaaaaaaaau, 0x70);       // w & ~(w << 1 & 0xaa..): magnitudes in place
    const uint32_t sign = w & 0xaaaaaaaau;
    lo = (int)__builtin_amdgcn_bitop3_b32(mag, sign << 2, 0x33333333u, 0xe4);             // bits of the mask from the first, the others from the second
    hi = (int)__builtin_amdgcn_bitop3_b32(mag >> 2, sign, 0x33333333u, 0xe4);
}

struct ProductArgs {
    const char* blob;
    int64_t blob_stride, codes_bytes;
    int n_kt;
    const Tile* tiles;
    const int* tile_rows;               // up: which row of x each row of a tile is (down: the places in the sorted order)
    const char *rows, *exps;            // in two parts
    char *h, *h_exps;                   // up: rows of n_out numbers in two parts
    float* z;                           // down: rows of n_out numbers
    int n_out;
};

// Scale of group g of the 256 k that a lane's scales belong to
template <int GPT>
struct Scales;
template <> struct Scales<2> { typedef uint32_t type; };
template <> struct Scales<4> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
__device__ __forceinline__ float scale_at(uint32_t d, int g) { return __uint_as_float(g ? d & 0xffff0000u : d << 16); }
__device__ __forceinline__ float scale_at(Scales<4>::type d, int g) { return __uint_as_float(g & 1 ? d[g >> 1] & 0xffff0000u : d[g >> 1] << 16); }

// x (eight-bit) times b (four-bit) into acc; ex's byte BYTE: the rows' power of two; the column's, 2^1, makes q of q / 2
template <int BYTE>
__device__ __forceinline__ v4f product(v8i x, const int (&b)[4], v4f acc, int ex)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, (v8i){b[0], b[1], b[2], b[3], 0, 0, 0, 0}, acc, 0, 4, BYTE, ex, 0, 128);
}

// A lane group's two exponents, in the lower bytes of a dword (what lies behind them, of the next group or the next buffer of the
// workspace, is not used; a load of 16 bits is widened where the compiler likes, and the wait for it stands there)
__device__ __forceinline__ int load_exponents(const char* p)
{
    int e;
    __builtin_memcpy(&e, p, 4);
    return e;
}

__device__ __forceinline__ v8i join(v4i a, v4i b) { return (v8i){a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}; }

// Up to 8 rows, each of them in the instruction twice, hi and lo.  Its row 4 q + i leaves in number i of lane group q, so with 2 L rows (L = 1, 2, 4)
// row r's parts stand at 4 (r / L) + r % L and 8 further on: a lane then has L numbers to scale and add, not four.
template <int L>
__device__ __forceinline__ int row_of_lane(int col) { return (col >> 2 & 1) * L + (col & (L - 1)); }

// Half j of a lane's 256 k of one column block, rows x in one part each, onto y
template <int GPT, int J, int L>
__device__ __forceinline__ void multiply(v8i x, int e, v4i w, typename Scales<GPT>::type sc, float (&y)[L])
{
    int b[4];
    to_fp4((uint32_t)w[2 * J], b[0], b[1]);
    to_fp4((uint32_t)w[2 * J + 1], b[2], b[3]);
    const v4f zero = {0, 0, 0, 0};
    auto add = [&](v4f p, float scale) {
#pragma unroll
        for (int i = 0; i < L; ++i) y[i] = fmaf(p[i], scale, y[i]);
    };
    if constexpr (GPT == 2) add(product<J>(x, b, zero, e), scale_at(sc, J));
    else {
        add(product<J>(x, {b[0], b[1], 0, 0}, zero, e), scale_at(sc, 2 * J));
        add(product<J>(x, {0, 0, b[2], b[3]}, zero, e), scale_at(sc, 2 * J + 1));
    }
}

template <int L>
__device__ __forceinline__ void hold(float (&y)[2][L])       // the sums are here now, the products not carried on
{
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < L; ++i) asm volatile("" : "+v"(y[n][i]));
}

// f with the L that up to 8 rows need
template <typename F>
__device__ __forceinline__ void with_rows(int rows, F f)
{
    if (rows <= 2) f(std::integral_constant<int, 1>{});
    else if (rows <= 4) f(std::integral_constant<int, 2>{});
    else f(std::integral_constant<int, 4>{});
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const void* p, int64_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(uint32_t)min(bytes, (int64_t)0xffffffff), 0x00020000);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t resource32(const void* p, int bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}

// (the reciprocal is good to one step of fp32; an infinite exponential gives 0)
__device__ __forceinline__ float silu_mul(float g, float u) { return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * u; }

// |h| where it counts for the power of two that numbers share: infinities and NaN stay what they are beside any
__device__ __forceinline__ float finite_or_zero(float h)
{
    h = fabsf(h);
    return h < INFINITY ? h : 0.0f;
}

// exponent field of the largest of 16 lanes' numbers
__device__ __forceinline__ int largest_field(float m)
{
    m = fmaxf(m, dpp_move_f32<0xB1>(m));
    m = fmaxf(m, dpp_move_f32<0x4E>(m));
    m = fmaxf(m, dpp_move_f32<0x141>(m));
    m = fmaxf(m, dpp_move_f32<0x140>(m));
    return (int)(__float_as_uint(m) >> 23);
}

// What the wave of a pair of blocks leaves of h, in two parts (every wave of the workgroup calls it).  The workgroup's P pairs are the
// units c0 .. c0 + P/2 - 1 and those four further on of the 128 numbers u of h.  s_mem: P * 16 * 36 bytes.
template <int P, int L, typename F>
__device__ __forceinline__ void store_h(char* hs, char* he, int inter, int rows, F place, char* s_mem, float (&y)[2][L], int p, bool mine, int u, int c0, int threads)
{
    constexpr int R = 4 * L;            // (half of them: hi's and lo's sums have met, lanes 32 apart hold the same)
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, q = lane >> 4;
    int* const s_top = reinterpret_cast<int*>(s_mem);        // [P][R]: exponent field of the largest |h| of a row's unit
    char* const s_out = s_mem + P * R * 4;                   // [R][2 parts][P units][16]
    float h[L];
    if (mine) {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            h[i] = silu_mul(y[0][i], y[1][i]);
            const int top = largest_field(finite_or_zero(h[i]));
            if (col == 0) s_top[p * R + q * L + i] = top;
        }
    }
    __syncthreads();
    if (mine) {
        const int byte = 2 * (col & 7) + (col >> 3);
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int m = q * L + i;
            const int ex = shared_exponent(max(s_top[p % (P / 2) * R + m], s_top[(p % (P / 2) + P / 2) * R + m]));
            uint32_t hi, lo;
            split2(h[i], 0.0f, scale_down(ex), hi, lo);
            s_out[((m * 2 + 0) * P + p) * 16 + byte] = (char)hi;
            s_out[((m * 2 + 1) * P + p) * 16 + byte] = (char)lo;
            if (p < P / 2 && col == 0 && m < rows) he[(int64_t)place(m) * moe::exp_bytes(inter) + u / 2 * 8 + (c0 + p) * 2 + (u & 1)] = (char)ex;
        }
    }
    __syncthreads();
    for (int i = tid; i < rows * 2 * P; i += threads) {      // 16 bytes: a unit of a part of a row
        const int m = i / (2 * P), part = i / P % 2, pp = i % P;
        const int to_unit = c0 + pp % (P / 2) + pp / (P / 2) * 4;
        *reinterpret_cast<uint4*>(hs + (int64_t)place(m) * moe::row_bytes(inter) + u * 256 + part * 128 + to_unit * 16) =
            *reinterpret_cast<const uint4*>(s_out + i * 16);
    }
}

// Sums of a pair of blocks: hi's and lo's, then the ranges of K, in their order, in local memory ([KS - 1][P][2 L][64])
template <int KS, int P, int L>
__device__ __forceinline__ void join_sums(float (&y)[2][L], float* part, int p, int kr, int lane)
{
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < L; ++i) y[n][i] += __shfl_xor(y[n][i], 32);
    if constexpr (KS > 1) {
        if (kr > 0) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < L; ++i) part[(((kr - 1) * P + p) * 2 * L + n * L + i) * 64 + lane] = y[n][i];
        }
        __syncthreads();
        if (kr == 0) {
#pragma unroll
            for (int k = 0; k < KS - 1; ++k)
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int i = 0; i < L; ++i) y[n][i] += part[((k * P + p) * 2 * L + n * L + i) * 64 + lane];
        }
        __syncthreads();
    }
}

// Few rows: bound by the weights' way from memory (384 choices of 128 experts of 4096 x 1024, nearly all of which have some: 268 MB of gate and up in
// 45 us, 6 TB/s, 134 MB of down in 27; the loads alone 42.6 and 22.8).  A workgroup: four waves = 4 / KS pairs of column blocks times KS ranges of K, up to
// eight rows of one expert, hi in rows 0 to 7 of the instruction, lo in 8 to 15.  UP: a pair is a block of gate columns and one of up columns;
// silu(gate) * up leaves in two parts.  Not UP: two blocks; sums leave in fp32.  The next four tiles of weights of each column block are
// under way while one is multiplied; rows come through local memory, four tiles of K (over all ranges) at a time.  Every load
// is unconditional, what lies past a wave's range is out of its resource and reads as zeros, so that the waits count exactly.
constexpr int FEW_W = 4, FEW_WAVES = 4, FEW_ROWS = 8;
constexpr int NT = 2;                   // weights pass through the caches once

template <int KS>
struct FewShape {
    static constexpr int P = FEW_WAVES / KS, CK = 4 / KS, R = FEW_ROWS, STRIDE = CK * 512 + 16, BUFFER = KS * R * STRIDE, EXPS = KS * R * CK * 8;
    static constexpr int THREADS = FEW_WAVES * 64, PIECES = KS * CK;
    static_assert(THREADS == R * 32, "a thread fetches 16 bytes of its row's 512 of each tile");
    // what leaves: the ranges' sums, the largest numbers and two parts of h
    static constexpr int LEAVE = std::max((KS - 1) * P * 2048, P * 16 * 36), LDS = 2 * BUFFER + 2 * EXPS + 512 + LEAVE;
};

template <bool UP, int KS, int GPT>
__global__ void __launch_bounds__(FEW_WAVES * 64, GPT == 2 ? 4 : 3) moe_few_kernel(ProductArgs a, int64_t row_bytes_all)
{
    typedef FewShape<KS> S;
    constexpr int P = S::P, CK = S::CK, R = S::R, STRIDE = S::STRIDE, BUFFER = S::BUFFER, EXPS = S::EXPS, THREADS = S::THREADS;
    extern __shared__ char s_mem[];                          // [2][KS][R][STRIDE], exponents [2][KS][R][CK * 8], 512 bytes for no one; what leaves
    char* const s_leave = s_mem + 2 * BUFFER + 2 * EXPS + 512;
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Tile tile = a.tiles[blockIdx.y];
    // which rows (of what may be there: how many are is not known yet)
    const int* const tile_rows = a.tile_rows + (int64_t)blockIdx.y * R;
    const int r_in = tid / 32, r_e = tid % R, t_e = tid / R; // KS * CK * R threads: the exponents of a row's tile each
    const bool has_e = tid < KS * CK * R;
    uint32_t row = UP ? tile_rows[r_in] : r_in, row_e = UP ? tile_rows[r_e] : r_e;
    if (tile.rows == 0) return;
    with_rows(tile.rows, [&](auto l_c) {
        constexpr int L = decltype(l_c)::value;
        const int p = wave % P, kr = wave / P;
        const int steps = (a.n_kt + KS - 1) / KS;
        const int kt0 = kr * steps, my_steps = max(0, min(steps, a.n_kt - kt0));
        const char* const blob = a.blob + tile.expert * a.blob_stride;
        // pairs of a workgroup lie so that the units g and g + 4 of 128 numbers of h are both its own
        constexpr int GROUPS = 8 / P;
        const int group = blockIdx.x, pair = UP ? group / GROUPS * 8 + group % GROUPS * (P / 2) + p % (P / 2) + p / (P / 2) * 4 : group * P + p;
        __amdgpu_buffer_rsrc_t wr[2], sr[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int64_t t = (int64_t)(2 * pair + c) * a.n_kt + kt0;
            wr[c] = resource32(blob + t * 1024, my_steps * 1024);
            sr[c] = resource32(blob + a.codes_bytes + t * 32 * GPT, my_steps * 32 * GPT);
        }
        v4i w[FEW_W][2];
        typename Scales<GPT>::type sc[FEW_W][2];
        auto load_weights = [&](int s, int slot) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                w[slot][c] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(wr[c], s * 1024 + lane * 16, 0, NT));
                if constexpr (GPT == 2) sc[slot][c] = __builtin_amdgcn_raw_buffer_load_b32(sr[c], s * 64 + col * 4, 0, 0);
                else sc[slot][c] = __builtin_bit_cast(Scales<4>::type, __builtin_amdgcn_raw_buffer_load_b64(sr[c], s * 128 + col * 8, 0, 0));
            }
        };

        // a row that is not there is out of range
        const __amdgpu_buffer_rsrc_t rr = resource(a.rows, row_bytes_all), er = resource(a.exps, row_bytes_all / 64);
        const int n_in = r_in < tile.rows ? a.n_kt : 0, n_in_e = has_e && r_e < tile.rows ? a.n_kt : 0;     // tiles of K that the row has
        if (!UP) {
            row += tile.first;
            row_e += tile.first;
        }
        const uint32_t src = row * (uint32_t)(a.n_kt * 512) + tid % 32 * 16, src_e = row_e * (uint32_t)(a.n_kt * 8);
        char* const to = s_mem + r_in * STRIDE + tid % 32 * 16;
        // (the other threads write beside them: without a branch, past which the compiler would carry the products and all their operands)
        char* const to_e = s_mem + 2 * BUFFER + (has_e ? ((t_e / CK * R + r_e) * CK + t_e % CK) * 8 : 2 * EXPS + (tid & 63) * 8);
        const int next_e = has_e ? EXPS : 0;
        v4i staged[S::PIECES];
        uint2 staged_e;
        auto fetch = [&](int s) {           // s: first of the CK steps
#pragma unroll
            for (int i = 0; i < S::PIECES; ++i) {
                const int kt = i / CK * steps + i % CK + s;
                staged[i] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rr, kt < n_in ? src + kt * 512 : 0xffffffffu, 0, 0));
            }
            const int kt = t_e / CK * steps + t_e % CK + s;
            staged_e = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(er, kt < n_in_e ? src_e + kt * 8 : 0xffffffffu, 0, 0));
        };
        auto put = [&](int buffer) {
#pragma unroll
            for (int i = 0; i < S::PIECES; ++i) *reinterpret_cast<v4i*>(to + buffer * BUFFER + i / CK * R * STRIDE + i % CK * 512) = staged[i];
            *reinterpret_cast<uint2*>(to_e + buffer * next_e) = staged_e;
        };
        // in the order of the loop, whose waits count what is under way from either side
        fetch(0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < FEW_W; ++i) {
            load_weights(i, i);
            __builtin_amdgcn_sched_barrier(0);
        }
        put(0);
        __syncthreads();

        const int unit = 4 * (q & 1) + (q >> 1);
        const int lo_exp = (col >> 3) * 0x0505;
        const int row_in = kr * R + row_of_lane<L>(col);
        const char* const at = s_mem + row_in * STRIDE + unit * 16 + (col >> 3) * 128;
        const char* const at_e = s_mem + 2 * BUFFER + row_in * CK * 8 + q * 2;
        int turn = 0;                   // the buffer that a chunk of four steps begins in
        float y[2][L] = {};
        // step s, with the weights in slot i, or what is left behind the last four
        auto step = [&](int s, auto i_c, auto rest_c) {
            constexpr int i = decltype(i_c)::value;
            constexpr bool REST = decltype(rest_c)::value;
            if (i % CK == 0 && !(REST && i + CK >= FEW_W)) fetch(s + CK);
            const int buffer = (i / CK + turn) & 1;
            // (up-converted only now: a turn early, as they come, the weights would take twice the registers)
            asm volatile("" : "+v"(w[i][0]), "+v"(w[i][1]), "+v"(sc[i][0]), "+v"(sc[i][1]));
            const char* const x0 = at + buffer * BUFFER + i % CK * 512;
            const int e = *reinterpret_cast<const uint16_t*>(at_e + buffer * EXPS + i % CK * 8) - lo_exp;
            auto half = [&](auto jc) {
                constexpr int j = decltype(jc)::value;
                const v8i x = join(*reinterpret_cast<const v4i*>(x0 + j * 256), *reinterpret_cast<const v4i*>(x0 + j * 256 + 32));
#pragma unroll
                for (int n = 0; n < 2; ++n) multiply<GPT, j>(x, e, w[i][n], sc[i][n], y[n]);
            };
            half(std::integral_constant<int, 0>{});
            half(std::integral_constant<int, 1>{});
            // here, and not where they are read: carried on, the products' operands would take every register
            hold(y);
            __builtin_amdgcn_sched_barrier(0);
            if (!REST) load_weights(s + FEW_W, i);
            if (i % CK == CK - 1) {
                put((i / CK + 1 + turn) & 1);
                __syncthreads();
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        typedef std::integral_constant<bool, false> Loop;
        typedef std::integral_constant<bool, true> Rest;
        int s = 0;
        for (; s + FEW_W <= steps; s += FEW_W) {
            step(s, std::integral_constant<int, 0>{}, Loop{});
            step(s + 1, std::integral_constant<int, 1>{}, Loop{});
            step(s + 2, std::integral_constant<int, 2>{}, Loop{});
            step(s + 3, std::integral_constant<int, 3>{}, Loop{});
            if (CK == 4) turn ^= 1;
        }
        if (s < steps) step(s, std::integral_constant<int, 0>{}, Rest{});
        if (s + 1 < steps) step(s + 1, std::integral_constant<int, 1>{}, Rest{});
        if (s + 2 < steps) step(s + 2, std::integral_constant<int, 2>{}, Rest{});
        join_sums<KS, P>(y, reinterpret_cast<float*>(s_leave), p, kr, lane);
        if constexpr (UP) {
            store_h<P>(a.h, a.h_exps, a.n_out, tile.rows, [&](int m) { return tile.first + m; }, s_leave, y, p, kr == 0, group / GROUPS, group % GROUPS * (P / 2), THREADS);
        } else if (kr == 0) {
#pragma unroll
            for (int i = 0; i < L; ++i) {
                const int m = q * L + i;
                if (m < tile.rows) {
                    float* const out = a.z + (int64_t)(tile.first + m) * a.n_out + pair * 32 + col;
                    out[0] = y[0][i];
                    out[16] = y[1][i];
                }
            }
        }
    });
}

// Many rows: bound by the matrix pipe and the vector instructions beside it.  A workgroup: four waves of 64 columns each (two pairs of
// blocks), up to 32 rows of one expert (16, where there are no more: RT = 1).  As wide a wave as that because each wave reads every row's
// operands: with 32 columns a wave 1806 choices of 64 experts of 2048 x 768 took 26.8 us for gate and up, not 24.3.  Tiles of 64 rows (two waves a
// SIMD) took 175 and 108 us for the sizes below, those of 32 168 and 103 at that time.  A stage is 128 of K: its rows go from global to local memory directly, a KiB (256 bytes of four
// rows) per instruction, in a ring of four; the 16-byte piece p of row r stands at p ^ (r mod 16), so that reads of 16 rows
// touch every bank once.  Weights and exponents of 256 of K are asked for two tiles ahead.
//
// Of a stage's column blocks the products of the last one begin behind the barrier at which the next stage's rows are there; those are read
// into registers as the products let go of them.  What may be under way at a barrier is counted (moe_plan.h).  An operation more than counted makes
// the wait longer; one fewer, a load that the compiler joins with another or drops, would let a barrier pass before its rows have landed.  So every load is
// unconditional, and the compiled kernel's own order is walked by a test.
//
// 16384 choices of 64 experts of 2048 x 1024: 142 to 161 us as the clock goes (1.6 to 2.1 GHz) for gate and up, 86 to 100 for down, of which the
// products are 63 and 32 at 2.1 GHz (32 cycles each).  A workgroup takes 1.2 us to know its tile, 3.1 until rows are there, 15 for 2048 of K and 2.6 to leave;
// a SIMD has two of its three waves in the loop at a time.  Neither the loads nor any one kind of vector instruction bounds the loop by itself
// (left out one by one: 127 to 133 us for 132).
constexpr int TILE_ROWS = 32, RING = moe::TILE_AHEAD + 1;
static_assert((RING & (RING - 1)) == 0, "a stage's place in the ring");

template <bool UP, int GPT>
__global__ void __launch_bounds__(256, GPT == 2 ? 3 : 2) moe_tile_kernel(ProductArgs a, int64_t row_bytes_all, const int* n_tiles, int col_groups)
{
    __shared__ __align__(16) char s_mem[RING * TILE_ROWS * 256];
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // the workgroups of an XCD take tiles in a row: row tiles of an expert meet its weights in that die's L2
    const int total = *n_tiles * col_groups, per = (total + 7) / 8, idx = blockIdx.x >> 3, lin = (blockIdx.x & 7) * per + idx;
    if (idx >= per || lin >= total) return;
    const int cg = lin % col_groups;
    const int* const tile_rows = a.tile_rows + (int64_t)(lin / col_groups) * TILE_ROWS;
    const Tile tile = a.tiles[lin / col_groups];
    int pair[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) pair[n] = cg * 8 + (UP ? wave + 4 * n : wave * 2 + n);
    const char* const blob = a.blob + tile.expert * a.blob_stride;
    const char *codes[4], *scales[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const int64_t t = (int64_t)(2 * pair[c / 2] + c % 2) * a.n_kt;
        codes[c] = blob + t * 1024;
        scales[c] = blob + a.codes_bytes + t * 32 * GPT;
    }
    auto row_of = [&](int r) -> int64_t {                    // (rows that are not there: the last one again)
        r = min(r, tile.rows - 1);
        return UP ? tile_rows[r] : tile.first + r;
    };
    auto body = [&](auto rt_c) {
        constexpr int RT = decltype(rt_c)::value, BUFFER = RT * 16 * 256;
        const __amdgpu_buffer_rsrc_t rows = resource(a.rows, row_bytes_all);
        uint32_t src[RT];
        uint32_t exps[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = (wave * RT + r) * 4 + q;         // of the KiB that this wave brings
            src[r] = (uint32_t)row_of(row) * (uint32_t)(a.n_kt * 512) + (col ^ (row & 15)) * 16;
            exps[r] = (uint32_t)row_of(r * 16 + col) * (uint32_t)(a.n_kt * 8) + q * 2;
        }
        struct Weights {
            v4i w[4];
            typename Scales<GPT>::type sc[4];
            int e[RT];
        } wa, wb;
        auto load_weights = [&](int kt, Weights& r) {        // (past the last tile: that one again, the loads are counted)
            kt = min(kt, a.n_kt - 1);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                r.w[c] = *reinterpret_cast<const v4i*>(codes[c] + (int64_t)kt * 1024 + lane * 16);
                r.sc[c] = *reinterpret_cast<const typename Scales<GPT>::type*>(scales[c] + (int64_t)kt * 32 * GPT + col * 2 * GPT);
            }
#pragma unroll
            for (int i = 0; i < RT; ++i) r.e[i] = load_exponents(a.exps + (exps[i] + (uint32_t)kt * 8));
        };
        auto load_rows = [&](int stage) {
            char* const to = s_mem + (stage & (RING - 1)) * BUFFER + wave * RT * 1024;
            const uint32_t off = (uint32_t)min(stage, 2 * a.n_kt - 1) * 256;
#pragma unroll
            for (int r = 0; r < RT; ++r) load_to_lds(rows, (int8_t*)to + r * 1024, src[r], off);
        };
        int at[4];                      // hi and lo, lower and upper 16 bytes of a lane's operand
        const int unit = 4 * (q & 1) + (q >> 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] = col * 256 + (((i >> 1) * 8 + unit + (i & 1) * 2) ^ col) * 16;
        v4f y[RT][4] = {};
        // Under way: the next column block's weights in four bits, and the last products, to be scaled and added.  Vector instructions
        // of the block before and the block behind stand between a block's products (sched_barrier), so that neither waits for the other.
        int b[4];
        v4f p[RT] = {};
        float p_scale = 0.0f;
        auto add = [&](int r, int c) {
#pragma unroll
            for (int i = 0; i < 4; ++i) y[r][c][i] = fmaf(p[r][i], p_scale, y[r][c][i]);
        };
        v8i hi[RT], lo[RT];
        auto part = [&](int s, int r, int i) {
            const char* const x = s_mem + (s & (RING - 1)) * BUFFER + r * 4096;
            return join(*reinterpret_cast<const v4i*>(x + at[2 * i]), *reinterpret_cast<const v4i*>(x + at[2 * i + 1]));
        };
        auto stage = [&](int s, auto jc, const Weights& wt, const Weights& next) {       // next: the weights of the stage behind, half 1 - j
            constexpr int j = decltype(jc)::value;
            const v4f zero = {0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (c == 3) {
                    wait_loads<moe::tile_at_stage(RT)>();
                    bare_barrier();
                    load_rows(s + moe::TILE_AHEAD);
                    __builtin_amdgcn_sched_barrier(0);
                }
                const v4i& w = c < 3 ? wt.w[c + 1] : next.w[0];
                const int half = c < 3 ? j : 1 - j;
                int n[4];
#pragma unroll
                for (int g = 0; g < GPT / 2; ++g) {
                    const int bg[4] = {g == 0 ? b[0] : 0, g == 0 ? b[1] : 0, GPT == 2 || g ? b[2] : 0, GPT == 2 || g ? b[3] : 0};
                    const int last = g ? c : (c + 3) % 4;
                    v4f q[RT];
                    q[0] = product<j>(lo[0], bg, zero, wt.e[0] - 0x0505);
                    if (g == 0) to_fp4((uint32_t)w[2 * half], n[0], n[1]);
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (RT == 2) q[1] = product<j>(lo[1], bg, zero, wt.e[1] - 0x0505);
                    if (g == GPT / 2 - 1) to_fp4((uint32_t)w[2 * half + 1], n[2], n[3]);
                    __builtin_amdgcn_sched_barrier(0);
                    if (c == 3 && g == GPT / 2 - 1) {
#pragma unroll
                        for (int r = 0; r < RT; ++r) lo[r] = part(s + 1, r, 1);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    q[0] = product<j>(hi[0], bg, q[0], wt.e[0]);
                    add(0, last);
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (RT == 2) {
                        q[1] = product<j>(hi[1], bg, q[1], wt.e[1]);
                        add(1, last);
                    }
                    p_scale = scale_at(wt.sc[c], GPT / 2 * j + g);
                    __builtin_amdgcn_sched_barrier(0);
                    if (c == 3 && g == GPT / 2 - 1) {
#pragma unroll
                        for (int r = 0; r < RT; ++r) hi[r] = part(s + 1, r, 0);
                        __builtin_amdgcn_sched_barrier(0);
                    }
#pragma unroll
                    for (int r = 0; r < RT; ++r) p[r] = q[r];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) b[i] = n[i];
            }
        };
        // in the order of the loop: stage 0's wait counts what the others do
        load_weights(0, wa);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < moe::TILE_AHEAD; ++s) load_rows(s);
        __builtin_amdgcn_sched_barrier(0);
        load_weights(1, wb);
        to_fp4((uint32_t)wa.w[0][0], b[0], b[1]);
        to_fp4((uint32_t)wa.w[0][1], b[2], b[3]);
        wait_loads<moe::tile_at_start(RT)>();
        bare_barrier();
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            lo[r] = part(0, r, 1);
            hi[r] = part(0, r, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        auto tile_of_k = [&](int kt, Weights& wt, const Weights& next) {
            stage(2 * kt, std::integral_constant<int, 0>{}, wt, wt);
            // the second half of the tile needs its weights still: the next but one's follow it
            stage(2 * kt + 1, std::integral_constant<int, 1>{}, wt, next);
            load_weights(kt + 2, wt);
            __builtin_amdgcn_sched_barrier(0);
        };
        int kt = 0;                     // (two at a time without a branch between them, past which the compiler would count fewer loads)
        for (; kt + 1 < a.n_kt; kt += 2) {
            tile_of_k(kt, wa, wb);
            tile_of_k(kt + 1, wb, wa);
        }
        if (kt < a.n_kt) tile_of_k(kt, wa, wb);
#pragma unroll
        for (int r = 0; r < RT; ++r) add(r, 3);
        wait_loads<0>();                // what was asked for past the end has landed
        __syncthreads();
        if constexpr (UP) {
            // the wave's two pairs are the units g = wave and g + 4 of 128 numbers of h: they share a power of two
            char* const s_out = s_mem;                       // [rows][2 parts][8 units][16], then exponents [rows][4]
            char* const s_exp = s_mem + TILE_ROWS * 256;
            const int byte = 2 * (col & 7) + (col >> 3);
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int m = r * 16 + q * 4 + i;
                    const float h0 = silu_mul(y[r][0][i], y[r][1][i]), h1 = silu_mul(y[r][2][i], y[r][3][i]);
                    const int ex = shared_exponent(largest_field(fmaxf(finite_or_zero(h0), finite_or_zero(h1))));
                    uint32_t hi, lo;
                    split2(h0, h1, scale_down(ex), hi, lo);
                    char* const to16 = s_out + m * 256 + wave * 16 + byte;
                    to16[0] = (char)hi;
                    to16[64] = (char)(hi >> 8);
                    to16[128] = (char)lo;
                    to16[192] = (char)(lo >> 8);
                    s_exp[m * 4 + wave] = (char)ex;          // (the same from 16 lanes)
                }
            __syncthreads();
            if (tid < tile.rows * 4)
                a.h_exps[(int64_t)(tile.first + tid / 4) * moe::exp_bytes(a.n_out) + cg / 2 * 8 + tid % 4 * 2 + (cg & 1)] = s_exp[tid];
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const int m = r * 16 + tid / 16;
                if (m < tile.rows)
                    *reinterpret_cast<uint4*>(a.h + (int64_t)(tile.first + m) * moe::row_bytes(a.n_out) + cg * 256 + tid % 16 * 16) =
                        *reinterpret_cast<const uint4*>(s_out + m * 256 + tid % 16 * 16);
            }
        } else {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int m = r * 16 + q * 4 + i;
                    if (m < tile.rows) {
                        float* const out = a.z + (int64_t)(tile.first + m) * a.n_out + pair[0] * 32 + col;
#pragma unroll
                        for (int c = 0; c < 4; ++c) out[16 * c] = y[r][c][i];
                    }
                }
        }
    };
    if (tile.rows <= 16) body(std::integral_constant<int, 1>{});
    else body(std::integral_constant<int, 2>{});
}

// ---------------------------------------------------------------- up to 64 choices in two launches

// Every workgroup finds out for itself which rows share an expert: lane i of a wave holds choice i.  Tiles of up to eight
// choices of one expert, in the order of their first ones.  One row of 8 experts of 4096 x 1024 (25 MB, 3.8 us at the rate of a large read): 7.9 + 6.9 us,
// launch and four trips to memory one behind the other (choices, rows or weights' addresses, weights, sums) each; four launches 21.5.
struct Choice {
    int id, tile, row;                  // of lane i's choice: its expert (-1: none), its tile, its row there
    int tiles;                          // all of them
};

__device__ __forceinline__ Choice choose(const int32_t* ids, int A, int E)
{
    const int lane = threadIdx.x & 63;
    Choice c;
    const int id = lane < A ? ids[lane] : -1;
    const bool live = (unsigned)id < (unsigned)E;
    const uint64_t before = ((uint64_t)1 << lane) - 1;
    uint64_t same = same_lanes(id, live, 32 - __clz(E));
    const int nth = __popcll(same & before);
    const uint64_t firsts = __ballot(live && nth % 8 == 0);
    // the first choice of the lane's tile: eight choices of the expert further on for each tile before it
    for (int n = nth / 8; __any(live && n > 0); --n)
        if (n > 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) same &= same - 1;
        }
    c.id = live ? id : -1;
    c.row = nth % 8;
    c.tile = live ? __popcll(firsts & (((uint64_t)1 << (__ffsll((unsigned long long)same) - 1)) - 1)) : -1;
    c.tiles = __popcll(firsts);
    return c;
}

constexpr int TINY_EARLY = 2;          // rows of x that are brought in before it is known whose they are
constexpr int TINY_W = 4;              // tiles of weights under way

// A workgroup: a tile and `units` groups of two pairs of blocks.  It brings its rows into two parts in local memory itself, all of K,
// and then streams weights past them, a group's end under the next one's loads; h leaves by the number of its choice.
template <int GPT>
__global__ void __launch_bounds__(512, 2) moe_tiny_up_kernel(ExpertsArgs a, char* hs, char* he, int units, int lds_rows)
{
    constexpr int P = moe::TINY_P, KS = moe::TINY_KS;
    extern __shared__ char s_all[];                          // what leaves, choices [8], rows [lds_rows][2 K + 16], exponents [lds_rows][K / 32]
    char *const s_leave = s_all, *const s_mem = s_all + moe::TINY_LEAVE;
    int* const s_row = reinterpret_cast<int*>(s_all + moe::TINY_SUMS);
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int A = (int)(a.M * a.top_k), n_kt = (int)(a.e.hidden / 256);
    const int stride = n_kt * 512 + 16, blocks = n_kt * 8;
    char* const s_exp = s_mem + lds_rows * stride;
    auto bring = [&](int rows, auto source) {                // 32 numbers at a time
        for (int r = 0, b = tid; r < rows; b += 512) {
            while (r < rows && b >= blocks) {
                b -= blocks;
                ++r;
            }
            if (r < rows) split_block(a.x + source(r) * a.ldx, b, s_mem + r * stride, s_exp + r * blocks);
        }
    };
    // one or two rows of x are brought in before it is known which choices they are
    const bool early = a.M <= TINY_EARLY;
    const Choice c = choose(a.ids, A, a.e.n_experts);
    if (early) bring((int)a.M, [](int r) { return (int64_t)r; });
    if ((int)blockIdx.y >= c.tiles) return;
    const uint64_t mine = __ballot(c.tile == (int)blockIdx.y);
    const int rows = __popcll(mine), expert = __builtin_amdgcn_readlane(c.id, __ffsll((unsigned long long)mine) - 1);
    with_rows(rows, [&](auto l_c) {
        constexpr int L = decltype(l_c)::value;
        const int p = wave % P, kr = wave / P;
        const int steps = (n_kt + KS - 1) / KS, steps4 = (steps + TINY_W - 1) / TINY_W * TINY_W;
        const int kt0 = kr * steps, my_steps = max(0, min(steps, n_kt - kt0));
        const char* const blob = (const char*)a.e.gate_up + expert * a.e.gate_up_stride;
        constexpr int GROUPS = 8 / P;       // pairs of a workgroup lie so that the units g and g + 4 of 128 numbers of h are both its own
        struct Weights {                    // of the wave's first column block, its range of K; the second one follows
            const char *codes, *scales;
            int tiles;
        };
        auto weights_of = [&](int unit) {
            const int group = blockIdx.x * units + unit;
            const int pair = group / GROUPS * 8 + group % GROUPS * (P / 2) + p % (P / 2) + p / (P / 2) * 4;
            const int64_t t = (int64_t)(2 * pair) * n_kt + kt0;
            return Weights{blob + t * 1024, blob + a.up.codes_bytes + t * 32 * GPT, unit < units ? my_steps : 0};
        };
        v4i w[TINY_W][2];
        typename Scales<GPT>::type sc[TINY_W][2];
        auto load_weights = [&](const Weights& r, int s, int slot) {
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const __amdgpu_buffer_rsrc_t wr = resource32(r.codes + (int64_t)n * n_kt * 1024, r.tiles * 1024);
                const __amdgpu_buffer_rsrc_t sr = resource32(r.scales + (int64_t)n * n_kt * 32 * GPT, r.tiles * 32 * GPT);
                w[slot][n] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(wr, s * 1024 + lane * 16, 0, NT));
                if constexpr (GPT == 2) sc[slot][n] = __builtin_amdgcn_raw_buffer_load_b32(sr, s * 64 + col * 4, 0, 0);
                else sc[slot][n] = __builtin_bit_cast(Scales<4>::type, __builtin_amdgcn_raw_buffer_load_b64(sr, s * 128 + col * 8, 0, 0));
            }
        };
        Weights now = weights_of(0);
#pragma unroll
        for (int i = 0; i < TINY_W; ++i) {                       // in the order of the loop, whose waits count what is under way from either side
            load_weights(now, i, i);
            __builtin_amdgcn_sched_barrier(0);
        }

        if (wave == 0 && c.tile == (int)blockIdx.y) s_row[c.row] = lane;
        __syncthreads();
        if (!early) {
            bring(rows, [&](int r) { return (int64_t)(s_row[r] / a.top_k); });
            __syncthreads();
        }

        const int lo_exp = (col >> 3) * 0x0505;
        const int nth = min(row_of_lane<L>(col), rows - 1), row = early ? s_row[nth] / a.top_k : nth;         // (rows that are not there: the last one again)
        const char* const at = s_mem + row * stride + (4 * (q & 1) + (q >> 1)) * 16 + (col >> 3) * 128;
        const char* const at_e = s_exp + row * blocks + q * 2;
        for (int unit = 0; unit < units; ++unit) {
            const Weights then = weights_of(unit + 1);
            float y[2][L] = {};
            for (int s = 0; s < steps4; s += TINY_W) {
                const bool last = s + TINY_W >= steps4;
                const Weights ahead = last ? then : now;
                const int s_ahead = last ? 0 : s + TINY_W;
#pragma unroll
                for (int i = 0; i < TINY_W; ++i) {
                    asm volatile("" : "+v"(w[i][0]), "+v"(w[i][1]), "+v"(sc[i][0]), "+v"(sc[i][1]));
                    const int kt = min(kt0 + s + i, n_kt - 1);         // (past the range: weights of zero, and numbers that are there)
                    const char* const x0 = at + kt * 512;
                    const int e = *reinterpret_cast<const uint16_t*>(at_e + kt * 8) - lo_exp;
                    auto half = [&](auto jc) {
                        constexpr int j = decltype(jc)::value;
                        const v8i x = join(*reinterpret_cast<const v4i*>(x0 + j * 256), *reinterpret_cast<const v4i*>(x0 + j * 256 + 32));
#pragma unroll
                        for (int n = 0; n < 2; ++n) multiply<GPT, j>(x, e, w[i][n], sc[i][n], y[n]);
                    };
                    half(std::integral_constant<int, 0>{});
                    half(std::integral_constant<int, 1>{});
                    hold(y);
                    __builtin_amdgcn_sched_barrier(0);
                    load_weights(ahead, s_ahead + i, i);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            join_sums<KS, P>(y, reinterpret_cast<float*>(s_leave), p, kr, lane);
            const int group = blockIdx.x * units + unit;
            store_h<P>(hs, he, (int)a.e.inter, rows, [&](int m) { return s_row[m]; }, s_leave, y, p, kr == 0, group / GROUPS, group % GROUPS * (P / 2), 512);
            __syncthreads();
            now = then;
        }
    });
}

// A workgroup: one block of columns, eight waves.  All tiles one behind the other are a run of K that the waves share out; a wave adds
// a tile's rows, weighted, to its sums of every row of Y, and the waves' sums meet in their order.
template <int GPT>
__global__ void __launch_bounds__(512, 2) moe_tiny_down_kernel(ExpertsArgs a, const char* hs, const char* he)
{
    extern __shared__ char s_mem[];                          // sums [8][M][16]
    __shared__ int s_row[64][8], s_expert[64], s_rows[64];
    __shared__ float s_weight[64];
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int A = (int)(a.M * a.top_k), M = (int)a.M, n_kt = (int)(a.e.inter / 256);
    const Choice c = choose(a.ids, A, a.e.n_experts);
    if (wave == 0) {
        s_rows[lane] = 0;
        if (c.id >= 0) {
            s_row[c.tile][c.row] = lane;
            s_expert[c.tile] = c.id;
            atomicMax(&s_rows[c.tile], c.row + 1);
            s_weight[lane] = a.weights[lane];
        }
    }
    float* const sums = reinterpret_cast<float*>(s_mem) + wave * M * 16;
    for (int i = lane; i < M * 16; i += 64) sums[i] = 0.0f;
    __syncthreads();

    const int all = c.tiles * n_kt, begin = all * wave / 8, end = all * (wave + 1) / 8;
    const int64_t cb = blockIdx.x;
    const char* const codes = (const char*)a.e.down + cb * n_kt * 1024 + lane * 16;
    const char* const scales = (const char*)a.e.down + a.down.codes_bytes + cb * n_kt * 32 * GPT + col * 2 * GPT;
    const int in_row = (4 * (q & 1) + (q >> 1)) * 16 + (col >> 3) * 128;
    const int lo_exp = (col >> 3) * 0x0505;
    constexpr int L = 4;                // (fewer for fewer rows: three times the code, and no faster)
    const int nth = row_of_lane<L>(col);
    struct Slot {
        v4i w, x[4];
        typename Scales<GPT>::type sc;
        int e;
    } slot[TINY_W];
    // the next step to load, its tile and what is its own
    int next = begin, tile_l = begin / n_kt, kt_l = begin - tile_l * n_kt;
    const char *codes_l = codes, *scales_l = scales, *x_l = hs, *e_l = he;
    auto enter = [&]() {                // tile_l's weights and rows
        const int expert = __builtin_amdgcn_readfirstlane(s_expert[tile_l]), row = s_row[tile_l][min(nth, s_rows[tile_l] - 1)];
        codes_l = codes + expert * a.e.down_stride;
        scales_l = scales + expert * a.e.down_stride;
        x_l = hs + row * moe::row_bytes(a.e.inter) + in_row;
        e_l = he + row * moe::exp_bytes(a.e.inter) + q * 2;
    };
    auto load = [&](Slot& t) {
        if (next < end) {
            t.w = __builtin_nontemporal_load(reinterpret_cast<const v4i*>(codes_l + (int64_t)kt_l * 1024));
            t.sc = *reinterpret_cast<const typename Scales<GPT>::type*>(scales_l + kt_l * 32 * GPT);
#pragma unroll
            for (int j = 0; j < 4; ++j) t.x[j] = *reinterpret_cast<const v4i*>(x_l + kt_l * 512 + j / 2 * 256 + j % 2 * 32);
            t.e = load_exponents(e_l + kt_l * 8);
            if (++next < end && ++kt_l == n_kt) {
                kt_l = 0;
                ++tile_l;
                enter();
            }
        }
    };
    if (begin < end) enter();
#pragma unroll
    for (int i = 0; i < TINY_W; ++i) load(slot[i]);
    float y[L] = {};
    int tile = begin / n_kt, left = n_kt - (begin - tile * n_kt);
    for (int s = begin; s < end; s += TINY_W) {
#pragma unroll
        for (int i = 0; i < TINY_W; ++i) {
            if (s + i < end) {
                const int e = slot[i].e - lo_exp;
                multiply<GPT, 0>(join(slot[i].x[0], slot[i].x[1]), e, slot[i].w, slot[i].sc, y);
                multiply<GPT, 1>(join(slot[i].x[2], slot[i].x[3]), e, slot[i].w, slot[i].sc, y);
                load(slot[i]);
                if (--left == 0 || s + i + 1 == end) {   // the tile's rows, or the wave's share of them
#pragma unroll
                    for (int r = 0; r < L; ++r) y[r] += __shfl_xor(y[r], 32);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {        // the rows of a lane group and only then the next one's: two may be one row of Y
                        if (q == h) {
#pragma unroll
                            for (int r = 0; r < L; ++r)
                                if (h * L + r < s_rows[tile]) {
                                    const int at = s_row[tile][h * L + r];
                                    sums[at / a.top_k * 16 + col] += s_weight[at] * y[r];
                                }
                        }
                        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                        __builtin_amdgcn_wave_barrier();
                    }
#pragma unroll
                    for (int r = 0; r < L; ++r) y[r] = 0.0f;
                    ++tile;
                    left = n_kt;
                }
            }
        }
    }
    __syncthreads();
    for (int i = tid; i < M * 16; i += 512) {
        const int64_t m = i / 16, n = cb * 16 + i % 16;
        float t = a.base ? __uint_as_float((uint32_t)a.base[m * a.ldb + n] << 16) : 0.0f;
#pragma unroll
        for (int v = 0; v < 8; ++v) t += reinterpret_cast<const float*>(s_mem)[v * M * 16 + i];
        a.Y[m * a.ldy + n] = (uint16_t)pack_bf16(t, t);
    }
}

// Y = base + the weighted rows of z, in the order of the slots; four rows of z under way together.  Memory: 16384 rows of 2048 22 us, 6 TB/s; few rows:
// latency, 4.7 us.  z is in fp32: in fp16 beside a power of two for 32 columns this launch took 14 us there (and the call 3 % less, while 1806 rows
// took 3 % more), and two experts that nearly cancel left 0.04 of their difference wrong.
__global__ void __launch_bounds__(256) moe_combine_kernel(ExpertsArgs a, const int* place, const float* z)
{
    const int64_t m = blockIdx.x;
    const int n = (blockIdx.y * 256 + threadIdx.x) * 8;
    if (n >= a.e.hidden) return;
    float y[8] = {};
    if (a.base) {
        const uint4 b = *reinterpret_cast<const uint4*>(a.base + m * a.ldb + n);
        const uint32_t d[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[2 * i] = __uint_as_float(d[i] << 16);
            y[2 * i + 1] = __uint_as_float(d[i] & 0xffff0000u);
        }
    }
    for (int j = 0; j < a.top_k; j += 4) {
        int at[4];
        float w[4];
        float4 p[4], q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] = j + i < a.top_k ? place[m * a.top_k + j + i] : -1;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (at[i] >= 0) {
                w[i] = a.weights[m * a.top_k + j + i];
                const float4* const t = reinterpret_cast<const float4*>(z + (int64_t)at[i] * a.e.hidden + n);
                p[i] = t[0];
                q[i] = t[1];
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (at[i] < 0) continue;
            y[0] = fmaf(w[i], p[i].x, y[0]); y[1] = fmaf(w[i], p[i].y, y[1]); y[2] = fmaf(w[i], p[i].z, y[2]); y[3] = fmaf(w[i], p[i].w, y[3]);
            y[4] = fmaf(w[i], q[i].x, y[4]); y[5] = fmaf(w[i], q[i].y, y[5]); y[6] = fmaf(w[i], q[i].z, y[6]); y[7] = fmaf(w[i], q[i].w, y[7]);
        }
    }
    *reinterpret_cast<uint4*>(a.Y + m * a.ldy + n) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
}

template <bool UP, int KS, int GPT>
int launch_few(const ProductArgs& a, int64_t tiles, int64_t row_bytes_all, hipStream_t stream)
{
    typedef FewShape<KS> S;
    auto* const kern = moe_few_kernel<UP, KS, GPT>;
    const int rc = ensure_dynamic_lds((const void*)kern, S::LDS, "w2_moe_experts");
    if (rc) return rc;
    const int pairs = UP ? a.n_out / 16 : a.n_out / 32;
    hipLaunchKernelGGL(kern, dim3((unsigned)(pairs / S::P), (unsigned)tiles), dim3(S::THREADS), S::LDS, stream, a, row_bytes_all);
    return 0;
}

template <bool UP, int GPT>
int launch_product(const ProductArgs& a, const moe::Plan& p, int64_t row_bytes_all, const int* n_tiles, hipStream_t stream)
{
    if (!p.few) {
        const int groups = UP ? a.n_out / 128 : a.n_out / 256;
        hipLaunchKernelGGL((moe_tile_kernel<UP, GPT>), dim3((unsigned)((p.tiles * groups + 7) / 8 * 8)), dim3(256), 0, stream, a, row_bytes_all, n_tiles, groups);
        return 0;
    }
    return (UP ? p.ks_up : p.ks_down) == 1 ? launch_few<UP, 1, GPT>(a, p.tiles, row_bytes_all, stream) : launch_few<UP, 2, GPT>(a, p.tiles, row_bytes_all, stream);
}

}  // namespace

size_t experts_workspace_bytes(const w2_experts_t& e, int64_t M, int top_k)
{
    return moe::workspace(e.hidden, e.inter, e.n_experts, e.G, M, top_k).total;
}

namespace {

template <int GPT>
int launch_tiny(const ExpertsArgs& a, const moe::Tiny& t, char* hs, char* he, hipStream_t stream)
{
    const int rc = ensure_dynamic_lds((const void*)moe_tiny_up_kernel<GPT>, t.lds_all, "w2_moe_experts");
    if (rc) return rc;
    hipLaunchKernelGGL((moe_tiny_up_kernel<GPT>), dim3((unsigned)(a.e.inter / 16 / moe::TINY_P / t.units), (unsigned)t.tiles), dim3(512), t.lds_all, stream, a, hs,
                       he, t.units, t.rows);
    hipLaunchKernelGGL((moe_tiny_down_kernel<GPT>), dim3((unsigned)(a.e.hidden / 16)), dim3(512), (size_t)a.M * 512, stream, a, (const char*)hs,
                       (const char*)he);
    return check_launch("w2_moe_experts");
}

}  // namespace

int launch_moe_experts(const ExpertsArgs& all, hipStream_t stream)
{
    const int64_t most = moe::most_rows(all.e.hidden, all.e.inter, all.top_k);
    if (all.M > most) {                 // rows by rows
        ExpertsArgs part = all;
        for (int64_t m = 0; m < all.M; m += most) {
            part.M = std::min(most, all.M - m);
            part.x = all.x + m * all.ldx;
            part.ids = all.ids + m * all.top_k;
            part.weights = all.weights + m * all.top_k;
            if (all.base) part.base = all.base + m * all.ldb;
            part.Y = all.Y + m * all.ldy;
            const int rc = launch_moe_experts(part, stream);
            if (rc) return rc;
        }
        return 0;
    }
    const ExpertsArgs& a = all;
    const int64_t A = a.M * a.top_k, hidden = a.e.hidden, inter = a.e.inter;
    const moe::Workspace ws = moe::workspace(hidden, inter, a.e.n_experts, a.e.G, a.M, a.top_k);
    char* const w = (char*)a.workspace;
    const moe::Tiny tiny = moe::tiny(hidden, inter, a.e.n_experts, a.e.G, A);
    if (tiny.fits) return a.e.G == 128 ? launch_tiny<2>(a, tiny, w + ws.hs, w + ws.he, stream) : launch_tiny<4>(a, tiny, w + ws.hs, w + ws.he, stream);
    const moe::Plan plan = moe::plan(hidden, inter, a.e.n_experts, a.e.G, A);
    int* const n_tiles = (int*)(w + ws.tiles);
    Tile* const tile = (Tile*)(w + ws.tiles + 256);
    int* const tile_rows = (int*)(w + ws.tile_rows);
    int* const place = (int*)(w + ws.place);
    const int64_t convert = (a.M * (hidden / 32) + 1023) / 1024;
    hipLaunchKernelGGL(moe_prepare_kernel, dim3((unsigned)(1 + convert)), dim3(1024), 0, stream, a, n_tiles, tile, plan.tiles, plan.few ? 3 : 5,
                       make_divider((uint32_t)a.top_k), tile_rows, place, w + ws.xs, w + ws.xe);
    ProductArgs u = {};
    u.blob = (const char*)a.e.gate_up; u.blob_stride = a.e.gate_up_stride; u.codes_bytes = (int64_t)a.up.codes_bytes;
    u.n_kt = (int)(hidden / 256); u.tiles = tile; u.tile_rows = tile_rows;
    u.rows = w + ws.xs; u.exps = w + ws.xe; u.h = w + ws.hs; u.h_exps = w + ws.he; u.n_out = (int)inter;
    ProductArgs d = {};
    d.blob = (const char*)a.e.down; d.blob_stride = a.e.down_stride; d.codes_bytes = (int64_t)a.down.codes_bytes;
    d.n_kt = (int)(inter / 256); d.tiles = tile; d.rows = w + ws.hs; d.exps = w + ws.he; d.z = (float*)(w + ws.z); d.n_out = (int)hidden;
    const int64_t x_bytes = a.M * (int64_t)moe::row_bytes(hidden), h_bytes = A * (int64_t)moe::row_bytes(inter);
    int rc;
    if (a.e.G == 128) {
        if ((rc = launch_product<true, 2>(u, plan, x_bytes, n_tiles, stream))) return rc;
        if ((rc = launch_product<false, 2>(d, plan, h_bytes, n_tiles, stream))) return rc;
    } else {
        if ((rc = launch_product<true, 4>(u, plan, x_bytes, n_tiles, stream))) return rc;
        if ((rc = launch_product<false, 4>(d, plan, h_bytes, n_tiles, stream))) return rc;
    }
    hipLaunchKernelGGL(moe_combine_kernel, dim3((unsigned)a.M, (unsigned)((hidden + 2047) / 2048)), dim3(256), 0, stream, a, (const int*)place,
                       (const float*)d.z);
    return check_launch("w2_moe_experts");
}

}  // namespace w2
