// Rows through their 2-bit experts: gate and up projection, silu(gate) * up, down projection, sum over a row's experts.
//
// The matrix instruction is the one for eight-bit rows and four-bit columns (16 x 16 x 128, E4M3 x E2M1, a power of two for every 32 k of
// a row): a 2-bit weight -2, -1, 0, 1 IS a four-bit number (-1, -0.5, 0, 0.5 with the column's power of two at 2), seven
// instructions turn 16 of them out of a packed dword, and a row's numbers are the sum of two eight-bit ones: E4M3 has four
// significant bits and bf16 eight, so hi = round(x), lo = round(x - hi) is exact wherever lo's exponent reaches, which is down
// to 2^-14 of the largest of the 32 numbers that share a power of two (off by 2^-22 of it below).  Against bf16 instructions
// that is a third of the vector work per weight, and the products of hi and of lo together take no longer than one bf16
// product (4300 TFLOP/s for both formats of eight and four bits, measured; half that for the pair).  What the instruction gives
// away: of 8 neighbouring products, bits 13 places below the largest one's exponent are cut off.
//
// Rows in memory ("xs", "hs"): for every 256 k [2 halves of 128 k][hi, lo][8 units][16 bytes], a unit being 16 k in the order in which
// the up-convert leaves the weights' nibbles, 0 8 1 9 2 10 3 11 4 12 5 13 6 14 7 15; exponents [4 g][2 halves] bytes beside
// them, g = the units g and g + 4 of a half, which is one lane group's 32 k of the instruction.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "block_ops.h"
#include "ffn_ops.h"
#include "moe_plan.h"

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

// ---------------------------------------------------------------- before the products: who goes where, and x in two parts

// Workgroup 0 sorts the choices by expert (stable: which rows share a tile is the same every time); the others convert x, a
// thread 32 numbers.
__global__ void __launch_bounds__(1024) moe_prepare_kernel(ExpertsArgs a, Tile* tiles, int64_t max_tiles, int rows, int* sorted, int* place,
                                                           char* xs, char* xe)
{
    __shared__ int s_count[16][1024];   // of each wave's share, then where its rows of each expert begin
    __shared__ int s_sum[2][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int E = a.e.n_experts;
    if (blockIdx.x > 0) {
        const int64_t blocks = a.e.hidden / 32, i = (int64_t)(blockIdx.x - 1) * 1024 + tid;
        if (i >= a.M * blocks) return;
        const int64_t m = i / blocks, b = i - m * blocks;
        const int64_t kt = b / 8;
        const int half = (int)(b & 7) >> 2, g = (int)(b & 3);
        const uint16_t* src = a.x + m * a.ldx + kt * 256 + half * 128 + g * 16;
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
        char* dst = xs + m * moe::row_bytes(a.e.hidden) + kt * 512 + half * 256 + g * 16;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uint32_t hi[8], lo[8];
            // numbers n and n + 8 of the unit are neighbours
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                const uint32_t lw = d[u][n / 2], hw = d[u][4 + n / 2];
                const float p = __uint_as_float(n & 1 ? lw & 0xffff0000u : lw << 16), q = __uint_as_float(n & 1 ? hw & 0xffff0000u : hw << 16);
                split2(p, q, f, hi[n], lo[n]);
            }
            *reinterpret_cast<uint4*>(dst + u * 64) = make_uint4(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16, hi[4] | hi[5] << 16, hi[6] | hi[7] << 16);
            *reinterpret_cast<uint4*>(dst + u * 64 + 128) = make_uint4(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16, lo[4] | lo[5] << 16, lo[6] | lo[7] << 16);
        }
        xe[m * moe::exp_bytes(a.e.hidden) + kt * 8 + g * 2 + half] = (char)e;
        return;
    }
    const int A = (int)(a.M * a.top_k);
    for (int i = tid; i < 16 * 1024; i += 1024) (&s_count[0][0])[i] = 0;
    __syncthreads();
    const int share = (A + 1023) / 1024 * 64, begin = min(A, wave * share), end = min(A, begin + share);
    for (int i = begin + lane; i < end; i += 64) {
        const int id = a.ids[i];
        if ((unsigned)id < (unsigned)E) atomicAdd(&s_count[wave][id], 1);
    }
    __syncthreads();
    // thread e: expert e's rows, and where they and its tiles begin
    int count = 0;
    for (int w = 0; w < 16; ++w) count += s_count[w][tid];
    const int n_tiles = (count + rows - 1) / rows;
    int first = count, tile = n_tiles;                       // inclusive sums over the experts
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
    for (int t = 0; t < n_tiles; ++t) tiles[tile + t] = Tile{tid, first + t * rows, min(rows, count - t * rows), 0};
    for (int64_t t = all_tiles + tid; t < max_tiles; t += 1024) tiles[t] = Tile{0, 0, 0, 0};
    for (int w = 0; w < 16; ++w) {
        const int n = s_count[w][tid];
        s_count[w][tid] = first;
        first += n;
    }
    __syncthreads();
    for (int i0 = begin; i0 < end; i0 += 64) {
        const int i = i0 + lane;
        const int id = i < end ? a.ids[i] : -1;
        const bool live = (unsigned)id < (unsigned)E;
        uint64_t same = __ballot(live);
        for (int b = 0; b < 10; ++b) {
            const uint64_t set = __ballot(live && id >> b & 1);
            same &= id >> b & 1 ? set : ~set;
        }
        const int before = __popcll(same & (((uint64_t)1 << lane) - 1));
        const int at = live ? s_count[wave][id] : 0;
        if (live) {
            sorted[at + before] = i;
            if (before == 0) s_count[wave][id] = at + __popcll(same);
        }
        if (i < end) place[i] = live ? at + before : -1;
    }
}

// ---------------------------------------------------------------- the products

// 16 weights of a dword -> 16 four-bit numbers of the values q / 2: [0] the fields 0 and 2 of each byte, [1] 1 and 3.  q in two's complement
// (b1 b0): sign b1, magnitude b0 | (b1 & ~b0) << 1.
__device__ __forceinline__ void to_fp4(uint32_t w, int& lo, int& hi)
{
    const uint32_t t = w << 1;
    const uint32_t mag = w & ~(t & 0xaaaaaaaau);             // magnitudes in place
    const uint32_t sign = w & 0xaaaaaaaau;
    lo = (int)((mag & 0x33333333u) | (sign << 2 & 0xccccccccu));
    hi = (int)((mag >> 2 & 0x33333333u) | (sign & 0xccccccccu));
}

constexpr int STRIDE = 528;             // bytes of a row's 256 k in local memory: 512, its exponents, and 4 banks on to the next row

struct ProductArgs {
    const char* blob;
    int64_t blob_stride, codes_bytes;
    int n_kt;
    const Tile* tiles;
    const int* sorted;                  // up: whose rows; down: nullptr, rows lie in sorted order
    int top_k;
    const char *rows, *exps;            // in two parts
    char *h, *h_exps;                   // up: rows of n_out numbers in two parts
    float* z;                           // down: rows of n_out numbers
    int n_out;
};

// A workgroup: eight waves = 8 / KS pairs of column blocks times KS ranges of K, up to 16 * RT rows of one expert.  UP: a pair
// is a block of gate columns and one of up columns; silu(gate) * up leaves in two parts.  Not UP: two blocks; sums leave in fp32.
template <bool UP, int RT, int KS, int GPT>
__global__ void __launch_bounds__(512) moe_product_kernel(ProductArgs a)
{
    constexpr int R = 16 * RT, P = 8 / KS, NP = RT * KS;
    extern __shared__ char s_mem[];                          // [2 buffers][KS][R][STRIDE]
    __shared__ int s_src[R];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, q = lane >> 4;
    const Tile tile = a.tiles[blockIdx.y];
    if (tile.rows == 0) return;
    // pairs of a workgroup lie so that the units g and g + 4 of 128 numbers of h are both its own
    const int p = wave % P, kr = wave / P;
    int pair;
    if (UP) pair = blockIdx.x / KS * 8 + blockIdx.x % KS * (P / 2) + p % (P / 2) + p / (P / 2) * 4;
    else pair = blockIdx.x * P + p;
    const int steps = (a.n_kt + KS - 1) / KS;
    const char* const blob = a.blob + tile.expert * a.blob_stride;

    // weights of the wave's column blocks, from its first k tile on
    const int kt0 = kr * steps, my_steps = max(0, min(steps, a.n_kt - kt0));
    const char* codes[2];
    const char* scales[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int64_t t = (int64_t)(2 * pair + c) * a.n_kt + kt0;
        codes[c] = blob + t * 1024 + lane * 16;
        scales[c] = blob + a.codes_bytes + (t * 16 + col) * GPT * 2;
    }
    typedef typename std::conditional<GPT == 2, uint32_t, uint2>::type Scales;
    uint4 w[2];
    Scales sc[2];
    auto load_weights = [&](int s) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            w[c] = *reinterpret_cast<const uint4*>(codes[c] + (int64_t)s * 1024);
            sc[c] = *reinterpret_cast<const Scales*>(scales[c] + (int64_t)s * 32 * GPT);
        }
    };
    if (my_steps > 0) load_weights(0);

    if (tid < R) {
        const int r = min(tid, tile.rows - 1);
        s_src[tid] = UP ? a.sorted[tile.first + r] / a.top_k : tile.first + r;
    }
    __syncthreads();
    const char *src[NP], *src_e = nullptr;
    int kt_of[NP], to[NP];
    const int row_b = a.n_kt * 512;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int piece = tid + i * 512, r = piece / 32 % R, k = piece / (32 * R);
        src[i] = a.rows + (int64_t)s_src[r] * row_b + (int64_t)k * steps * 512 + piece % 32 * 16;
        kt_of[i] = k * steps;
        to[i] = (k * R + r) * STRIDE + piece % 32 * 16;
    }
    int kt_e = 0, to_e = 0;
    if (tid < R * KS) {
        src_e = a.exps + (int64_t)s_src[tid % R] * a.n_kt * 8 + (int64_t)(tid / R) * steps * 8;
        kt_e = tid / R * steps;
        to_e = tid * STRIDE + 512;
    }
    uint4 staged[NP];
    uint2 staged_e = make_uint2(0, 0);
    auto fetch = [&](int s) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            staged[i] = make_uint4(0, 0, 0, 0);
            if (kt_of[i] + s < a.n_kt) staged[i] = *reinterpret_cast<const uint4*>(src[i] + s * 512);
        }
        if (src_e && kt_e + s < a.n_kt) staged_e = *reinterpret_cast<const uint2*>(src_e + s * 8);
    };
    auto put = [&](int buffer) {
        char* const at = s_mem + buffer * (KS * R * STRIDE);
#pragma unroll
        for (int i = 0; i < NP; ++i) *reinterpret_cast<uint4*>(at + to[i]) = staged[i];
        if (src_e) *reinterpret_cast<uint2*>(at + to_e) = staged_e;
    };
    fetch(0);
    put(0);
    __syncthreads();

    v4f y[RT][2] = {};
    const bool packed = RT == 1 && tile.rows <= 8;           // hi in rows 0 to 7 of the instruction, lo in 8 to 15
    const int row = packed ? col & 7 : col;
    const int unit = 4 * (q & 1) + (q >> 1);
    for (int s = 0; s < steps; ++s) {
        if (s + 1 < steps) fetch(s + 1);
        if (s < my_steps) {
            uint4 now[2] = {w[0], w[1]};
            Scales f[2] = {sc[0], sc[1]};
            if (s + 1 < my_steps) load_weights(s + 1);
            const char* const at = s_mem + (s & 1) * (KS * R * STRIDE) + kr * R * STRIDE;
            int e[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) e[r] = *reinterpret_cast<const uint16_t*>(at + (r * 16 + row) * STRIDE + 512 + q * 2);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                int b[2][4];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    to_fp4(j ? now[c].z : now[c].x, b[c][0], b[c][1]);
                    to_fp4(j ? now[c].w : now[c].y, b[c][2], b[c][3]);
                }
                auto group = [&](int c, int g) -> float {   // scale of group g of this column's 256 k
                    uint32_t d;
                    if constexpr (GPT == 2) d = f[c];
                    else d = g < 2 ? f[c].x : f[c].y;
                    return __uint_as_float(g & 1 ? d & 0xffff0000u : d << 16);
                };
                auto part = [&](int r, int lo) -> v8i {
                    const char* t = at + (r * 16 + row) * STRIDE + j * 256 + lo * 128 + unit * 16;
                    const v4i x = *reinterpret_cast<const v4i*>(t), z = *reinterpret_cast<const v4i*>(t + 32);
                    return (v8i){x[0], x[1], x[2], x[3], z[0], z[1], z[2], z[3]};
                };
                auto mul = [&](v8i x, v8i b8, v4f acc, int ex) -> v4f {
                    // format 0: E4M3 rows, 4: E2M1 columns; the column's power of two, 2^1, makes q of q / 2
                    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, b8, acc, 0, 4, 0, ex, 0, 128);
                };
                if (packed) {
                    const int ex = ((e[0] >> (8 * j)) & 255) - (col >> 3) * 5;
                    const v8i x = part(0, col >> 3);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        if constexpr (GPT == 2) {
                            const v4f acc = mul(x, (v8i){b[c][0], b[c][1], b[c][2], b[c][3], 0, 0, 0, 0}, (v4f){0, 0, 0, 0}, ex);
                            y[0][c] += acc * group(c, j);
                        } else {
                            const v4f a0 = mul(x, (v8i){b[c][0], b[c][1], 0, 0, 0, 0, 0, 0}, (v4f){0, 0, 0, 0}, ex);
                            const v4f a1 = mul(x, (v8i){0, 0, b[c][2], b[c][3], 0, 0, 0, 0}, (v4f){0, 0, 0, 0}, ex);
                            y[0][c] += a0 * group(c, 2 * j);
                            y[0][c] += a1 * group(c, 2 * j + 1);
                        }
                    }
                } else {
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        const int ex = (e[r] >> (8 * j)) & 255;
                        const v8i hi = part(r, 0), lo = part(r, 1);
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            if constexpr (GPT == 2) {
                                const v8i b8 = {b[c][0], b[c][1], b[c][2], b[c][3], 0, 0, 0, 0};
                                v4f acc = mul(lo, b8, (v4f){0, 0, 0, 0}, ex - 5);
                                acc = mul(hi, b8, acc, ex);
                                y[r][c] += acc * group(c, j);
                            } else {
                                const v8i b0 = {b[c][0], b[c][1], 0, 0, 0, 0, 0, 0}, b1 = {0, 0, b[c][2], b[c][3], 0, 0, 0, 0};
                                v4f a0 = mul(lo, b0, (v4f){0, 0, 0, 0}, ex - 5), a1 = mul(lo, b1, (v4f){0, 0, 0, 0}, ex - 5);
                                a0 = mul(hi, b0, a0, ex);
                                a1 = mul(hi, b1, a1, ex);
                                y[r][c] += a0 * group(c, 2 * j);
                                y[r][c] += a1 * group(c, 2 * j + 1);
                            }
                        }
                    }
                }
            }
        }
        if (s + 1 < steps) put((s + 1) & 1);
        __syncthreads();
    }
    if (packed) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[0][c][i] += __shfl_xor(y[0][c][i], 32);
    }
    // ranges of K meet in local memory, in their order
    if constexpr (KS > 1) {
        v4f* const part = reinterpret_cast<v4f*>(s_mem);     // [KS - 1][P][RT * 2][64]
        if (kr > 0) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int c = 0; c < 2; ++c) part[(((kr - 1) * P + p) * RT * 2 + r * 2 + c) * 64 + lane] = y[r][c];
        }
        __syncthreads();
        if (kr == 0) {
            for (int k = 0; k < KS - 1; ++k)
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int c = 0; c < 2; ++c) y[r][c] += part[((k * P + p) * RT * 2 + r * 2 + c) * 64 + lane];
        }
        __syncthreads();
    }
    if constexpr (!UP) {
        if (kr > 0) return;
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int m = r * 16 + q * 4 + i;
                if (m < tile.rows) {
                    float* const out = a.z + (int64_t)(tile.first + m) * a.n_out + pair * 32 + col;
                    out[0] = y[r][0][i];
                    out[16] = y[r][1][i];
                }
            }
    } else {
        float* const s_top = reinterpret_cast<float*>(s_mem);          // [P][R]: the largest |h| of a row's unit
        char* const s_out = s_mem + P * R * 4;                         // [R][2 parts][P units][16]
        float h[RT][4];
        if (kr == 0) {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float g = y[r][0][i];
                    h[r][i] = g / (1.0f + __expf(-g)) * y[r][1][i];
                    float m = fabsf(h[r][i]);
                    if (!(m < INFINITY)) m = INFINITY;       // a NaN counts as the largest exponent
                    m = fmaxf(m, dpp_move_f32<0xB1>(m));
                    m = fmaxf(m, dpp_move_f32<0x4E>(m));
                    m = fmaxf(m, dpp_move_f32<0x141>(m));
                    m = fmaxf(m, dpp_move_f32<0x140>(m));
                    if (col == 0) s_top[p * R + r * 16 + q * 4 + i] = m;
                }
        }
        __syncthreads();
        const int u = blockIdx.x / KS, c0 = blockIdx.x % KS * (P / 2);     // 128 numbers of h, the first of the units here
        if (kr == 0) {
            const int slot = col & 7, byte = 2 * slot + (col >> 3);
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int m = r * 16 + q * 4 + i;
                    const float top = fmaxf(s_top[p % (P / 2) * R + m], s_top[(p % (P / 2) + P / 2) * R + m]);
                    const int ex = shared_exponent((int)(__float_as_uint(top) >> 23));
                    uint32_t hi, lo;
                    split2(h[r][i], 0.0f, scale_down(ex), hi, lo);
                    s_out[((m * 2 + 0) * P + p) * 16 + byte] = (char)hi;
                    s_out[((m * 2 + 1) * P + p) * 16 + byte] = (char)lo;
                    if (p < P / 2 && col == 0 && m < tile.rows)
                        a.h_exps[(int64_t)(tile.first + m) * (a.n_out / 32) + u / 2 * 8 + (c0 + p) * 2 + (u & 1)] = (char)ex;
                }
        }
        __syncthreads();
        for (int i = tid; i < R * 2 * P; i += 512) {         // 16 bytes: a unit of a part of a row
            const int m = i / (2 * P), part = i / P % 2, pp = i % P;
            if (m < tile.rows) {
                const int to_unit = c0 + pp % (P / 2) + pp / (P / 2) * 4;
                *reinterpret_cast<uint4*>(a.h + (int64_t)(tile.first + m) * a.n_out * 2 + u * 256 + part * 128 + to_unit * 16) =
                    *reinterpret_cast<const uint4*>(s_out + i * 16);
            }
        }
    }
}

// Y = base + the weighted rows of z, in the order of the slots
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
    for (int j = 0; j < a.top_k; ++j) {
        const int at = place[m * a.top_k + j];
        if (at < 0) continue;
        const float w = a.weights[m * a.top_k + j];
        const float4* t = reinterpret_cast<const float4*>(z + (int64_t)at * a.e.hidden + n);
        const float4 p = t[0], q = t[1];
        y[0] = fmaf(w, p.x, y[0]); y[1] = fmaf(w, p.y, y[1]); y[2] = fmaf(w, p.z, y[2]); y[3] = fmaf(w, p.w, y[3]);
        y[4] = fmaf(w, q.x, y[4]); y[5] = fmaf(w, q.y, y[5]); y[6] = fmaf(w, q.z, y[6]); y[7] = fmaf(w, q.w, y[7]);
    }
    *reinterpret_cast<uint4*>(a.Y + m * a.ldy + n) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
}

template <bool UP, int RT, int KS, int GPT>
int launch_product(const ProductArgs& a, int64_t tiles, hipStream_t stream)
{
    constexpr int P = 8 / KS;
    const size_t lds = (size_t)2 * KS * 16 * RT * STRIDE;
    auto* const kern = moe_product_kernel<UP, RT, KS, GPT>;
    const int rc = ensure_dynamic_lds((const void*)kern, lds, "w2_moe_experts");
    if (rc) return rc;
    const int pairs = UP ? a.n_out / 16 : a.n_out / 32;
    ProductArgs b = a;
    for (int64_t t = 0; t < tiles; t += 65535) {             // what a grid's y takes
        b.tiles = a.tiles + t;
        hipLaunchKernelGGL(kern, dim3((unsigned)(pairs / P), (unsigned)std::min<int64_t>(tiles - t, 65535)), dim3(512), lds, stream, b);
    }
    return 0;
}

template <bool UP, int GPT>
int launch_shape(const ProductArgs& a, int rt, int ks, int64_t tiles, hipStream_t stream)
{
    if (rt == 1) return ks == 1 ? launch_product<UP, 1, 1, GPT>(a, tiles, stream) : ks == 2 ? launch_product<UP, 1, 2, GPT>(a, tiles, stream)
                                                                                            : launch_product<UP, 1, 4, GPT>(a, tiles, stream);
    if (rt == 2) return ks == 1 ? launch_product<UP, 2, 1, GPT>(a, tiles, stream) : launch_product<UP, 2, 2, GPT>(a, tiles, stream);
    return launch_product<UP, 4, 1, GPT>(a, tiles, stream);
}

}  // namespace

size_t experts_workspace_bytes(const w2_experts_t& e, int64_t M, int top_k)
{
    return moe::workspace(e.hidden, e.inter, e.n_experts, M, top_k).total;
}

int launch_moe_experts(const ExpertsArgs& a, hipStream_t stream)
{
    const int64_t A = a.M * a.top_k, hidden = a.e.hidden, inter = a.e.inter;
    const moe::Workspace ws = moe::workspace(hidden, inter, a.e.n_experts, a.M, a.top_k);
    char* const w = (char*)a.workspace;
    const int rt = moe::pick_rt(A, a.e.n_experts);
    const int64_t tiles = moe::most_tiles(A, a.e.n_experts, 16 * rt);
    Tile* const tile = (Tile*)(w + ws.tiles);
    int* const sorted = (int*)(w + ws.sorted);
    int* const place = (int*)(w + ws.place);
    const int64_t convert = (a.M * (hidden / 32) + 1023) / 1024;
    hipLaunchKernelGGL(moe_prepare_kernel, dim3((unsigned)(1 + convert)), dim3(1024), 0, stream, a, tile, tiles, 16 * rt, sorted, place,
                       w + ws.xs, w + ws.xe);
    ProductArgs u = {};
    u.blob = (const char*)a.e.gate_up; u.blob_stride = a.e.gate_up_stride; u.codes_bytes = (int64_t)a.up.codes_bytes;
    u.n_kt = (int)(hidden / 256); u.tiles = tile; u.sorted = sorted; u.top_k = a.top_k;
    u.rows = w + ws.xs; u.exps = w + ws.xe; u.h = w + ws.hs; u.h_exps = w + ws.he; u.n_out = (int)inter;
    ProductArgs d = {};
    d.blob = (const char*)a.e.down; d.blob_stride = a.e.down_stride; d.codes_bytes = (int64_t)a.down.codes_bytes;
    d.n_kt = (int)(inter / 256); d.tiles = tile; d.rows = w + ws.hs; d.exps = w + ws.he; d.z = (float*)(w + ws.z); d.n_out = (int)hidden;
    const int ks_u = moe::pick_ks(rt, tiles * (inter / 128), u.n_kt), ks_d = moe::pick_ks(rt, tiles * (hidden / 256), d.n_kt);
    int rc;
    if (a.e.G == 128) {
        if ((rc = launch_shape<true, 2>(u, rt, ks_u, tiles, stream))) return rc;
        if ((rc = launch_shape<false, 2>(d, rt, ks_d, tiles, stream))) return rc;
    } else {
        if ((rc = launch_shape<true, 4>(u, rt, ks_u, tiles, stream))) return rc;
        if ((rc = launch_shape<false, 4>(d, rt, ks_d, tiles, stream))) return rc;
    }
    hipLaunchKernelGGL(moe_combine_kernel, dim3((unsigned)a.M, (unsigned)((hidden + 2047) / 2048)), dim3(256), 0, stream, a, (const int*)place,
                       (const float*)(w + ws.z));
    return check_launch("w2_moe_experts");
}

}  // namespace w2
