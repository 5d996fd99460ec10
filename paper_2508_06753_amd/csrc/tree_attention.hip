// Attention of each request's drafted tokens over its pages of the cache.
//
// The query rows of a cache head are packed, row rho = (token i) * G + (query head g), so that a group's heads share what
// is read of K and V.  Scores are held transposed: S^T = K Q^T by 16x16x32 matrix instructions puts 4 keys of one query row
// in a lane, which is the operand layout of P^T in O^T = V^T P^T once the 32 keys of a step are numbered as (tile 0, 4q + i),
// (tile 1, 4q + i), q = lane / 16: no weight crosses lanes.  V^T operands come from local memory by the transposing read.
// Running maximum and sum per query row (m, l) in fp32; the outputs are rescaled only when a maximum has grown by more than
// 8 powers of two, which fp32 sums and bf16 weights carry without loss; the sum is reduced over the lanes at the end.
//
// tree_few_kernel: up to 32 packed rows (decoding, small trees).  Every wave of a workgroup takes other keys.
// tree_tile_kernel: workgroups of 64 or 128 packed rows, 16 or 32 a wave, over shared stages of K and V.
// Keys of a request are cut into chunks for several workgroups where the batch alone does not fill the machine; partial
// results meet in tree_join_kernel.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "block_ops.h"

namespace w2 {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.4426950408889634f;
constexpr float SLACK = 8.0f;            // powers of two a maximum may grow by before the outputs are rescaled
constexpr int MAX_CHUNKS = 128;

__device__ __align__(16) const uint32_t g_zeros[4] = {0, 0, 0, 0};

__device__ __forceinline__ v4f mfma(const v4i& a, const v4i& b, const v4f& c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

// two floats to bf16, round to nearest even
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    typedef float v2f __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f){lo, hi}, v2bf));
}

// 16-byte pieces of a row of DT numbers are stored XORed by this, so that 16 rows at one piece lie in 16 different places
// of the 256 bytes that local memory delivers at once
template <int DT>
__device__ __forceinline__ int swizzle(int key) { return DT == 64 ? (key >> 1) & 7 : key & 15; }

struct Plan {
    int few;                             // tree_few_kernel, else tree_tile_kernel
    int rt;                              // 16-row tiles a wave
    int dt;                              // head_dim padded to 64, 128 or 256
    int tiles;                           // row tiles of a request
    int chunk;                           // keys of a workgroup, a multiple of 32 * waves
    int chunks;                          // of the longest request
};

Plan make_plan(int64_t n_requests, int64_t max_rows, int G, int n_kv, int D, int64_t max_len, int64_t total_len)
{
    Plan p;
    const int64_t rows = max_rows * G;
    p.dt = D <= 64 ? 64 : D <= 128 ? 128 : 256;
    p.few = rows <= (p.dt < 256 ? 32 : 16);
    p.rt = p.few ? (rows <= 16 ? 1 : 2) : p.dt < 256 && (rows % 128 == 0 || rows % 128 > 64 || rows > 640) ? 2 : 1;
    const int rows_per_wg = p.few ? 16 * p.rt : 64 * p.rt;
    p.tiles = (int)((rows + rows_per_wg - 1) / rows_per_wg);
    if (total_len <= 0 || total_len > n_requests * max_len) total_len = n_requests * max_len;
    // workgroups for about two on every CU, of at least 128 (few) or 256 keys each
    const int64_t least = p.few ? 128 : 256, want = 512;
    int64_t chunk = (total_len * n_kv * p.tiles + want - 1) / want;
    chunk = std::max(chunk, (max_len + MAX_CHUNKS - 1) / MAX_CHUNKS);
    if (max_rows * G * n_kv >= (int64_t)1 << 26) chunk = std::max(chunk, max_len);     // (more than a grid of the join counts)
    chunk = (std::max(chunk, least) + 127) / 128 * 128;
    p.chunk = (int)std::min<int64_t>(chunk, (int64_t)1 << 31 >> 1);
    p.chunks = (int)std::max<int64_t>(1, (max_len + p.chunk - 1) / p.chunk);
    return p;
}

}  // namespace

// partial results: O [chunk][row][head][D] fp32, then (maximum, sum) [chunk][row][head]
size_t tree_workspace_bytes(int64_t n_requests, int64_t M, int n_q, int n_kv, int D, int64_t max_rows, int64_t max_len, int64_t total_len)
{
    if (M == 0 || n_requests == 0 || max_rows == 0) return 0;
    const Plan p = make_plan(n_requests, std::min(max_rows, M), n_q / n_kv, n_kv, D, max_len, total_len);
    return p.chunks < 2 ? 0 : (size_t)p.chunks * M * n_q * (D + 2) * sizeof(float);
}

namespace {

struct Work {
    TreeArgs a;
    Divider by_g, by_tiles;
    float c;                             // |scale| * log2 e
    int flip;                            // scale < 0: queries change sign
    int tiles, chunk, chunks, n_kv;
    float* part_o;
    float2* part_ml;
};

// A request's rows and keys as one workgroup sees them.
struct Span {
    int64_t first;                       // first row
    int T, rows, len, ctx;               // drafted tokens, packed rows, keys, committed keys
    int n_chunks;
};

__device__ __forceinline__ Span make_span(const Work& w, int r)
{
    Span s;
    const int64_t lo = max((int64_t)w.a.row_start[r], (int64_t)0), hi = min((int64_t)w.a.row_start[r + 1], w.a.M);
    s.first = lo;
    s.T = (int)max(min(hi - lo, w.a.M), (int64_t)0);
    s.rows = (int)min((int64_t)s.T, w.a.max_rows) * w.a.G;
    const int64_t len = min(min((int64_t)w.a.kv_len[r], w.a.max_len), w.a.table_cols * w.a.cache.page_size);
    s.len = (int)max(len, (int64_t)0);
    s.ctx = s.len - s.T;
    s.n_chunks = max(1, (int)(((uint32_t)s.len + (uint32_t)w.chunk - 1) / (uint32_t)w.chunk));
    return s;
}

// Which of the keys base .. base + 3 (base a multiple of 4 from a tile's start on) the row sees, as 4 bits.
__device__ __forceinline__ uint32_t seen4(const TreeArgs& a, const Span& sp, int64_t row, int t, uint64_t word0, uint32_t base)
{
    const int j = (int)(base - (uint32_t)sp.ctx);            // drafted number of the first key
    if (!a.mask) return j > t ? 0u : t - j >= 3 ? 15u : (2u << (t - j)) - 1u;
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bool on = true;
        if (j + i >= 0) {
            const int w = (j + i) >> 6;
            on = w < a.mask_words;
            if (on) on = ((w == 0 ? word0 : a.mask[row * a.mask_words + w]) >> ((j + i) & 63)) & 1;
        }
        bits |= (uint32_t)on << i;
    }
    return bits;
}

// Where a key's row of the cache lies, in elements, without its head; `valid` false: not seen, a safe place.
__device__ __forceinline__ void locate(const TreeArgs& a, uint32_t key, int page, bool valid, int64_t* k_off, int64_t* v_off)
{
    const uint32_t at = divide(key, a.page);
    const int64_t place = key - (int64_t)at * a.cache.page_size;
    const int64_t p = valid ? page : 0;
    *k_off = p * a.cache.k_page_stride + place * a.cache.k_slot_stride;
    *v_off = p * a.cache.v_page_stride + place * a.cache.v_slot_stride;
}

template <int RT>
struct Rows {                            // a lane's query rows: row 16 rt + (lane & 15) of the wave's
    int64_t row[RT];                     // row of q and out
    int t[RT], head[RT];                 // drafted number, query head
    bool live[RT];
    uint64_t word[RT];                   // first word of the mask
};

template <int RT>
__device__ __forceinline__ Rows<RT> make_rows(const Work& w, const Span& sp, int rho0, int hk, int l16)
{
    Rows<RT> x;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int rho = rho0 + 16 * rt + l16;
        x.live[rt] = rho < sp.rows;
        const int safe = x.live[rt] ? rho : 0;
        x.t[rt] = (int)divide((uint32_t)safe, w.by_g);
        x.head[rt] = hk * w.a.G + safe - x.t[rt] * w.a.G;
        x.row[rt] = sp.first + x.t[rt];
        x.word[rt] = w.a.mask ? w.a.mask[x.row[rt] * w.a.mask_words] : 0;
    }
    return x;
}

// Query operands: row 16 rt + l16, numbers 32 ks + 8 q .. + 7
template <int DT, int RT>
__device__ __forceinline__ void load_q(const Work& w, const Rows<RT>& x, int q, v4i (&qf)[RT][DT / 32])
{
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int ks = 0; ks < DT / 32; ++ks) {
            const int d = 32 * ks + 8 * q;
            v4i v = {0, 0, 0, 0};
            if (x.live[rt] && d < w.a.D) v = *reinterpret_cast<const v4i*>(w.a.q + x.row[rt] * w.a.ldq + (int64_t)x.head[rt] * w.a.D + d);
            if (w.flip)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] ^= 0x80008000;
            qf[rt][ks] = v;
        }
}

// Weights of 32 keys (tiles s[0], s[1]) for one row tile; updates m, l and tells by how much the outputs shrink.
__device__ __forceinline__ float softmax_step(v4f (&s)[2], float c, float& m, float& l)
{
    float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    float shrink = 1.0f;
    if (__any((mx - m) * c > SLACK || (m == -INFINITY && mx != -INFINITY))) {
        const float up = fmaxf(m, mx);
        shrink = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - up) * c);
        l *= shrink;
        m = up;
    }
    const float off = m == -INFINITY ? 0.0f : -m * c;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[t][i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], c, off));
            l += s[t][i];
        }
    return shrink;
}

// The result of packed row (row, head), numbers d .. d + 3: rounded to q's type, or a chunk's part of it.
__device__ __forceinline__ void store4(const Work& w, bool whole, int chunk, int64_t row, int head, int d, const float4& o)
{
    if (d >= w.a.D) return;                                  // D and d are multiples of 4
    if (whole) {
        uint2 v;
        v.x = pack_bf16(o.x, o.y);
        v.y = pack_bf16(o.z, o.w);
        *reinterpret_cast<uint2*>(w.a.out + row * w.a.ldo + (int64_t)head * w.a.D + d) = v;
    } else {
        *reinterpret_cast<float4*>(w.part_o + (((int64_t)chunk * w.a.M + row) * w.a.n_q + head) * w.a.D + d) = o;
    }
}

__device__ __forceinline__ void store_stats(const Work& w, bool whole, int chunk, int64_t row, int head, float m, float l)
{
    if (!whole) w.part_ml[((int64_t)chunk * w.a.M + row) * w.a.n_q + head] = make_float2(m, l);
    else if (w.a.lse) w.a.lse[row * w.a.n_q + head] = l == 0.0f ? -INFINITY : (m * w.c + __log2f(l)) * (1.0f / LOG2E);
}

// ---------------------------------------------------------------------------------------------- few rows
constexpr int FEW_WAVES = 4;

template <int DT, int RT>
__global__ void __launch_bounds__(64 * FEW_WAVES) tree_few_kernel(Work w)
{
    constexpr int KS = DT / 32;
    constexpr int TILE = 32 * DT * 2;                        // a wave's 32 keys of V
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hk = blockIdx.x % w.n_kv, chunk = blockIdx.x / w.n_kv, r = blockIdx.y;
    const Span sp = make_span(w, r);
    if (sp.rows == 0 || chunk >= sp.n_chunks) return;
    const uint32_t k0 = (uint32_t)chunk * w.chunk, k1 = min((uint32_t)sp.len, k0 + w.chunk);
    const uint32_t ctx = max(sp.ctx, 0);
    const Rows<RT> x = make_rows<RT>(w, sp, 0, hk, l16);
    v4i qf[RT][KS];
    load_q<DT, RT>(w, x, q, qf);

    const uint16_t* const kh = w.a.cache.k + hk * w.a.cache.k_head_stride;
    const uint16_t* const vh = w.a.cache.v + hk * w.a.cache.v_head_stride;
    const int32_t* const table = w.a.table + r * w.a.ld_table;
    char* const vs = smem + wave * TILE;

    float m[RT], l[RT];
    v4f o[RT][DT / 16];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -INFINITY;
        l[rt] = 0.0f;
#pragma unroll
        for (int d = 0; d < DT / 16; ++d) o[rt][d] = (v4f){0.f, 0.f, 0.f, 0.f};
    }

    // a lane's keys of a step: l16 and 16 + l16
    auto page_of = [&](uint32_t base, int t) { return table[divide(min(base + 16 * t + l16, k1 - 1), w.a.page)]; };
    v4i kf[2][KS], vf[2][KS];
    int ids[2];
    uint32_t valid_next = 0, valid;
    int64_t voff[2];
    auto place = [&](uint32_t base, int64_t (&koff)[2]) {
        valid_next = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t key = base + 16 * t + l16;
            const bool ok = key < k1 && ids[t] >= 0 && ids[t] < w.a.cache.n_pages;
            valid_next |= ((uint32_t)__ballot(ok) & 0xffffu) << (16 * t);
            locate(w.a, min(key, k1 - 1), ids[t], ok, &koff[t], &voff[t]);
        }
    };
    auto load_k = [&](const int64_t (&koff)[2]) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int d = 32 * ks + 8 * q;
                kf[t][ks] = *reinterpret_cast<const v4i*>(kh + koff[t] + (d < w.a.D ? d : 0));
            }
    };
    auto load_v = [&]() {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int d = 32 * ks + 8 * q;
                vf[t][ks] = *reinterpret_cast<const v4i*>(vh + voff[t] + (d < w.a.D ? d : 0));
            }
    };

    uint32_t base = k0 + 32 * wave;
    constexpr uint32_t STEP = 32 * FEW_WAVES;
    if (base < k1) {
        int64_t koff[2];
        ids[0] = page_of(base, 0);
        ids[1] = page_of(base, 1);
        place(base, koff);
        ids[0] = page_of(base + STEP, 0);
        ids[1] = page_of(base + STEP, 1);
        load_k(koff);
        load_v();
        valid = valid_next;
    }
    for (; base < k1; base += STEP) {
        v4f s[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s[rt][t] = (v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) s[rt][t] = mfma(kf[t][ks], qf[rt][ks], s[rt][t]);
            }
        // the next keys are asked for as soon as these have met the queries (past the end: the last ones again)
        int64_t koff[2];
        place(base + STEP, koff);
        ids[0] = page_of(base + 2 * STEP, 0);
        ids[1] = page_of(base + 2 * STEP, 1);
        load_k(koff);

        if (valid != 0xffffffffu || base + 32 > ctx) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    uint32_t on = valid >> (16 * t + 4 * q) & 15u;
                    if (base + 32 > ctx) on &= seen4(w.a, sp, x.row[rt], x.t[rt], x.word[rt], base + 16 * t + 4 * q);
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[rt][t][i] = on >> i & 1 ? s[rt][t][i] : -INFINITY;
                }
        }
        v4i hi[RT], lo[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const float shrink = softmax_step(s[rt], w.c, m[rt], l[rt]);
            if (__any(shrink != 1.0f))
#pragma unroll
                for (int d = 0; d < DT / 16; ++d) o[rt][d] *= shrink;
            // weights in two bf16 parts: 16 bits of them meet V; the matrix pipe has the room
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const uint32_t h = pack_bf16(s[rt][t][i], s[rt][t][i + 1]);
                    hi[rt][2 * t + i / 2] = (int)h;
                    lo[rt][2 * t + i / 2] = (int)pack_bf16(s[rt][t][i] - __uint_as_float(h << 16),
                                                           s[rt][t][i + 1] - __uint_as_float(h & 0xffff0000u));
                }
        }
        // V to local memory, rows that are not seen by anybody as zeros
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = 16 * t + l16;
            const bool ok = valid >> key & 1;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int piece = 4 * ks + q;
                v4i v = vf[t][ks];
                if (!ok || 8 * piece >= w.a.D) v = (v4i){0, 0, 0, 0};
                *reinterpret_cast<v4i*>(vs + key * DT * 2 + ((piece ^ swizzle<DT>(key)) << 4)) = v;
            }
        }
        load_v();
        valid = valid_next;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int d = 0; d < DT / 16; ++d) {
            v4i vt;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int key = 16 * t + 4 * q + (l16 >> 2), piece = 2 * d + ((l16 >> 1) & 1);
                const v4s p = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(
                    vs + key * DT * 2 + ((piece ^ swizzle<DT>(key)) << 4) + 8 * (l16 & 1)));
                const uint2 u = __builtin_bit_cast(uint2, p);
                vt[2 * t] = (int)u.x;
                vt[2 * t + 1] = (int)u.y;
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                o[rt][d] = mfma(vt, hi[rt], o[rt][d]);
                o[rt][d] = mfma(vt, lo[rt], o[rt][d]);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }

    // the waves' parts meet in local memory, one row tile at a time
    constexpr int LD = DT + 4;
    float* const os = reinterpret_cast<float*>(smem);                         // [wave][16][LD]
    float* const ms = os + FEW_WAVES * 16 * LD;                               // [wave][16], then l
    float* const ls = ms + FEW_WAVES * 16;
    const bool whole = sp.n_chunks == 1;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float sum = l[rt];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        __syncthreads();
        if (q == 0) {
            ms[wave * 16 + l16] = m[rt];
            ls[wave * 16 + l16] = sum;
        }
#pragma unroll
        for (int d = 0; d < DT / 16; ++d)
            *reinterpret_cast<v4f*>(os + (wave * 16 + l16) * LD + 16 * d + 4 * q) = o[rt][d];
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * DT / 4; e += 64 * FEW_WAVES) {
            const int n = e / (DT / 4), d = e % (DT / 4) * 4;
            const int rho = 16 * rt + n;
            if (rho >= sp.rows) continue;
            float top = -INFINITY, all = 0.0f;
#pragma unroll
            for (int v = 0; v < FEW_WAVES; ++v) top = fmaxf(top, ms[v * 16 + n]);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int v = 0; v < FEW_WAVES; ++v) {
                const float mv = ms[v * 16 + n], f = mv == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((mv - top) * w.c);
                const float4 ov = *reinterpret_cast<const float4*>(os + (v * 16 + n) * LD + d);
                if (mv != -INFINITY) {
                    all = fmaf(ls[v * 16 + n], f, all);
                    acc.x = fmaf(ov.x, f, acc.x);
                    acc.y = fmaf(ov.y, f, acc.y);
                    acc.z = fmaf(ov.z, f, acc.z);
                    acc.w = fmaf(ov.w, f, acc.w);
                }
            }
            const int t = (int)divide((uint32_t)rho, w.by_g), head = hk * w.a.G + rho - t * w.a.G;
            const float inv = all == 0.0f ? 0.0f : 1.0f / all;
            if (whole) acc = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
            store4(w, whole, chunk, sp.first + t, head, d, acc);
            if (d == 0) store_stats(w, whole, chunk, sp.first + t, head, top, all);
        }
    }
}

// ---------------------------------------------------------------------------------------------- many rows
constexpr int TILE_WAVES = 4;
template <int DT> constexpr int stage_keys() { return DT == 256 ? 32 : 64; }
template <int DT> constexpr int stage_bytes() { return stage_keys<DT>() * DT * 2; }          // of K, and of V again

template <int DT, int RT>
__global__ void __launch_bounds__(64 * TILE_WAVES, DT == 256 ? 1 : 2) tree_tile_kernel(Work w)
{
    constexpr int KS = DT / 32, SK = stage_keys<DT>(), SB = stage_bytes<DT>();
    constexpr int LOADS = SB / 1024 / TILE_WAVES;            // of 64 pieces of 16 bytes, of K and of V, a wave and stage
    constexpr int PIECES = DT / 8;                           // of a row
    extern __shared__ __align__(16) char smem[];             // two stages of K and V
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // eight units (head, chunk) of a request side by side, then their next row tile: the tiles of a unit read the same keys, and
    // workgroups that are eight apart share an L2
    const uint32_t side = w.n_kv * w.chunks % 8 == 0 ? 3 : 0;
    const uint32_t group = divide(blockIdx.x >> side, w.by_tiles);
    const int tile = (blockIdx.x >> side) - group * w.tiles, unit = (group << side) + (blockIdx.x & ((1 << side) - 1));
    const int hk = unit % w.n_kv, chunk = unit / w.n_kv, r = blockIdx.y;
    const Span sp = make_span(w, r);
    const int rho_wg = tile * 64 * RT;
    if (rho_wg >= sp.rows || chunk >= sp.n_chunks) return;
    const int rho0 = rho_wg + wave * 16 * RT;
    const uint32_t k0 = (uint32_t)chunk * w.chunk, ctx = max(sp.ctx, 0);
    uint32_t k1 = min((uint32_t)sp.len, k0 + w.chunk);
    if (!w.a.mask) {                                         // causal: nothing past the tile's last token
        const int last = (int)divide((uint32_t)min(rho_wg + 64 * RT, sp.rows) - 1, w.by_g);
        k1 = max(k0, min(k1, (uint32_t)max(sp.ctx + last + 1, 0)));
    }
    const Rows<RT> x = make_rows<RT>(w, sp, rho0, hk, l16);
    v4i qf[RT][KS];
    load_q<DT, RT>(w, x, q, qf);

    const uint16_t* const kh = w.a.cache.k + hk * w.a.cache.k_head_stride;
    const uint16_t* const vh = w.a.cache.v + hk * w.a.cache.v_head_stride;
    const int32_t* const table = w.a.table + r * w.a.ld_table;

    float m[RT], l[RT];
    v4f o[RT][DT / 16];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -INFINITY;
        l[rt] = 0.0f;
#pragma unroll
        for (int d = 0; d < DT / 16; ++d) o[rt][d] = (v4f){0.f, 0.f, 0.f, 0.f};
    }

    // lane = key of a stage, for its page
    auto page_of = [&](uint32_t base) { return table[divide(min(base + (lane & (SK - 1)), k1 - 1), w.a.page)]; };
    auto fetch = [&](uint32_t base, int id, char* buf) -> uint64_t {
        const uint32_t key = base + (lane & (SK - 1));
        const bool ok = key < k1 && id >= 0 && id < w.a.cache.n_pages;
        int64_t koff, voff;
        locate(w.a, min(key, k1 - 1), id, ok, &koff, &voff);
        const uint64_t valid = __ballot(ok);
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int at = (wave * LOADS + j) * 64 + lane, row = at / PIECES, slot = at % PIECES;
            const int d = (slot ^ swizzle<DT>(row)) * 8;
            const int64_t ko = ((int64_t)__shfl((int)(koff >> 32), row) << 32) | (uint32_t)__shfl((int)koff, row);
            const int64_t vo = ((int64_t)__shfl((int)(voff >> 32), row) << 32) | (uint32_t)__shfl((int)voff, row);
            const bool there = (valid >> row & 1) && d < w.a.D;
            const void* const ka = there ? (const void*)(kh + ko + d) : (const void*)g_zeros;
            const void* const va = there ? (const void*)(vh + vo + d) : (const void*)g_zeros;
            char* const kd = buf + (wave * LOADS + j) * 1024;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)ka, (__attribute__((address_space(3))) void*)kd, 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)va, (__attribute__((address_space(3))) void*)(kd + SB), 16, 0, 0);
        }
        return valid;
    };

    uint64_t valid = 0, valid_next = 0;
    int id = 0;
    if (k0 < k1) {
        id = page_of(k0);
        valid = fetch(k0, id, smem);
        id = page_of(k0 + SK);
    }
    int buf = 0;
    for (uint32_t base = k0; base < k1; base += SK, buf ^= 1) {
        char* const ks_ = smem + buf * 2 * SB;
        char* const vs = ks_ + SB;
        __syncthreads();                                     // (waits for this stage's loads) every wave's part of the stage is there
        if (base + SK < k1) {
            valid_next = fetch(base + SK, id, smem + (buf ^ 1) * 2 * SB);
            id = page_of(base + 2 * SK);
        }
#pragma unroll
        for (int half = 0; half < SK / 32; ++half) {
            const uint32_t kb = base + 32 * half;
            v4f s[RT][2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int key = 32 * half + 16 * t + l16;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) s[rt][t] = (v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const v4i kf = *reinterpret_cast<const v4i*>(ks_ + key * DT * 2 + (((4 * ks + q) ^ swizzle<DT>(key)) << 4));
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) s[rt][t] = mfma(kf, qf[rt][ks], s[rt][t]);
                }
            }
            const uint32_t v32 = (uint32_t)(valid >> (32 * half));
            if (v32 != 0xffffffffu || kb + 32 > ctx) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        uint32_t on = v32 >> (16 * t + 4 * q) & 15u;
                        if (kb + 32 > ctx) on &= seen4(w.a, sp, x.row[rt], x.t[rt], x.word[rt], kb + 16 * t + 4 * q);
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[rt][t][i] = on >> i & 1 ? s[rt][t][i] : -INFINITY;
                    }
            }
            v4i p[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float shrink = softmax_step(s[rt], w.c, m[rt], l[rt]);
                if (__any(shrink != 1.0f))
#pragma unroll
                    for (int d = 0; d < DT / 16; ++d) o[rt][d] *= shrink;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; i += 2) p[rt][2 * t + i / 2] = (int)pack_bf16(s[rt][t][i], s[rt][t][i + 1]);
            }
#pragma unroll
            for (int d = 0; d < DT / 16; ++d) {
                v4i vt;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int key = 32 * half + 16 * t + 4 * q + (l16 >> 2), piece = 2 * d + ((l16 >> 1) & 1);
                    const v4s u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(
                        vs + key * DT * 2 + ((piece ^ swizzle<DT>(key)) << 4) + 8 * (l16 & 1)));
                    const uint2 u2 = __builtin_bit_cast(uint2, u);
                    vt[2 * t] = (int)u2.x;
                    vt[2 * t + 1] = (int)u2.y;
                }
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) o[rt][d] = mfma(vt, p[rt], o[rt][d]);
            }
        }
        valid = valid_next;
    }

    const bool whole = sp.n_chunks == 1;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float sum = l[rt];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (!x.live[rt]) continue;
        const float inv = !whole ? 1.0f : sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int d = 0; d < DT / 16; ++d)
            store4(w, whole, chunk, x.row[rt], x.head[rt], 16 * d + 4 * q,
                   make_float4(o[rt][d][0] * inv, o[rt][d][1] * inv, o[rt][d][2] * inv, o[rt][d][3] * inv));
        if (q == 0) store_stats(w, whole, chunk, x.row[rt], x.head[rt], m[rt], sum);
    }
}

// ---------------------------------------------------------------------------------------------- chunks of a request joined
// One wave per (row, query head) of a request; a lane holds 4 numbers.
__global__ void __launch_bounds__(256) tree_join_kernel(Work w)
{
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int head = (int)(unit % w.a.n_q), i = (int)(unit / w.a.n_q);
    const Span sp = make_span(w, blockIdx.y);
    if (i >= sp.T || i >= w.a.max_rows || sp.n_chunks < 2) return;
    const int64_t row = sp.first + i;
    const int64_t at = row * w.a.n_q + head, step = w.a.M * w.a.n_q;
    float top = -INFINITY;
    float2 mine[MAX_CHUNKS / 64];
#pragma unroll
    for (int e = 0; e < MAX_CHUNKS / 64; ++e) {
        mine[e] = make_float2(-INFINITY, 0.0f);
        if (e * 64 + lane < sp.n_chunks) mine[e] = w.part_ml[(int64_t)(e * 64 + lane) * step + at];
        top = fmaxf(top, mine[e].x);
    }
    top = wave_max_f32(top);
    float all = 0.0f, f[MAX_CHUNKS / 64];
#pragma unroll
    for (int e = 0; e < MAX_CHUNKS / 64; ++e) {
        f[e] = mine[e].x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((mine[e].x - top) * w.c);
        all = fmaf(mine[e].y, f[e], all);
    }
#pragma unroll
    for (int off = 32; off; off >>= 1) all += __shfl_xor(all, off);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const int d = 4 * lane;
    for (int c = 0; c < sp.n_chunks; ++c) {
        const float g = __shfl(c < 64 ? f[0] : f[1], c & 63);
        if (g == 0.0f || d >= w.a.D) continue;
        const float4 v = *reinterpret_cast<const float4*>(w.part_o + ((int64_t)c * step + at) * w.a.D + d);
        acc.x = fmaf(v.x, g, acc.x);
        acc.y = fmaf(v.y, g, acc.y);
        acc.z = fmaf(v.z, g, acc.z);
        acc.w = fmaf(v.w, g, acc.w);
    }
    const float inv = all == 0.0f ? 0.0f : 1.0f / all;
    store4(w, true, 0, row, head, d, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
    if (lane == 0) store_stats(w, true, 0, row, head, top, all);
}

template <int DT, int RT>
int launch_few(const Work& w, hipStream_t stream)
{
    constexpr int merge = FEW_WAVES * 16 * (DT + 4) * 4 + 2 * FEW_WAVES * 16 * 4, tiles = FEW_WAVES * 32 * DT * 2;
    constexpr int lds = merge > tiles ? merge : tiles;
    if (int rc = ensure_dynamic_lds((const void*)tree_few_kernel<DT, RT>, lds, "w2_tree_attention")) return rc;
    hipLaunchKernelGGL((tree_few_kernel<DT, RT>), dim3(w.chunks * w.n_kv, (unsigned)w.a.n_requests), dim3(64 * FEW_WAVES), lds, stream, w);
    return check_launch("w2_tree_attention");
}

template <int DT, int RT>
int launch_tile(const Work& w, hipStream_t stream)
{
    constexpr int lds = 4 * stage_bytes<DT>();
    if (int rc = ensure_dynamic_lds((const void*)tree_tile_kernel<DT, RT>, lds, "w2_tree_attention")) return rc;
    const int64_t blocks = (int64_t)w.chunks * w.n_kv * w.tiles;
    if (blocks >= (int64_t)1 << 24) return fail(W2_ERR_UNSUPPORTED_SHAPE, "w2_tree_attention: a request's rows are more than a grid counts");
    hipLaunchKernelGGL((tree_tile_kernel<DT, RT>), dim3((unsigned)blocks, (unsigned)w.a.n_requests), dim3(64 * TILE_WAVES), lds, stream, w);
    return check_launch("w2_tree_attention");
}

}  // namespace

int launch_tree_attention(const TreeArgs& a, hipStream_t stream)
{
    const int n_kv = a.cache.n_heads;
    const int64_t max_len = std::min(a.max_len, a.table_cols * a.cache.page_size);
    Plan p = make_plan(a.n_requests, a.max_rows, a.G, n_kv, a.D, max_len, a.total_len);
    Work w = {};
    w.a = a;
    w.a.max_len = max_len;
    const size_t per = (size_t)a.M * a.n_q * (a.D + 2) * sizeof(float);
    const int64_t room = std::min<int64_t>((int64_t)(a.workspace_bytes / per), MAX_CHUNKS);
    if (p.chunks > room) {                                   // no room for so many parts: longer chunks
        p.chunks = (int)std::max<int64_t>(1, room);
        p.chunk = (int)((max_len + p.chunks - 1) / p.chunks + 127) / 128 * 128;
        p.chunk = std::max(p.chunk, 128);
        p.chunks = (int)std::max<int64_t>(1, (max_len + p.chunk - 1) / p.chunk);
    }
    w.by_g = make_divider((uint32_t)a.G);
    w.by_tiles = make_divider((uint32_t)p.tiles);
    // (a scale of zero as the smallest number: unseen keys stay at -infinity)
    w.c = std::max(fabsf(a.scale) * LOG2E, 1e-30f);
    w.flip = a.scale < 0.0f;
    w.tiles = p.tiles;
    w.chunk = p.chunk;
    w.chunks = p.chunks;
    w.n_kv = n_kv;
    w.part_o = (float*)a.workspace;
    w.part_ml = (float2*)((float*)a.workspace + (size_t)p.chunks * a.M * a.n_q * a.D);
    int rc;
    if (p.few) {
        if (p.dt == 64) rc = p.rt == 1 ? launch_few<64, 1>(w, stream) : launch_few<64, 2>(w, stream);
        else if (p.dt == 128) rc = p.rt == 1 ? launch_few<128, 1>(w, stream) : launch_few<128, 2>(w, stream);
        else rc = launch_few<256, 1>(w, stream);
    } else {
        if (p.dt == 64) rc = p.rt == 1 ? launch_tile<64, 1>(w, stream) : launch_tile<64, 2>(w, stream);
        else if (p.dt == 128) rc = p.rt == 1 ? launch_tile<128, 1>(w, stream) : launch_tile<128, 2>(w, stream);
        else rc = launch_tile<256, 1>(w, stream);
    }
    if (rc || p.chunks < 2) return rc;
    const int64_t waves = a.max_rows * a.n_q;
    hipLaunchKernelGGL(tree_join_kernel, dim3((unsigned)((waves + 3) / 4), (unsigned)a.n_requests), dim3(256), 0, stream, w);
    return check_launch("w2_tree_attention");
}

}  // namespace w2
