// Attention of each request's drafted tokens over its pages of the cache.
//
// The query rows of a cache head are packed, row rho = (token i) * G + (query head g), so that a group's heads share what
// is read of K and V.  Scores are held transposed: S^T = K Q^T puts keys of one query row in a lane, which is the operand
// layout of P^T in O^T = V^T P^T once the 32 keys of a step are numbered to suit: no weight crosses lanes.  V^T operands come
// from local memory by the transposing read.  Running maximum and sum per query row (m, l) in fp32; the outputs are rescaled
// only when a maximum has grown by more than 8 powers of two: weights up to 256, which neither fp32 sums nor bf16 weights overflow
// by; the sum is reduced over the lanes at the end.
//
// Times by the caller's clock among other calls; kernels alone, in a trace, where one is named.
// tree_few_kernel: up to 32 packed rows (decoding, small trees), 16x16x32 instructions.  Every wave of a workgroup takes other
// keys, which go to local memory past the registers, and nothing else waits for them.  Weights meet V in two bf16 parts, 16 bits:
// the matrix pipe has the room.  Bound by memory: 48 requests of one token, up to 8000 keys, 8 heads of 128: 967 MB in 155 us alone,
// 6.2 TB/s (a plain read of so much: 7.1).  One request of 700 keys: 9.8 us alone, a launch and six trips to memory.
// tree_tile_kernel: workgroups of 64 or 128 packed rows, 32 a wave, over a ring of shared stages of 32 keys, 32x32x16
// instructions.  Weights are rounded to bf16 once (against 64 bits the outputs are off by 0.0023 of their norm, 0.0017 of it
// the outputs' own rounding): a second part would be half as many products again.  Up to 64 rows bound by memory and by how
// evenly the keys are dealt out (16 requests of 36 rows, 174 MB: 38 us alone, 4.6 TB/s); above by what a wave does one after the
// other, with room in local memory and registers for two waves a SIMD: 2 requests of 320 rows, up to 120000 keys: 212 GFLOP in
// 299 us with the join's 9, 0.73 PFLOP/s, the matrix pipe busy a third of the time, vector instructions (16 exponentials a lane
// and stage) another; heads of 64, whose exponentials take longer than their products: 4 requests of 1000 tokens, 81 GFLOP in
// 123 us, vector issue a half.  With a mask it is a kernel of its own: what it does about keys that no row sees costs prompts 1 to
// 3 % where it is a branch of theirs.
// Keys of a request are cut into chunks for several workgroups where the batch alone does not fill the machine; partial
// results meet in tree_join_kernel.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "block_ops.h"
#include "tree_plan.h"
#include "w2_small_common.h"

namespace w2 {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.4426950408889634f;
constexpr float SLACK = 8.0f;            // powers of two a maximum may grow by before the outputs are rescaled

__device__ __align__(16) const uint32_t g_zeros[4] = {0, 0, 0, 0};

// an index that is the same in every lane, by the scalar unit
typedef const __attribute__((address_space(4))) int32_t* scalar_ptr;
__device__ __forceinline__ int scalar_load(const int32_t* p, int64_t i) { return ((scalar_ptr)(uintptr_t)p)[i]; }

__device__ __forceinline__ v4f mfma(const v4i& a, const v4i& b, const v4f& c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

// 16 bytes a lane from wherever the lane says to local memory, lane after lane from dst on
// (CACHE 2: read once, not to be kept)
template <int CACHE>
__device__ __forceinline__ void load_lds(const void* src, char* dst)
{
    asm volatile("" : "+v"(src));                            // (one load from a chosen address, not a choice of two loads: they are counted)
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)dst, 16, 0, CACHE);
}
// from a place that is the same in every lane, `off` bytes on
template <int CACHE>
__device__ __forceinline__ void load_lds_run(const char* run, uint32_t off, char* dst)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) char*)run + off, (__attribute__((address_space(3))) void*)dst, 16, 0, CACHE);
}
__device__ __forceinline__ void load_lds4(const void* src, char* dst)        // 4 bytes a lane
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)dst, 4, 0, 0);
}

// every read of local memory that was issued has delivered (what it read may be overwritten)
__device__ __forceinline__ void wait_reads()
{
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xc07f);                      // lgkmcnt 0
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// 16-byte pieces of a row of DT numbers are stored XORed by this: 16 rows at one piece (scores) lie in 16 different places of
// the 256 bytes that local memory delivers at once, and 8 rows at a pair of pieces (values) in 8 different pairs
template <int DT>
__device__ __forceinline__ int swizzle(int key) { return DT == 64 ? ((key & 6) | ((key >> 3) & 1)) : (((key & 7) << 1) | ((key >> 3) & 1)); }

// (fmaxf makes sure of every operand first, one instruction each)
__device__ __forceinline__ float max2(float a, float b)
{
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
// (the numbers may come straight from a matrix instruction: it is given the time that it needs, which the compiler does not
// see to for such a block)
__device__ __forceinline__ float max8(const v4f& a, const v4f& b)
{
    float r;
    asm("s_nop 15\n\ts_nop 7\n\t"
        "v_max3_f32 %0, %1, %2, %3\n\tv_max3_f32 %0, %0, %4, %5\n\tv_max3_f32 %0, %0, %6, %7\n\tv_max_f32 %0, %0, %8"
        : "=&v"(r)
        : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]));
    return r;
}

// V^T operands of four blocks of 16 numbers: lane (q, l16) gets numbers 16 d + l16 of keys 4q ..+ 3 of both tiles.  Rows of
// the cache are read transposed, 4 keys by 16 numbers for 16 lanes.  One block with its own wait: the compiler would wait
// here for every load to local memory that is under way, since it cannot tell that they go elsewhere.
template <int TILE_STEP>
__device__ __forceinline__ void read_vt(const uint32_t (&at)[4], v4i (&out)[4])
{
    uint2 a0, a1, b0, b1, c0, c1, d0, d1;
    asm volatile("ds_read_b64_tr_b16 %0, %8\n\t"
                 "ds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %2, %9\n\t"
                 "ds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %4, %10\n\t"
                 "ds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %6, %11\n\t"
                 "ds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(a0), "=&v"(a1), "=&v"(b0), "=&v"(b1), "=&v"(c0), "=&v"(c1), "=&v"(d0), "=&v"(d1)
                 : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(TILE_STEP)
                 : "memory");
    out[0] = (v4i){(int)a0.x, (int)a0.y, (int)a1.x, (int)a1.y};
    out[1] = (v4i){(int)b0.x, (int)b0.y, (int)b1.x, (int)b1.y};
    out[2] = (v4i){(int)c0.x, (int)c0.y, (int)c1.x, (int)c1.y};
    out[3] = (v4i){(int)d0.x, (int)d0.y, (int)d1.x, (int)d1.y};
}

__device__ __forceinline__ uint32_t lds_address(const char* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p; }

// Where a lane reads V^T of block d from: its key of a tile, the piece's place in the row
template <int DT>
__device__ __forceinline__ uint32_t vt_offset(int d, int q, int l16)
{
    const int key = 4 * q + (l16 >> 2), piece = 2 * d + ((l16 >> 1) & 1);
    return (uint32_t)(key * DT * 2 + ((piece ^ swizzle<DT>(key)) << 4) + 8 * (l16 & 1));
}

// Maximum, sum over the four lanes that hold a query row (lane & 15)
__device__ __forceinline__ float max_over_q(float x)
{
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const float y = max2(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
    return max2(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

}  // namespace

// partial results: O [chunk][row][head][D] fp32, then (maximum, sum) [chunk][row][head]
size_t tree_workspace_bytes(int64_t n_requests, int64_t M, int n_q, int n_kv, int D, int64_t max_rows, int64_t max_len, int64_t total_len)
{
    if (M == 0 || n_requests == 0 || max_rows == 0) return 0;
    const tree::Plan p = tree::make_plan(n_requests, std::min(max_rows, M), n_q / n_kv, n_kv, D, max_len, total_len);
    return p.chunks < 2 ? 0 : (size_t)p.chunks * M * n_q * (D + 2) * sizeof(float);
}

namespace {

struct Work {
    TreeArgs a;
    Divider by_g, by_tiles;
    float c;                             // |scale| * log2 e
    int flip;                            // scale < 0: queries change sign
    int same;                            // K and V have the same strides
    uint32_t n_pages, chunk;
    int tiles, chunks, n_kv;
    float* part_o;
    float2* part_ml;
};

// A request's rows and keys as one workgroup sees them.
struct Span {
    int64_t first;                       // first row
    int T, rows, len, ctx;               // drafted tokens, packed rows, keys that are not left out, committed keys (may be more)
    int n_chunks;
};

__device__ __forceinline__ Span make_span(const Work& w, int r)
{
    Span s;
    const int64_t lo = max((int64_t)scalar_load(w.a.row_start, r), (int64_t)0), hi = min((int64_t)scalar_load(w.a.row_start, r + 1), w.a.M);
    s.first = lo;
    s.T = (int)max(min(hi - lo, w.a.M), (int64_t)0);
    s.rows = (int)min((int64_t)s.T, w.a.max_rows) * w.a.G;
    // (keys past max_len and the page table are left out; the drafted ones are the last of all)
    const int keys = max(scalar_load(w.a.kv_len, r), 0);
    s.len = (int)min(min((int64_t)keys, w.a.max_len), w.a.table_cols * w.a.cache.page_size);
    s.ctx = keys - s.T;
    s.n_chunks = max(1, (int)(((uint32_t)s.len + w.chunk - 1) / w.chunk));
    return s;
}

// Workgroups that are eight apart run on one die: a die that saw one head only would ask one or two of its cache's channels
// for everything, since a head's rows lie a whole key apart.  The head of a workgroup turns with its chunk and request.
__device__ __forceinline__ int head_of(const Work& w, uint32_t unit, int chunk, int r)
{
    return (int)((unit + (uint32_t)chunk + (uint32_t)r) % (uint32_t)w.n_kv);
}

// Which of the keys base .. base + 3 (base a multiple of 4 from a tile's start on) the row sees, as 4 bits.
template <bool MASK>
__device__ __forceinline__ uint32_t seen4(const TreeArgs& a, const Span& sp, int64_t row, int t, uint64_t word0, uint32_t base)
{
    const int j = (int)(base - (uint32_t)sp.ctx);            // drafted number of the first key
    if (!MASK) return j > t ? 0u : t - j >= 3 ? 15u : (2u << (t - j)) - 1u;
    if (j <= -4) return 15u;
    if (j < 0) return (uint32_t)((word0 << -j) | ((1u << -j) - 1u)) & 15u;
    const uint64_t* const words = a.mask + row * a.mask_words;
    const int at = j >> 6, shift = j & 63;
    uint64_t bits = (at == 0 ? word0 : at < a.mask_words ? words[at] : 0) >> shift;
    if (shift > 60 && at + 1 < a.mask_words) bits |= words[at + 1] << (64 - shift);
    return (uint32_t)bits & 15u;
}

// Where a key's row of the cache lies, in elements, without its head; `valid` false: not seen, a safe place.  (Strides are
// below 2^31: one 32 x 32 -> 64 bit product each.)
__device__ __forceinline__ void locate(const Work& w, uint32_t key, int page, bool valid, uint64_t& k_off, uint64_t& v_off)
{
    const w2_kv_cache_t& c = w.a.cache;
    const uint32_t at = divide(key, w.a.page), place = key - at * (uint32_t)c.page_size, p = valid ? page : 0;
    k_off = (uint64_t)p * (uint32_t)c.k_page_stride + (uint64_t)place * (uint32_t)c.k_slot_stride;
    v_off = k_off;
    if (!w.same) v_off = (uint64_t)p * (uint32_t)c.v_page_stride + (uint64_t)place * (uint32_t)c.v_slot_stride;
}

// Pages of a multiple of 16 places (P16): 16 keys from a multiple of 16 on lie in one page, and an instruction that loads rows
// to local memory takes rows of one such run: where the two runs of a step begin is worked out by the scalar unit, a lane
// adds where its 16 bytes lie in a run, the same for every step.
// Where, in bytes, the run that starts at `key` lies in the cache, without its head
struct Run {
    uint64_t k, v;
};
__device__ __forceinline__ Run make_run(const Work& w, uint32_t key, uint32_t page)
{
    const w2_kv_cache_t& c = w.a.cache;
    const uint32_t place = key - divide(key, w.a.page) * (uint32_t)c.page_size;
    Run x;
    x.k = x.v = ((uint64_t)page * (uint32_t)c.k_page_stride + (uint64_t)place * (uint32_t)c.k_slot_stride) * 2;
    if (!w.same) x.v = ((uint64_t)page * (uint32_t)c.v_page_stride + (uint64_t)place * (uint32_t)c.v_slot_stride) * 2;
    return x;
}

// Which of the 32 keys from base on are there, their two runs in pages id[0] and id[1]
__device__ __forceinline__ uint32_t valid_keys(const Work& w, uint32_t base, uint32_t k1, const int (&id)[2])
{
    if (base + 32 <= k1 && (uint32_t)id[0] < w.n_pages && (uint32_t)id[1] < w.n_pages) return 0xffffffffu;
    uint32_t valid = 0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const uint32_t key = base + 16 * t;
        if (key < k1 && (uint32_t)id[t] < w.n_pages) valid |= (k1 - key >= 16 ? 0xffffu : (1u << (k1 - key)) - 1u) << (16 * t);
    }
    return valid;
}

// a 64-bit number of another lane
__device__ __forceinline__ uint64_t from_lane(uint64_t x, int lane)
{
    return (uint64_t)(uint32_t)__shfl((int)(x >> 32), lane) << 32 | (uint32_t)__shfl((int)x, lane);
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

// Scores of the 32 keys at kb against RT row tiles
template <int DT, int RT>
__device__ __forceinline__ void scores(const char* kb, int l16, int q, const v4i (&qf)[RT][DT / 32], v4f (&s)[RT][2])
{
    constexpr int KS = DT / 32;
    v4i kf[2][KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = 16 * t + l16;
            kf[t][ks] = *reinterpret_cast<const v4i*>(kb + key * DT * 2 + (((4 * ks + q) ^ swizzle<DT>(key)) << 4));
        }
    __builtin_amdgcn_sched_barrier(0);                       // all reads first, then the products as they arrive
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int t = 0; t < 2; ++t) s[rt][t] = (v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) s[rt][t] = mfma(kf[t][ks], qf[rt][ks], s[rt][t]);
}

// A drafted key that no row sees (a tree filled up to its size) may hold anything: its weights are zeros, and its value has to be
// made one.  Bits of keys, over the rows in 16 lanes (`halves`: 32)
__device__ __forceinline__ uint32_t any_row(uint32_t x, bool halves)
{
    x |= (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true);       // quad_perm [1,0,3,2]
    x |= (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true);       // quad_perm [2,3,0,1]
    x |= (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xf, 0xf, true);      // row_half_mirror
    x |= (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x140, 0xf, 0xf, true);      // row_mirror
    if (!halves) return x;
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return r[0] | r[1];
}
// masks of the eight values of a V^T operand, for the keys of eight bits
__device__ __forceinline__ v4i value_masks(uint32_t seen)
{
    v4i m;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int lo = (int)(seen << (31 - 2 * e)) >> 31, hi = (int)(seen << (30 - 2 * e)) >> 31;
        m[e] = (lo & 0xffff) | (hi & (int)0xffff0000);
    }
    return m;
}

// The running maximum (times c; -infinity: nothing seen yet), what is added to scores before the exponential, the lane's
// part of the sum.
struct Running {
    float top = -INFINITY, off = 0.0f, sum = 0.0f;
};

// Weights of 32 keys (tiles s[0], s[1]) for one row tile.
template <int N>
__device__ __forceinline__ void softmax_step(v4f (&s)[2], float c, Running& run, v4f (&o)[N])
{
    const float mx = max_over_q(max8(s[0], s[1]));
    // (a maximum of -infinity has no difference from itself: not a number, no change)
    if (__builtin_amdgcn_ballot_w64(fmaf(mx, c, -run.top) > SLACK)) {
        const float up = fmaxf(run.top, mx * c);
        const float shrink = run.top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(run.top - up);
        run.sum *= shrink;
        run.top = up;
        run.off = up == -INFINITY ? 0.0f : -up;
#pragma unroll
        for (int d = 0; d < N; ++d) o[d] *= shrink;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[t][i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], c, run.off));
            run.sum += s[t][i];
        }
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
    else if (w.a.lse) w.a.lse[row * w.a.n_q + head] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * (1.0f / LOG2E);
}

// ---------------------------------------------------------------------------------------------- few rows
template <int DT, int RT, int W, bool P16>
__global__ void __launch_bounds__(64 * W, DT == 256 ? 1 : 2) tree_few_kernel(Work w)
{
    constexpr int KS = DT / 32;
    constexpr int TILE = 32 * DT * 2;                        // a wave's 32 keys of K, and of V again
    constexpr int LOADS = TILE / 1024, PIECES = DT / 8;
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int chunk = blockIdx.x / w.n_kv, r = blockIdx.y, hk = head_of(w, blockIdx.x, chunk, r);
    const Span sp = make_span(w, r);
    if (sp.rows == 0 || chunk >= sp.n_chunks) return;
    const uint32_t k0 = (uint32_t)chunk * w.chunk, k1 = min((uint32_t)sp.len, k0 + w.chunk);
    const uint32_t ctx = max(sp.ctx, 0);

    const uint16_t* const kh = w.a.cache.k + hk * w.a.cache.k_head_stride;
    const uint16_t* const vh = w.a.cache.v + hk * w.a.cache.v_head_stride;
    const int32_t* const table = w.a.table + r * w.a.ld_table;
    char* const kb = smem + wave * 2 * TILE;
    char* const vb = kb + TILE;

    uint32_t valid = 0, valid_next = 0;
    // Pages of a step and, from them, where its rows lie.  Without P16: lane = key of a step (twice).
    struct Pages { int id[2]; };
    auto pages_of = [&](uint32_t base) {
        Pages p = {};
        if constexpr (P16) {
#pragma unroll
            for (int t = 0; t < 2; ++t) p.id[t] = scalar_load(table, divide(min(base + 16 * t, k1 - 1), w.a.page));
        } else {
            p.id[0] = table[divide(min(base + (lane & 31), k1 - 1), w.a.page)];
        }
        return p;
    };
    Run runs[2] = {};
    uint64_t koff = 0, voff = 0;
    auto place = [&](uint32_t base, const Pages& p) {
        if constexpr (P16) {
            valid_next = valid_keys(w, base, k1, p.id);
#pragma unroll
            for (int t = 0; t < 2; ++t)                      // (a run without a valid key: page 0, zeros are taken instead)
                runs[t] = make_run(w, base + 16 * t, valid_next >> (16 * t) & 0xffff ? p.id[t] : 0);
        } else {
            const uint32_t key = base + (lane & 31);
            const bool ok = key < k1 && (uint32_t)p.id[0] < w.n_pages;
            locate(w, min(key, k1 - 1), p.id[0], ok, koff, voff);
            valid_next = (uint32_t)__builtin_amdgcn_ballot_w64(ok);
        }
    };
    // whole rows of the cache side by side, 1 KiB an instruction; rows that nobody sees come from a place that holds zeros
    auto fetch = [&](bool is_v, char* dst) {
        const uint32_t slot_bytes = 2 * (uint32_t)(is_v ? w.a.cache.v_slot_stride : w.a.cache.k_slot_stride);
        if (P16 && valid_next == 0xffffffffu && w.a.D == DT) {
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const int at = j * 64 + lane, row = at / PIECES, d = (at % PIECES ^ swizzle<DT>(row)) * 8, t = j * 64 / PIECES / 16;
                const char* const run = (const char*)(is_v ? vh : kh) + (is_v ? runs[t].v : runs[t].k);
                load_lds_run<2>(run, (uint32_t)(row & 15) * slot_bytes + 2 * d, dst + j * 1024);
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int at = j * 64 + lane, row = at / PIECES, d = (at % PIECES ^ swizzle<DT>(row)) * 8, t = j * 64 / PIECES / 16;
            const char* src = (const char*)(is_v ? vh : kh) + 2 * d;
            if constexpr (P16) src += (is_v ? runs[t].v : runs[t].k) + (uint32_t)(row & 15) * slot_bytes;
            else src += 2 * from_lane(is_v ? voff : koff, row);
            load_lds<2>((valid_next >> row & 1) && d < w.a.D ? (const void*)src : (const void*)g_zeros, dst + j * 1024);
        }
    };

    constexpr uint32_t STEP = 32 * W;
    uint32_t base = k0 + 32 * wave;
    Pages pages = {};
    if (base < k1) {
        const Pages first = pages_of(base);
        pages = pages_of(base + STEP);
        place(base, first);
        fetch(false, kb);
        fetch(true, vb);
        valid = valid_next;
    }
    uint32_t vat[DT / 16];
#pragma unroll
    for (int d = 0; d < DT / 16; ++d) vat[d] = lds_address(vb) + vt_offset<DT>(d, q, l16);
    const Rows<RT> x = make_rows<RT>(w, sp, 0, hk, l16);
    v4i qf[RT][KS];
    load_q<DT, RT>(w, x, q, qf);
    Running run[RT];
    v4f o[RT][DT / 16];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int d = 0; d < DT / 16; ++d) o[rt][d] = (v4f){0.f, 0.f, 0.f, 0.f};
    if (base < k1) wait_loads<0>();                          // (the queries stand behind the first keys)

    // K of the next step is asked for as soon as this step's has met the queries, V when this step's has met the weights:
    // one buffer each.  Loads complete in order; what may be under way behind the one waited for is counted.
    for (; base < k1; base += STEP) {
        const bool more = base + STEP < k1;
        if (base != k0 + 32 * wave) wait_loads<LOADS>();     // K is there (V under way)
        v4f s[RT][2];
        scores<DT, RT>(kb, l16, q, qf, s);
        if (more) {
            const Pages next = pages;
            pages = pages_of(base + 2 * STEP);
            place(base + STEP, next);
            wait_reads();
            fetch(false, kb);
        }
        uint32_t seen = 0;                                   // by some row: the lane's keys, tile by tile
        bool hidden = false;                                 // keys that are there and not seen
        if (valid != 0xffffffffu || base + 32 > ctx) {
            uint32_t there = 0;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    uint32_t on = valid >> (16 * t + 4 * q) & 15u;
                    there |= on << 4 * t;
                    const uint32_t key = base + 16 * t + 4 * q;
                    if (base + 32 > ctx)
                        on &= w.a.mask ? seen4<true>(w.a, sp, x.row[rt], x.t[rt], x.word[rt], key) : seen4<false>(w.a, sp, x.row[rt], x.t[rt], 0, key);
                    seen |= on << 4 * t;
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[rt][t][i] = on >> i & 1 ? s[rt][t][i] : -INFINITY;
                }
            if (w.a.mask && base + 32 > ctx) {               // (keys that are not there are zeros already)
                seen = any_row(seen, false);
                hidden = __builtin_amdgcn_ballot_w64((there & ~seen) != 0) != 0;
            }
        }
        v4i hi[RT], lo[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            softmax_step(s[rt], w.c, run[rt], o[rt]);
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
        if (more) wait_loads<LOADS>();                       // V is there (the next K under way)
        else wait_loads<0>();
#pragma unroll
        for (int g = 0; g < DT / 64; ++g) {
            const uint32_t at[4] = {vat[4 * g], vat[4 * g + 1], vat[4 * g + 2], vat[4 * g + 3]};
            v4i vt[4];
            read_vt<16 * DT * 2>(at, vt);
            if (__builtin_expect(hidden, 0)) {
                asm volatile("" : "+v"(seen));               // (masks are made here, not held in registers by the common path)
                const v4i m = value_masks(seen);
#pragma unroll
                for (int e = 0; e < 4; ++e) vt[e] &= m;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    o[rt][4 * g + e] = mfma(vt[e], hi[rt], o[rt][4 * g + e]);
                    o[rt][4 * g + e] = mfma(vt[e], lo[rt], o[rt][4 * g + e]);
                }
        }
        if (more) {
            wait_reads();
            fetch(true, vb);
        }
        valid = valid_next;
    }

    // the waves' parts meet in local memory, one row tile at a time
    constexpr int LD = DT + 4;
    float* const os = reinterpret_cast<float*>(smem);                         // [wave][16][LD]
    float* const ms = os + W * 16 * LD;                               // [wave][16], then l
    float* const ls = ms + W * 16;
    const bool whole = sp.n_chunks == 1;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float sum = run[rt].sum;
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        __syncthreads();
        if (q == 0) {
            ms[wave * 16 + l16] = run[rt].top;
            ls[wave * 16 + l16] = sum;
        }
#pragma unroll
        for (int d = 0; d < DT / 16; ++d)
            *reinterpret_cast<v4f*>(os + (wave * 16 + l16) * LD + 16 * d + 4 * q) = o[rt][d];
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * DT / 4; e += 64 * W) {
            const int n = e / (DT / 4), d = e % (DT / 4) * 4;
            const int rho = 16 * rt + n;
            if (rho >= sp.rows) continue;
            float top = -INFINITY, all = 0.0f;
#pragma unroll
            for (int v = 0; v < W; ++v) top = fmaxf(top, ms[v * 16 + n]);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int v = 0; v < W; ++v) {
                // (a wave whose keys the row does not see adds nothing; one without a maximum whose sum is NaN has seen NaN)
                const float mv = ms[v * 16 + n], lv = ls[v * 16 + n], f = mv == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mv - top);
                const float4 ov = *reinterpret_cast<const float4*>(os + (v * 16 + n) * LD + d);
                if (mv != -INFINITY || lv != lv) {
                    all = fmaf(lv, f, all);
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
constexpr int RING = 4;                                      // stages of 32 keys in local memory
template <int DT> constexpr int stage_bytes() { return 32 * DT * 2; }                        // of K, and of V again
constexpr int ID_SLOTS = 8;                                  // a wave's pages of so many stages, 256 bytes each
template <int DT, int W, bool P16> constexpr int tile_lds() { return RING * 2 * stage_bytes<DT>() + (P16 ? 0 : W * ID_SLOTS * 256); }

typedef float v16f __attribute__((ext_vector_type(16)));

enum { CHECKED, WHOLE_HEADS, PADDED };                       // kinds of stages

__device__ __forceinline__ float max16(const v16f& s)
{
    float r;
    asm("s_nop 15\n\ts_nop 7\n\t"
        "v_max3_f32 %0, %1, %2, %3\n\tv_max3_f32 %0, %0, %4, %5\n\tv_max3_f32 %0, %0, %6, %7\n\tv_max3_f32 %0, %0, %8, %9\n\t"
        "v_max3_f32 %0, %0, %10, %11\n\tv_max3_f32 %0, %0, %12, %13\n\tv_max3_f32 %0, %0, %14, %15\n\tv_max_f32 %0, %0, %16"
        : "=&v"(r)
        : "v"(s[0]), "v"(s[1]), "v"(s[2]), "v"(s[3]), "v"(s[4]), "v"(s[5]), "v"(s[6]), "v"(s[7]), "v"(s[8]), "v"(s[9]), "v"(s[10]),
          "v"(s[11]), "v"(s[12]), "v"(s[13]), "v"(s[14]), "v"(s[15]));
    return r;
}

__device__ __forceinline__ v16f mfma32(const v4i& a, const v4i& b, const v16f& c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

// As swizzle(): here 4 rows at four pieces (values) have to lie in different places too
template <int DT>
__device__ __forceinline__ int swizzle32(int key) { return DT == 64 ? ((key & 2) << 1 | ((key >> 2) & 3)) : (((key & 3) << 2) | ((key >> 2) & 3)); }

// V^T operands of two blocks of 32 numbers, for the first and the second 16 keys of a stage.  at[block][j]: rows 8 j + 4 h ..
template <int BUF, int HALF>
__device__ __forceinline__ void read_vt32(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1, v4i (&out)[2][2])
{
    uint2 x0, x1, x2, x3, y0, y1, y2, y3;
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %1, %9 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %2, %8 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %4, %10 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %5, %11 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %6, %10 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(x0), "=&v"(x1), "=&v"(x2), "=&v"(x3), "=&v"(y0), "=&v"(y1), "=&v"(y2), "=&v"(y3)
                 : "v"(a0), "v"(a1), "v"(b0), "v"(b1), "n"(BUF), "n"(BUF + HALF)
                 : "memory");
    out[0][0] = (v4i){(int)x0.x, (int)x0.y, (int)x1.x, (int)x1.y};
    out[0][1] = (v4i){(int)x2.x, (int)x2.y, (int)x3.x, (int)x3.y};
    out[1][0] = (v4i){(int)y0.x, (int)y0.y, (int)y1.x, (int)y1.y};
    out[1][1] = (v4i){(int)y2.x, (int)y2.y, (int)y3.x, (int)y3.y};
}

// A wave holds 32 packed rows, one in lanes l and l + 32.  Scores: lane half h has keys 8 b + 4 h + i (b, i = 0..3) of a
// stage, which are slots 4 b + i of the weights' operands.  The scores of the next stage are multiplied while this stage's
// weights are made: matrix and vector instructions of one wave side by side.
template <int DT, int W, bool P16, bool MASK>
__global__ void __launch_bounds__(64 * W, W == 4 && DT < 256 ? 2 : 1) tree_tile_kernel(Work w)
{
    constexpr int KS = DT / 16, SB = stage_bytes<DT>();
    constexpr int LOADS = SB / 1024 / W;                     // of 64 pieces of 16 bytes, of K and of V, a wave and stage
    constexpr int PIECES = DT / 8;                           // of a row
    constexpr int NT = W == 2 ? 2 : 0;                       // (up to 64 rows are one tile: nobody else reads these keys)
    extern __shared__ __align__(16) char smem[];             // RING stages of K and V, pages
    const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // eight units (head, chunk) of a request side by side, then their next row tile: the tiles of a unit read the same keys, and
    // workgroups that are eight apart share an L2
    const uint32_t side = w.n_kv * w.chunks % 8 == 0 ? 3 : 0;
    const uint32_t group = divide(blockIdx.x >> side, w.by_tiles);
    const int tile = w.tiles - 1 - (int)((blockIdx.x >> side) - group * w.tiles);            // (causal: the longest first)
    const int unit = (group << side) + (blockIdx.x & ((1 << side) - 1));
    const int chunk = unit / w.n_kv, r = blockIdx.y;
    const int hk = head_of(w, unit, chunk, r);
    const Span sp = make_span(w, r);
    // the request's 32-row waves, spread evenly over its tiles: tiles that run alike stay close to each other in the keys, which
    // then come from the L2 once
    const int all_waves = (sp.rows + 31) / 32, tiles = (all_waves + W - 1) / W;
    if (tile >= tiles || chunk >= sp.n_chunks) return;
    const tree::Share own = tree::share(all_waves, tiles, tile);
    const int waves = own.count, rho_wg = 32 * own.first;
    const uint32_t k0 = (uint32_t)chunk * w.chunk, ctx = max(sp.ctx, 0);
    uint32_t k1 = min((uint32_t)sp.len, k0 + w.chunk);
    if (!MASK) {                                             // causal: nothing past the tile's last token
        const int last = (int)divide((uint32_t)min(rho_wg + 32 * waves, sp.rows) - 1, w.by_g);
        k1 = max(k0, min(k1, (uint32_t)max(sp.ctx + last + 1, 0)));
    }
    const int stages = (int)((k1 - k0 + 31) / 32);
    const uint16_t* const kh = w.a.cache.k + hk * w.a.cache.k_head_stride;
    const uint16_t* const vh = w.a.cache.v + hk * w.a.cache.v_head_stride;
    const int32_t* const table = w.a.table + r * w.a.ld_table;

    // Pages of a stage: P16: by the scalar unit, a stage before they are needed.  Else they go to local memory like its keys
    // (lane = key), RING - 1 stages before they are needed: a wave that waited for them in registers would wait for every load of
    // keys before them too.
    char* const ids = smem + RING * 2 * SB + wave * ID_SLOTS * 256;
    int next[2] = {0, 0}, page = 0;
    const int half = wave * LOADS * 64 / PIECES >= 16;       // the run that a wave's 8 rows of a stage lie in
    uint32_t koffs[LOADS], voffs[LOADS];                     // where a lane's pieces lie in a run
    bool real[LOADS];                                        // pieces of a head, not of what it is padded with
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
        const int at = (wave * LOADS + j) * 64 + lane, row = at / PIECES, d = (at % PIECES ^ swizzle32<DT>(row)) * 8;
        koffs[j] = (uint32_t)(row & 15) * 2 * (uint32_t)w.a.cache.k_slot_stride + 2 * d;
        voffs[j] = (uint32_t)(row & 15) * 2 * (uint32_t)w.a.cache.v_slot_stride + 2 * d;
        real[j] = d < w.a.D;
    }
    auto fetch_pages = [&](int st) {
        if constexpr (P16) {
#pragma unroll
            for (int t = 0; t < 2; ++t) next[t] = scalar_load(table, divide(min(k0 + (uint32_t)st * 32 + 16 * t, k1 - 1), w.a.page));
        } else {
            const uint32_t key = min(k0 + (uint32_t)st * 32 + l32, k1 - 1);
            load_lds4(table + divide(key, w.a.page), ids + (st & (ID_SLOTS - 1)) * 256);
        }
    };
    auto fetch = [&](int st, int buf) -> uint32_t {
        char* const dst = smem + buf * 2 * SB;
        if constexpr (P16) {
            const uint32_t base = k0 + (uint32_t)st * 32, valid = valid_keys(w, base, k1, next);
            const Run x = make_run(w, base + 16 * half, valid >> (16 * half) & 0xffff ? next[half] : 0);
            const char* const kr = (const char*)kh + x.k;
            const char* const vr = (const char*)vh + x.v;
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const int at = (wave * LOADS + j) * 64 + lane, row = at / PIECES, d = (at % PIECES ^ swizzle32<DT>(row)) * 8;
                const bool there = (valid >> row & 1) && d < w.a.D;
                char* const to = dst + (wave * LOADS + j) * 1024;
                load_lds<NT>(there ? (const void*)(kr + koffs[j]) : (const void*)g_zeros, to);
                load_lds<NT>(there ? (const void*)(vr + voffs[j]) : (const void*)g_zeros, to + SB);
            }
            return valid;
        }
        const uint32_t key = k0 + (uint32_t)st * 32 + l32;
        const int id = *reinterpret_cast<const int*>(ids + (st & (ID_SLOTS - 1)) * 256 + lane * 4);
        const bool ok = key < k1 && (uint32_t)id < w.n_pages;
        uint64_t koff, voff;
        locate(w, min(key, k1 - 1), id, ok, koff, voff);
        const uint32_t valid = (uint32_t)__builtin_amdgcn_ballot_w64(ok);
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int at = (wave * LOADS + j) * 64 + lane, row = at / PIECES, slot = at % PIECES;
            const int d = (slot ^ swizzle32<DT>(row)) * 8;
            const uint64_t ko = from_lane(koff, row), vo = w.same ? ko : from_lane(voff, row);
            const bool there = (valid >> row & 1) && d < w.a.D;
            char* const to = dst + (wave * LOADS + j) * 1024;
            load_lds<NT>(there ? (const void*)(kh + d + ko) : (const void*)g_zeros, to);
            load_lds<NT>(there ? (const void*)(vh + d + vo) : (const void*)g_zeros, to + SB);
        }
        return valid;
    };
    uint32_t valid[RING] = {};
    if (stages > 0) {
        if constexpr (!P16) {
#pragma unroll
            for (int st = 0; st < 2 * (RING - 1); ++st) fetch_pages(st);
            wait_loads<0>();
        }
#pragma unroll
        for (int st = 0; st < RING - 1; ++st)
            if (st < stages) {
                if constexpr (P16) fetch_pages(st);
                valid[st] = fetch(st, st);
            }
    }

    // the lane's query row, its operands: numbers 16 ks + 8 h ..+ 7
    const int rho = rho_wg + wave * 32 + l32;
    const bool idle = wave >= waves, live = !idle && rho < sp.rows;               // (idle: a wave without rows, which only loads)
    const int t = (int)divide((uint32_t)(live ? rho : 0), w.by_g), head = hk * w.a.G + (live ? rho : 0) - t * w.a.G;
    const int64_t row = sp.first + t;
    const uint64_t word = MASK ? w.a.mask[row * w.a.mask_words] : 0;
    v4i qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int d = 16 * ks + 8 * h;
        qf[ks] = (v4i){0, 0, 0, 0};
        if (live && d < w.a.D) qf[ks] = *reinterpret_cast<const v4i*>(w.a.q + row * w.a.ldq + (int64_t)head * w.a.D + d);
        if (w.flip)
#pragma unroll
            for (int e = 0; e < 4; ++e) qf[ks][e] ^= 0x80008000;
    }
    Running run;
    v16f o[DT / 32];
#pragma unroll
    for (int d = 0; d < DT / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;

    // addresses within a stage: K, pieces 2 ks + h of key l32; V^T, block d, rows 8 j + 4 h ..
    uint32_t kat[KS], vat[DT / 32][2];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kat[ks] = l32 * DT * 2 + (((2 * ks + h) ^ swizzle32<DT>(l32)) << 4);
#pragma unroll
    for (int d = 0; d < DT / 32; ++d)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int key = 8 * j + 4 * h + ((lane >> 2) & 3), piece = 4 * d + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
            vat[d][j] = lds_address(smem + SB) + key * DT * 2 + ((piece ^ swizzle32<DT>(key)) << 4) + 8 * (lane & 1);
        }
    auto read_k = [&](const char* kb, v4i (&kf)[KS]) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[ks] = *reinterpret_cast<const v4i*>(kb + kat[ks]);
    };
    auto zero = [](v16f& s) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.0f;
    };

    // V^T of blocks 2 g and 2 g + 1 of the stage in buffer bc
    auto read_v = [&](auto bc, int g, v4i (&vt)[2][2]) {
        constexpr int b = decltype(bc)::value;
        constexpr bool near = (b * 2 + 1) * SB < 65536;      // (within the reach of an instruction's offset)
        constexpr uint32_t far = near ? 0 : b * 2 * SB;
        read_vt32<near ? b * 2 * SB : 0, 16 * DT * 2>(vat[2 * g][0] + far, vat[2 * g][1] + far, vat[2 * g + 1][0] + far, vat[2 * g + 1][1] + far, vt);
    };
    // KIND: CHECKED, or a stage whose keys everybody sees, in the middle of a chunk whose pages are all there: nothing to check but
    // (PADDED) where a head ends.  cur: its scores, next: the next stage's.
    auto stage = [&](int st, auto bc, auto kind, v16f& cur, v16f& nxt) {
        constexpr int b = decltype(bc)::value, ahead = (b + RING - 1) % RING;
        constexpr bool INNER = decltype(kind)::value != CHECKED, WHOLE = decltype(kind)::value == WHOLE_HEADS;
        const uint32_t base = k0 + (uint32_t)st * 32;
        uint32_t seen = 0;                                   // by some row: the lane's keys
        bool hidden = false;                                 // keys that are there and not seen
        // the next stage is there; one behind it is under way
        if (INNER || st + 2 < stages) wait_loads<2 * LOADS>();
        else wait_loads<0>();
        bare_barrier();                                      // every wave's part of it, and no wave reads the stage before this one any more
        if constexpr (INNER) {
            const uint32_t mine = base + 32 * (RING - 1) + 16 * half;
            const Run x = make_run(w, mine, (uint32_t)page);
            page = scalar_load(table, divide(mine + 32, w.a.page));      // (mine + 32 < k1)
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                char* const to = smem + ahead * 2 * SB + (wave * LOADS + j) * 1024;
                if constexpr (WHOLE) {
                    load_lds_run<NT>((const char*)kh + x.k, koffs[j], to);
                    load_lds_run<NT>((const char*)vh + x.v, voffs[j], to + SB);
                } else {
                    load_lds<NT>(real[j] ? (const void*)((const char*)kh + x.k + koffs[j]) : (const void*)g_zeros, to);
                    load_lds<NT>(real[j] ? (const void*)((const char*)vh + x.v + voffs[j]) : (const void*)g_zeros, to + SB);
                }
            }
        } else {
            if (st + RING - 1 < stages) {
                if constexpr (P16) fetch_pages(st + RING - 1);
                else fetch_pages(st + 2 * (RING - 1));
                valid[ahead] = fetch(st + RING - 1, ahead);
            }
            if (valid[b] != 0xffffffffu || base + 32 > ctx) {
                uint32_t there = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t on = valid[b] >> (8 * e + 4 * h) & 15u;
                    if (MASK) there |= on << 4 * e;
                    if (base + 32 > ctx) on &= seen4<MASK>(w.a, sp, row, t, word, base + 8 * e + 4 * h);
                    if (MASK) seen |= on << 4 * e;
#pragma unroll
                    for (int i = 0; i < 4; ++i) cur[4 * e + i] = on >> i & 1 ? cur[4 * e + i] : -INFINITY;
                }
                if (MASK && base + 32 > ctx) {               // (keys that are not there are zeros already)
                    seen = any_row(seen, true);
                    hidden = __builtin_amdgcn_ballot_w64((there & ~seen) != 0) != 0;
                }
            }
        }
        if (idle) return;
        // the next stage's keys: on their way while the maximum is taken, where there are registers for them
        // (past the last stage: whatever the buffer holds, for scores that nobody uses)
        v4i kf[KS];
        if (DT < 256) read_k(smem + (b + 1) % RING * 2 * SB, kf);
        __builtin_amdgcn_sched_barrier(0);
        float mx = max16(cur);
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = max2(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
        if (__builtin_amdgcn_ballot_w64(fmaf(mx, w.c, -run.top) > SLACK)) {
            const float up = fmaxf(run.top, mx * w.c);
            const float shrink = run.top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(run.top - up);
            run.sum *= shrink;
            run.top = up;
            run.off = up == -INFINITY ? 0.0f : -up;
#pragma unroll
            for (int d = 0; d < DT / 32; ++d) o[d] *= shrink;
        }
        __builtin_amdgcn_sched_barrier(0);
        if (DT == 256) read_k(smem + (b + 1) % RING * 2 * SB, kf);
        v4i vt[2][2];
        read_v(bc, 0, vt);                                   // the first values' wait is the keys' too
        zero(nxt);
        v4i p[2];
        __builtin_amdgcn_sched_barrier(0);                   // all reads first; then a product, its share of the vector instructions, a product ...
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) nxt = mfma32(kf[ks], qf[ks], nxt);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            cur[i] = __builtin_amdgcn_exp2f(fmaf(cur[i], w.c, run.off));
            run.sum += cur[i];
        }
#pragma unroll
        for (int i = 0; i < 16; i += 2) p[i >> 3][(i & 7) >> 1] = (int)pack_bf16(cur[i], cur[i + 1]);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 56 / KS, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = 0; g < DT / 64; ++g) {
            if (g) read_v(bc, g, vt);
            if (MASK && !INNER && __builtin_expect(hidden, 0)) {
                asm volatile("" : "+v"(seen));               // (masks are made here, not held in registers by the common path)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const v4i m = value_masks(seen >> 8 * k);
#pragma unroll
                    for (int e = 0; e < 2; ++e) vt[e][k] &= m;
                }
            }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < 2; ++e) o[2 * g + e] = mfma32(vt[e][k], p[k], o[2 * g + e]);
        }
        // (the stage's reads have all delivered: the scores have been used, and the values wait for themselves)
    };
    v16f sa, sb;
    zero(sa);
    zero(sb);
    int inner = 0;                                           // stages of that kind, from the first on
    if (stages > 0) {
        if (P16) {
            inner = max(min((int)((k1 - k0) / 32) - RING, (int)((min(ctx, k1) - min(ctx, k0)) / 32)), 0) / RING * RING;
            const uint32_t p0 = divide(k0, w.a.page), p1 = divide(k1 - 1, w.a.page);
            bool all = inner > 0;
            if (all)
                for (uint32_t p = p0 + lane; p <= p1; p += 64) all &= (uint32_t)table[p] < w.n_pages;
            if (__builtin_amdgcn_ballot_w64(all) != ~(uint64_t)0) inner = 0;
            if (inner) page = scalar_load(table, divide(k0 + 32 * (RING - 1) + 16 * half, w.a.page));
        }
        if (stages > 2) wait_loads<4 * LOADS>();
        else if (stages > 1) wait_loads<2 * LOADS>();
        else wait_loads<0>();
        bare_barrier();
        v4i kf[KS];
        read_k(smem, kf);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sa = mfma32(kf[ks], qf[ks], sa);
    }
    static_assert(RING == 4, "the loops below");
    typedef std::integral_constant<int, 0> B0;
    typedef std::integral_constant<int, 1> B1;
    typedef std::integral_constant<int, 2> B2;
    typedef std::integral_constant<int, 3> B3;
    int st = 0;
    auto ring = [&](auto kind) {
        for (; st < inner; st += RING) {
            stage(st, B0{}, kind, sa, sb);
            stage(st + 1, B1{}, kind, sb, sa);
            stage(st + 2, B2{}, kind, sa, sb);
            stage(st + 3, B3{}, kind, sb, sa);
        }
    };
    if (w.a.D == DT) ring(std::integral_constant<int, WHOLE_HEADS>{});
    else ring(std::integral_constant<int, PADDED>{});
    // (the inner stages asked for three whole stages behind them)
    if (inner)
#pragma unroll
        for (int b = 0; b < RING - 1; ++b) valid[b] = 0xffffffffu;
    const std::integral_constant<int, CHECKED> checked;
    for (; st < stages; st += RING) {
        stage(st, B0{}, checked, sa, sb);
        if (st + 1 < stages) stage(st + 1, B1{}, checked, sb, sa);
        if (st + 2 < stages) stage(st + 2, B2{}, checked, sa, sb);
        if (st + 3 < stages) stage(st + 3, B3{}, checked, sb, sa);
    }

    const bool whole = sp.n_chunks == 1;
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(run.sum), __float_as_uint(run.sum), false, false);
    const float sum = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    if (!live) return;
    const float inv = !whole ? 1.0f : sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int d = 0; d < DT / 32; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            store4(w, whole, chunk, row, head, 32 * d + 8 * e + 4 * h,
                   make_float4(o[d][4 * e] * inv, o[d][4 * e + 1] * inv, o[d][4 * e + 2] * inv, o[d][4 * e + 3] * inv));
    if (h == 0) store_stats(w, whole, chunk, row, head, run.top, sum);
}

// ---------------------------------------------------------------------------------------------- chunks of a request joined
// D / 4 lanes (rounded up to a power of two, `width`) hold the numbers of a (row, query head) of a request; `share` such groups
// (a power of two) take turns at its chunks, eight at a time, and meet in local memory.
__global__ void __launch_bounds__(256) tree_join_kernel(Work w, int width, int share)
{
    __shared__ float4 sums[256];
    __shared__ float2 stats[256];
    const int per = 256 / (width * share), lane = threadIdx.x & (width - 1);
    const int sub = threadIdx.x / width & (share - 1), which = threadIdx.x / (width * share);
    const int64_t unit = (int64_t)blockIdx.x * per + which;
    const int i = (int)(unit / w.a.n_q), head = (int)(unit - (int64_t)i * w.a.n_q), d = 4 * lane;
    const Span sp = make_span(w, blockIdx.y);
    if (sp.n_chunks < 2 || (int)((int64_t)blockIdx.x * per / w.a.n_q) >= sp.T) return;       // (the same for the whole workgroup)
    const bool live = i < sp.T && i < w.a.max_rows;
    const int64_t at = (sp.first + (live ? i : 0)) * w.a.n_q + head, step = w.a.M * w.a.n_q;
    float top = -INFINITY, all = 0.0f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (live)
        for (int c0 = sub; c0 < sp.n_chunks; c0 += 8 * share) {
            float2 ml[8];
            float4 v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int c = c0 + e * share;
                ml[e] = make_float2(-INFINITY, 0.0f);
                v[e] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (c < sp.n_chunks) {
                    ml[e] = w.part_ml[c * step + at];
                    if (d < w.a.D) v[e] = *reinterpret_cast<const float4*>(w.part_o + (c * step + at) * w.a.D + d);
                }
            }
            float up = top;
#pragma unroll
            for (int e = 0; e < 8; ++e) up = fmaxf(up, ml[e].x);
            const float keep = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - up);
            all *= keep;
            acc = make_float4(acc.x * keep, acc.y * keep, acc.z * keep, acc.w * keep);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float f = ml[e].x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml[e].x - up);
                all = fmaf(ml[e].y, f, all);
                acc = make_float4(fmaf(v[e].x, f, acc.x), fmaf(v[e].y, f, acc.y), fmaf(v[e].z, f, acc.z), fmaf(v[e].w, f, acc.w));
            }
            top = up;
        }
    if (share > 1) {
        sums[threadIdx.x] = acc;
        stats[threadIdx.x] = make_float2(top, all);
        __syncthreads();
        if (sub) return;
        float up = top;
        for (int g = 1; g < share; ++g) up = fmaxf(up, stats[threadIdx.x + g * width].x);
        float sum = 0.0f;
        acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int g = 0; g < share; ++g) {
            const float2 ml = stats[threadIdx.x + g * width];
            const float4 v = sums[threadIdx.x + g * width];
            const float f = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.x - up);
            sum = fmaf(ml.y, f, sum);
            acc = make_float4(fmaf(v.x, f, acc.x), fmaf(v.y, f, acc.y), fmaf(v.z, f, acc.z), fmaf(v.w, f, acc.w));
        }
        top = up;
        all = sum;
    }
    if (!live) return;
    const float inv = all == 0.0f ? 0.0f : 1.0f / all;
    const int64_t row = sp.first + i;
    store4(w, true, 0, row, head, d, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
    if (lane == 0) store_stats(w, true, 0, row, head, top, all);
}

template <typename Kern>
int launch(Kern kern, const Work& w, int64_t blocks, int waves, int lds, hipStream_t stream)
{
    if (blocks >= (int64_t)1 << 24) return fail(W2_ERR_UNSUPPORTED_SHAPE, "w2_tree_attention: a request's rows are more than a grid counts");
    if (int rc = ensure_dynamic_lds((const void*)kern, lds, "w2_tree_attention")) return rc;
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks, (unsigned)w.a.n_requests), dim3(64 * waves), lds, stream, w);
    return check_launch("w2_tree_attention");
}

template <int DT, int RT, int W>
int launch_few(const Work& w, bool p16, hipStream_t stream)
{
    constexpr int merge = W * 16 * (DT + 4) * 4 + 2 * W * 16 * 4, tiles = W * 2 * 32 * DT * 2;
    const int64_t blocks = (int64_t)w.chunks * w.n_kv;
    return launch(p16 ? tree_few_kernel<DT, RT, W, true> : tree_few_kernel<DT, RT, W, false>, w, blocks, W, std::max(merge, tiles), stream);
}

template <int DT, int W, bool MASK>
int launch_tile(const Work& w, bool p16, hipStream_t stream)
{
    const int64_t blocks = (int64_t)w.chunks * w.n_kv * w.tiles;
    return p16 ? launch(tree_tile_kernel<DT, W, true, MASK>, w, blocks, W, tile_lds<DT, W, true>(), stream)
               : launch(tree_tile_kernel<DT, W, false, MASK>, w, blocks, W, tile_lds<DT, W, false>(), stream);
}

template <int DT>
int launch_tile(const Work& w, int waves, bool p16, hipStream_t stream)
{
    if (w.a.mask) return waves == 2 ? launch_tile<DT, 2, true>(w, p16, stream) : launch_tile<DT, 4, true>(w, p16, stream);
    return waves == 2 ? launch_tile<DT, 2, false>(w, p16, stream) : launch_tile<DT, 4, false>(w, p16, stream);
}

}  // namespace

int launch_tree_attention(const TreeArgs& a, hipStream_t stream)
{
    const int n_kv = a.cache.n_heads;
    const int64_t max_len = std::min(a.max_len, a.table_cols * a.cache.page_size);
    tree::Plan p = tree::make_plan(a.n_requests, a.max_rows, a.G, n_kv, a.D, max_len, a.total_len);
    const size_t per = (size_t)a.M * a.n_q * (a.D + 2) * sizeof(float);
    tree::fit(p, max_len, std::min<int64_t>((int64_t)(a.workspace_bytes / per), tree::MAX_CHUNKS));
    Work w = {};
    w.a = a;
    w.a.max_len = max_len;
    w.by_g = make_divider((uint32_t)a.G);
    w.by_tiles = make_divider((uint32_t)p.tiles);
    // (a scale of zero as the smallest number: unseen keys stay at -infinity)
    w.c = std::max(fabsf(a.scale) * LOG2E, 1e-30f);
    w.flip = a.scale < 0.0f;
    w.n_pages = (uint32_t)a.cache.n_pages;
    w.same = a.cache.k_page_stride == a.cache.v_page_stride && a.cache.k_slot_stride == a.cache.v_slot_stride;
    w.tiles = p.tiles;
    w.chunk = p.chunk;
    w.chunks = p.chunks;
    w.n_kv = n_kv;
    w.part_o = (float*)a.workspace;
    w.part_ml = (float2*)((float*)a.workspace + (size_t)p.chunks * a.M * a.n_q * a.D);
    // (chunks begin at multiples of 128 keys; a run of 16 rows has to span less than 2^31 bytes)
    const bool p16 = a.cache.page_size % 16 == 0 && std::max(a.cache.k_slot_stride, a.cache.v_slot_stride) < (int64_t)1 << 25;
    int rc;
    if (p.few) {
        if (p.dt == 256) rc = launch_few<256, 1, 4>(w, p16, stream);
        else if (p.rt == 2) rc = p.dt == 64 ? launch_few<64, 2, 4>(w, p16, stream) : launch_few<128, 2, 4>(w, p16, stream);
        else if (p.waves == 8) rc = p.dt == 64 ? launch_few<64, 1, 8>(w, p16, stream) : launch_few<128, 1, 8>(w, p16, stream);
        else rc = p.dt == 64 ? launch_few<64, 1, 4>(w, p16, stream) : launch_few<128, 1, 4>(w, p16, stream);
    } else {
        rc = p.dt == 64 ? launch_tile<64>(w, p.waves, p16, stream) : p.dt == 128 ? launch_tile<128>(w, p.waves, p16, stream) : launch_tile<256>(w, p.waves, p16, stream);
    }
    if (rc || p.chunks < 2) return rc;
    int width = 1;
    while (4 * width < a.D) width *= 2;
    int share = 1;
    while (8 * share < p.chunks && 2 * share * width <= 256) share *= 2;
    const int64_t units = 256 / (width * share), blocks = (a.max_rows * a.n_q + units - 1) / units;
    hipLaunchKernelGGL(tree_join_kernel, dim3((unsigned)blocks, (unsigned)a.n_requests), dim3(256), 0, stream, w, width, share);
    return check_launch("w2_tree_attention");
}

}  // namespace w2
