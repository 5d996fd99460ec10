// Norm and rotation of the query and key heads of a fused QKV projection, keys and values into the paged cache, in one
// pass over the rows.
//
// A lane holds 2 * VEC numbers of a head: the two sides of VEC pairs (halves: numbers VEC j.. and rd/2 + VEC j..;
// interleaved: 2 VEC numbers in a row), or, past the rotated part, two runs of VEC numbers that stay.  GL lanes (a power
// of two) hold a head, so a wave takes 64 / GL heads of a row at a time; the sum of squares is reduced over GL lanes,
// and the VEC angles that a lane needs are made once for all heads of the row that its wave takes.
//
// The angle: position * phase is a 64-bit integer product whose upper half is the fraction of a turn, exact to 2^-32
// whatever the position (fp32 positions times frequencies are off by 0.004 radians at 131072 already); the sine
// instruction takes turns.
//
// Bound by memory: 8191 rows of 40 + 2 * 8 heads of 128, 235 MB, in 53 us, 4.4 TB/s (a large copy: 4.75); 96 rows in 4.5 us, one in
// 4.0: a launch and two trips to memory.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "block_ops.h"

namespace w2 {

namespace {

template <int VEC> struct VecOf;
template <> struct VecOf<8> { typedef uint4 type; };
template <> struct VecOf<2> { typedef uint32_t type; };

template <int VEC>
struct Packed {                          // VEC bf16 numbers
    uint32_t w[VEC / 2];
    __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16); }
};

template <int VEC>
__device__ __forceinline__ Packed<VEC> load_vec(const uint16_t* p)
{
    const typename VecOf<VEC>::type v = *reinterpret_cast<const typename VecOf<VEC>::type*>(p);
    Packed<VEC> r;
    memcpy(&r, &v, sizeof r);
    return r;
}

template <int VEC>
__device__ __forceinline__ void store_vec(uint16_t* p, const Packed<VEC>& x)
{
    typename VecOf<VEC>::type v;
    memcpy(&v, &x, sizeof v);
    *reinterpret_cast<typename VecOf<VEC>::type*>(p) = v;
}

// Sum over groups of GL lanes: moves within a row of 16 lanes ride on the addition
template <int GL>
__device__ __forceinline__ float group_sum(float v)
{
    if (GL > 1) v += dpp_move_f32<0xB1>(v);                  // quad_perm [1,0,3,2]
    if (GL > 2) v += dpp_move_f32<0x4E>(v);                  // quad_perm [2,3,0,1]
    if (GL > 4) v += dpp_move_f32<0x141>(v);                 // row_half_mirror
    if (GL > 8) v += dpp_move_f32<0x140>(v);                 // row_mirror
    if (GL > 16) v += __shfl_xor(v, 16);
    if (GL > 32) v += __shfl_xor(v, 32);
    return v;
}

constexpr int AHEAD = 4;                 // steps of 64 / GL heads whose loads are under way together

// One wave: `per` steps of 64 / GL heads of one row.
template <int VEC, int GL>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(RopeArgs a, int per, Divider by_chunks, int chunks, float inv_d)
{
    constexpr int HEADS = 64 / GL;
    const int lane = threadIdx.x & 63, j = lane & (GL - 1), sub = lane / GL;
    const uint32_t unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t m = divide(unit, by_chunks);
    if (m >= (uint64_t)a.M) return;
    const int H = a.n_q + 2 * a.n_kv;
    const int h0 = (int)(unit - m * chunks) * per * HEADS, h1 = min(H, h0 + per * HEADS);

    // where the two runs of this lane lie in a head
    const int pairs = a.rd / 2;
    int at0, at1;
    if (a.interleaved) {
        at0 = 2 * VEC * j;
        at1 = at0 + VEC;
    } else if (j * VEC < pairs) {
        at0 = j * VEC;
        at1 = pairs + j * VEC;
    } else {
        at0 = a.rd + 2 * (j * VEC - pairs);
        at1 = at0 + VEC;
    }
    const bool has0 = at0 < a.D, has1 = at1 < a.D;
    const uint16_t* const x = a.x + (int64_t)m * a.ldx;

    Packed<VEC> u0[AHEAD], u1[AHEAD];
    auto load = [&](int hb) {
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            const int h = hb + s * HEADS + sub;
            u0[s] = u1[s] = Packed<VEC>{};
            if (h < h1 && has0) u0[s] = load_vec<VEC>(x + h * a.D + at0);
            if (h < h1 && has1) u1[s] = load_vec<VEC>(x + h * a.D + at1);
        }
    };
    load(h0);
    Packed<VEC> qw0 = {}, qw1 = {}, kw0 = {}, kw1 = {};
    if (a.qw && has0) qw0 = load_vec<VEC>(a.qw + at0);
    if (a.qw && has1) qw1 = load_vec<VEC>(a.qw + at1);
    if (a.kw && has0) kw0 = load_vec<VEC>(a.kw + at0);
    if (a.kw && has1) kw1 = load_vec<VEC>(a.kw + at1);

    float c[VEC], s[VEC];
    const uint32_t pos = a.rd ? (uint32_t)a.positions[m] : 0;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const int pair = j * VEC + i;
        c[i] = 1.0f;
        s[i] = 0.0f;
        if (pair < pairs) {
            const uint64_t turns = pos * a.phase[pair];
            const float t = (float)(int32_t)(turns >> 32) * 0x1p-32f;       // -1/2 .. 1/2
            c[i] = __builtin_amdgcn_cosf(t) * a.mscale;
            s[i] = __builtin_amdgcn_sinf(t) * a.mscale;
        }
    }
    const int64_t slot = a.slots ? a.slots[m] : (int64_t)m;
    const bool kept = slot >= 0 && slot < a.cache.n_pages * a.cache.page_size;
    const uint32_t page = kept ? divide((uint32_t)slot, a.page) : 0;
    const uint32_t place = kept ? (uint32_t)slot - page * (uint32_t)a.cache.page_size : 0;
    uint16_t* const q = a.q + (int64_t)m * a.ldq;
    uint16_t* const k = a.cache.k + page * a.cache.k_page_stride + place * a.cache.k_slot_stride;
    uint16_t* const v = a.cache.v + page * a.cache.v_page_stride + place * a.cache.v_slot_stride;

    for (int hb = h0; hb < h1; hb += AHEAD * HEADS) {
        if (hb != h0) load(hb);
#pragma unroll
        for (int st = 0; st < AHEAD; ++st) {
            const int h = hb + st * HEADS + sub;
            if (hb + st * HEADS >= h1) break;
            const bool is_q = h < a.n_q, is_v = h >= a.n_q + a.n_kv;
            float v0[VEC], v1[VEC], sq = 0.0f;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                v0[i] = u0[st].at(i);
                v1[i] = u1[st].at(i);
                sq = fmaf(v0[i], v0[i], fmaf(v1[i], v1[i], sq));
            }
            sq = group_sum<GL>(sq);
            if (is_q ? a.qw != nullptr : a.kw != nullptr) {
                const float r = rsqrtf(sq * inv_d + a.eps);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    v0[i] *= r * (is_q ? qw0.at(i) : kw0.at(i));
                    v1[i] *= r * (is_q ? qw1.at(i) : kw1.at(i));
                }
            }
            float y[2 * VEC];                                // the two runs, one after the other
            if (a.interleaved) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float e = 2 * i < VEC ? v0[(2 * i) % VEC] : v1[(2 * i) % VEC], o = 2 * i < VEC ? v0[(2 * i + 1) % VEC] : v1[(2 * i + 1) % VEC];
                    const bool turned = j * VEC + i < pairs;             // (the others meet nothing: they may be infinite)
                    y[2 * i] = turned ? e * c[i] - o * s[i] : e;
                    y[2 * i + 1] = turned ? o * c[i] + e * s[i] : o;
                }
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const bool turned = j * VEC + i < pairs;
                    y[i] = v0[i] * c[i] - (turned ? v1[i] : 0.0f) * s[i];
                    y[VEC + i] = v1[i] * c[i] + (turned ? v0[i] : 0.0f) * s[i];
                }
            }
            Packed<VEC> y0 = u0[st], y1 = u1[st];            // (values stay)
            if (!is_v)
#pragma unroll
                for (int i = 0; i < VEC / 2; ++i) {
                    y0.w[i] = pack_bf16(y[2 * i], y[2 * i + 1]);
                    y1.w[i] = pack_bf16(y[VEC + 2 * i], y[VEC + 2 * i + 1]);
                }
            uint16_t* const dst = is_q ? q + h * a.D : is_v ? v + (h - a.n_q - a.n_kv) * a.cache.v_head_stride : k + (h - a.n_q) * a.cache.k_head_stride;
            if (h < h1 && (is_q || kept)) {
                if (has0) store_vec<VEC>(dst + at0, y0);
                if (has1) store_vec<VEC>(dst + at1, y1);
            }
        }
    }
}

template <int VEC, int GL>
void launch_rope(const RopeArgs& a, hipStream_t stream)
{
    const int steps = (a.n_q + 2 * a.n_kv + 64 / GL - 1) / (64 / GL);
    // a wave takes as much of a row as leaves 32 waves on every CU: its angles are made once, its loads overlap
    const int per = (int)std::max<int64_t>(1, std::min<int64_t>(steps, (a.M * steps + 8191) / 8192));
    const int chunks = (steps + per - 1) / per;
    const int64_t blocks = (a.M * chunks + 3) / 4;
    hipLaunchKernelGGL((qk_norm_rope_kernel<VEC, GL>), dim3((unsigned)blocks), dim3(256), 0, stream, a, per, make_divider((uint32_t)chunks), chunks,
                       1.0f / (float)a.D);
}

template <int VEC>
void launch_rope(const RopeArgs& a, hipStream_t stream)
{
    const int lanes = (a.D + 2 * VEC - 1) / (2 * VEC);
    if (lanes <= 4) launch_rope<VEC, 4>(a, stream);
    else if (lanes <= 8) launch_rope<VEC, 8>(a, stream);
    else if (lanes <= 16) launch_rope<VEC, 16>(a, stream);
    else if (lanes <= 32) launch_rope<VEC, 32>(a, stream);
    else launch_rope<VEC, 64>(a, stream);
}

}  // namespace

int launch_qk_norm_rope(const RopeArgs& a, hipStream_t stream)
{
    // runs of 8 numbers need the second half of the rotated part, and what follows it, to start at a multiple of 8
    if (a.interleaved || a.rd % 16 == 0) launch_rope<8>(a, stream);
    else launch_rope<2>(a, stream);
    return check_launch("w2_qk_norm_rope");
}

}  // namespace w2
