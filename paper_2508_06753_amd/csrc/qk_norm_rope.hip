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
#include <hip/hip_runtime.h>

#include "block_ops.h"

namespace w2 {

template <int VEC> struct VecOf;
template <> struct VecOf<8> { typedef uint4 type; };
template <> struct VecOf<2> { typedef uint32_t type; };

template <int VEC>
__device__ __forceinline__ void load_vec(const uint16_t* p, uint16_t (&v)[VEC])
{
    typedef typename VecOf<VEC>::type V;
    const V w = *reinterpret_cast<const V*>(p);
    memcpy(v, &w, sizeof w);
}

template <int VEC>
__device__ __forceinline__ void store_vec(uint16_t* p, const uint16_t (&v)[VEC])
{
    typedef typename VecOf<VEC>::type V;
    V w;
    memcpy(&w, v, sizeof w);
    *reinterpret_cast<V*>(p) = w;
}

// One wave: `heads` heads of row m from head h0 on, in steps of 64 / GL.
template <int VEC, int GL>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(RopeArgs a, int chunks, int chunk_heads)
{
    const int lane = threadIdx.x & 63, j = lane & (GL - 1), sub = lane / GL;
    const int64_t unit = (int64_t)blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6);
    const int64_t m = unit / chunks;
    if (m >= a.M) return;
    const int H = a.n_q + 2 * a.n_kv;
    const int h0 = (int)(unit % chunks) * chunk_heads, h1 = min(H, h0 + chunk_heads);

    // where the two runs of this lane lie in a head, and whether its pairs are turned
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
    int64_t slot = a.slots ? a.slots[m] : m;
    const bool kept = slot >= 0 && slot < a.cache.n_pages * a.cache.page_size;
    const uint32_t page = kept ? divide((uint32_t)slot, a.page) : 0;
    const int64_t place = kept ? slot - (int64_t)page * a.cache.page_size : 0;

    for (int hb = h0; hb < h1; hb += 64 / GL) {
        const int h = hb + sub;
        const bool live = h < h1;
        const uint16_t* src = a.x + m * a.ldx + (int64_t)min(h, H - 1) * a.D;
        uint16_t u0[VEC] = {}, u1[VEC] = {};
        if (live && has0) load_vec<VEC>(src + at0, u0);
        if (live && has1) load_vec<VEC>(src + at1, u1);
        const bool is_q = h < a.n_q, is_v = h >= a.n_q + a.n_kv;
        const uint16_t* w = is_q ? a.qw : a.kw;
        float v0[VEC], v1[VEC], sq = 0.0f;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            v0[i] = bf16_f32(u0[i]);
            v1[i] = bf16_f32(u1[i]);
            sq = fmaf(v0[i], v0[i], fmaf(v1[i], v1[i], sq));
        }
#pragma unroll
        for (int off = GL / 2; off; off >>= 1) sq += __shfl_xor(sq, off);
        if (!is_v) {
            if (w) {
                const float r = rsqrtf(sq / (float)a.D + a.eps);
                uint16_t w0[VEC] = {}, w1[VEC] = {};
                if (has0) load_vec<VEC>(w + at0, w0);
                if (has1) load_vec<VEC>(w + at1, w1);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    v0[i] *= r * bf16_f32(w0[i]);
                    v1[i] *= r * bf16_f32(w1[i]);
                }
            }
            if (a.interleaved) {
                float v[2 * VEC];
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    v[i] = v0[i];
                    v[VEC + i] = v1[i];
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float x = v[2 * i], y = v[2 * i + 1];
                    v[2 * i] = x * c[i] - y * s[i];
                    v[2 * i + 1] = y * c[i] + x * s[i];
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    u0[i] = f32_bf16(v[i]);
                    u1[i] = f32_bf16(v[VEC + i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    u0[i] = f32_bf16(v0[i] * c[i] - v1[i] * s[i]);
                    u1[i] = f32_bf16(v1[i] * c[i] + v0[i] * s[i]);
                }
            }
        }
        uint16_t* dst;
        if (is_q) dst = a.q + m * a.ldq + (int64_t)h * a.D;
        else if (!is_v) dst = a.cache.k + page * a.cache.k_page_stride + place * a.cache.k_slot_stride + (h - a.n_q) * a.cache.k_head_stride;
        else dst = a.cache.v + page * a.cache.v_page_stride + place * a.cache.v_slot_stride + (h - a.n_q - a.n_kv) * a.cache.v_head_stride;
        if (live && (is_q || kept)) {
            if (has0) store_vec<VEC>(dst + at0, u0);
            if (has1) store_vec<VEC>(dst + at1, u1);
        }
    }
}

template <int VEC>
static void launch_rope(const RopeArgs& a, int gl, hipStream_t stream)
{
    const int H = a.n_q + 2 * a.n_kv, at_once = 64 / gl;
    const int steps = (H + at_once - 1) / at_once;
    const int64_t units = a.M * steps;
    const int64_t blocks = (units + 3) / 4;
#define W2_ROPE(GL) hipLaunchKernelGGL((qk_norm_rope_kernel<VEC, GL>), dim3((unsigned)blocks), dim3(256), 0, stream, a, steps, at_once)
    switch (gl) {
    case 1: W2_ROPE(1); break;
    case 2: W2_ROPE(2); break;
    case 4: W2_ROPE(4); break;
    case 8: W2_ROPE(8); break;
    case 16: W2_ROPE(16); break;
    case 32: W2_ROPE(32); break;
    default: W2_ROPE(64); break;
    }
#undef W2_ROPE
}

int launch_qk_norm_rope(const RopeArgs& a, hipStream_t stream)
{
    // runs of 8 numbers need the second half of the rotated part, and what follows it, to start at a multiple of 8
    const int vec = a.interleaved || a.rd % 16 == 0 ? 8 : 2;
    const int lanes = (a.D + 2 * vec - 1) / (2 * vec);
    int gl = 1;
    while (gl < lanes) gl *= 2;
    if (vec == 8) launch_rope<8>(a, gl, stream);
    else launch_rope<2>(a, gl, stream);
    return check_launch("w2_qk_norm_rope");
}

}  // namespace w2
