// How the rows and columns of w2_moe_experts are cut into workgroups, and where things lie in its workspace.  Host code.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/w2mm.h"

namespace w2 {
namespace moe {

// A row of x or h as the matrix instructions take it: 512 bytes for 256 numbers, and 8 bytes of exponents beside them.
constexpr size_t row_bytes(int64_t K) { return (size_t)K * 2; }
constexpr size_t exp_bytes(int64_t K) { return (size_t)K / 32; }

struct Workspace {                      // offsets in bytes, each a multiple of 256; none shrinks when M grows
    size_t tiles, sorted, place, xs, xe, hs, he, z, total;
};

inline int64_t most_tiles(int64_t A, int E, int rows) { return std::min<int64_t>(A, E + A / rows); }

inline Workspace workspace(int64_t hidden, int64_t inter, int E, int64_t M, int top_k)
{
    const int64_t A = M * top_k;
    Workspace w;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    w.tiles = take((size_t)most_tiles(A, E, 16) * 16);       // the shortest tiles are the most
    w.sorted = take((size_t)A * 4);
    w.place = take((size_t)A * 4);
    w.xs = take((size_t)M * row_bytes(hidden));
    w.xe = take((size_t)M * exp_bytes(hidden));
    w.hs = take((size_t)A * row_bytes(inter));
    w.he = take((size_t)A * exp_bytes(inter));
    w.z = take((size_t)A * hidden * 4);
    w.total = at;
    return w;
}

// Row tiles of 16 a workgroup's wave holds (rt) and the ranges that its waves cut K into (ks).
struct Shape {
    int rt, ks;
};

inline int pick_rt(int64_t A, int E)
{
    const int64_t used = std::min<int64_t>(A, E), per = A / used;
    return per <= 8 ? 1 : per <= 24 ? 2 : 4;
}

// blocks: workgroups of eight waves without ranges
inline int pick_ks(int rt, int64_t blocks, int64_t n_kt)
{
    int ks = 1;
    while (ks < 4 && rt * ks < 4 && blocks * ks < 512 && n_kt >= 4 * ks) ks *= 2;
    return ks;
}

}  // namespace moe
}  // namespace w2
