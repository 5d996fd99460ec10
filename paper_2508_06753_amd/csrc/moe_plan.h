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

inline int64_t most_tiles(int64_t A, int E, int rows) { return std::min<int64_t>(A, E + A / rows); }

struct Plan {
    bool few;                           // the kernel for few rows, or the one for many
    int rows;                           // of a tile, at most
    int64_t tiles;                      // at most
    int ks_up, ks_down;                 // few: ranges (1, 2) that the four waves of a workgroup cut K into
};

// pairs: of column blocks; used: tiles that are likely there
inline int ranges(int64_t used, int64_t pairs, int64_t n_kt) { return used * (pairs / 4) < 768 && n_kt >= 8 ? 2 : 1; }

// Choices per expert up to which the kernel for few rows takes them.  It reads an expert's weights once for every eight rows,
// the other one once for 32 and is bound by issue.  us a call at 6, 8 choices an expert (128 of 4096 x 1024, groups of 128): few 102, 114, many 101, 108; at 8, 16
// with groups of 64, whose products the matrix pipe does in halves (32 of 5120 x 2048): 87, 131 and 91, 119 (so they cross between the two; 16 is from before
// the kernel for many wrote its sums straight from registers, when it took 102 and 140).
constexpr int few_per_expert(int G) { return G == 128 ? 6 : 16; }

inline Plan plan(int64_t hidden, int64_t inter, int E, int G, int64_t A)
{
    Plan p;
    const int64_t used = std::min<int64_t>(A, E);
    p.few = A <= few_per_expert(G) * used;
    p.rows = p.few ? 8 : 32;
    p.tiles = most_tiles(A, E, p.rows);
    p.ks_up = ranges(used, inter / 16, hidden / 256);
    p.ks_down = ranges(used, hidden / 32, inter / 256);
    return p;
}

// Up to 64 choices (a lane of a wave each) and not too many weights: two launches that need nothing prepared, where the others are four.
// Their workgroups bring in all of their rows before the first product, which long streams of weights do not make up for.  us a call, two launches and four:
// 4096 x 1024, top 8, 1 to 4 tokens 15, 21, 31 and 22, 25, 34, 8 tokens 48 and 44; 5120 x 2048 with groups of 64, top 4, 1 and 2 tokens 23, 39 and 26, 31.
struct Tiny {
    bool fits;
    int tiles, rows;                    // at most, and rows of a tile
    int units;                          // groups of two pairs of blocks that a workgroup takes one behind the other
    size_t lds;                         // rows and their exponents
    size_t lds_all;                     // and what leaves: all that the gate and up launch asks for (its kernel declares none beside it)
};

// The gate and up launch's waves: two pairs of blocks times four ranges of K.  What leaves, in front of the rows: the sums of three ranges, or two
// parts of h with the largest numbers (fewer), and the choice that each row is.
constexpr int TINY_P = 2, TINY_KS = 4;
constexpr size_t TINY_SUMS = (TINY_KS - 1) * TINY_P * 2048, TINY_LEAVE = TINY_SUMS + 8 * 4, TINY_MOST_ROWS = (size_t)128 << 10;
static_assert(TINY_LEAVE % 16 == 0 && TINY_P * 16 * 36 <= TINY_SUMS && TINY_MOST_ROWS + TINY_LEAVE <= (size_t)160 << 10, "a CU's local memory");

inline Tiny tiny(int64_t hidden, int64_t inter, int E, int G, int64_t A)
{
    Tiny t;
    t.tiles = (int)most_tiles(A, E, 8);
    t.rows = (int)std::min<int64_t>(A, 8);                    // (or of x, where two of those are all)
    t.lds = (size_t)t.rows * (row_bytes(hidden) + 16 + exp_bytes(hidden));
    t.lds_all = t.lds + TINY_LEAVE;
    t.fits = A <= 64 && t.lds <= TINY_MOST_ROWS && t.tiles * hidden * inter <= (int64_t)1 << (G == 128 ? 27 : 26);
    const int64_t groups = inter / 32;
    t.units = 1;
    while (t.units < 8 && groups % (2 * t.units) == 0 && t.tiles * (groups / (2 * t.units)) >= 512) t.units *= 2;
    return t;
}

// Loads of a wave of the kernel for many rows that may still be under way at its counted waits (vector memory operations complete in order).  rt: row
// tiles of 16, and so its loads of rows in a stage of 128 of K.  Rows are asked for three stages ahead, at a stage's barrier; a tile of 256 of K's weights
// (4), scales (4) and exponents (rt) behind every second stage.
constexpr int TILE_AHEAD = 3;
constexpr int tile_weights(int rt) { return 8 + rt; }
// before the first stage, whose rows have landed: those of two more, and the second tile's weights
constexpr int tile_at_start(int rt) { return (TILE_AHEAD - 1) * rt + tile_weights(rt); }
// at the barrier of stage s: the rows of s + 1 have landed, which were asked for at that of s - 2; those of s + 2 and one tile's weights since
constexpr int tile_at_stage(int rt) { return (TILE_AHEAD - 2) * rt + tile_weights(rt); }

struct Workspace {                      // offsets in bytes, each a multiple of 256; none shrinks when M grows
    size_t tiles, tile_rows, place, xs, xe, hs, he, z;
    size_t ze;                          // room that no kernel uses, a byte for 32 sums: whoever walks the workspace finds it here
    size_t total;
};

// Rows that go together: their two parts lie within 2 GiB, offsets in 32 bits reach them, and their sums within 4 GiB
inline int64_t most_rows(int64_t hidden, int64_t inter, int top_k)
{
    const int64_t rows = std::min(((int64_t)1 << 31) / (int64_t)row_bytes(hidden),
                                  ((int64_t)1 << 31) / (top_k * std::max<int64_t>((int64_t)row_bytes(inter), hidden * 2)));
    return std::max<int64_t>(rows, 1);
}

inline Workspace workspace(int64_t hidden, int64_t inter, int E, int G, int64_t M, int top_k)
{
    M = std::min(M, most_rows(hidden, inter, top_k));
    const int64_t A = M * top_k;
    Workspace w;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    w.tiles = take(256 + (size_t)most_tiles(A, E, 8) * 16); // their number, and the tiles; the shortest ones are the most
    const Plan p = plan(hidden, inter, E, G, A);
    w.tile_rows = take((size_t)p.tiles * p.rows * 4);
    w.place = take((size_t)A * 4);
    w.xs = take((size_t)M * row_bytes(hidden));
    w.xe = take((size_t)M * exp_bytes(hidden));
    w.hs = take((size_t)A * row_bytes(inter));
    w.he = take((size_t)A * exp_bytes(inter));
    w.z = take((size_t)A * hidden * 4);
    w.ze = take((size_t)A * hidden / 32);
    w.total = at;
    return w;
}

}  // namespace moe
}  // namespace w2
