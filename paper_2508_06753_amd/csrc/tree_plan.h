// How the attention of drafted tokens (tree_attention.hip) is cut up: no HIP, so that a test can compile it by itself.
#pragma once
#include <stdint.h>

namespace w2 {

namespace tree {

// A request's 32-row waves (`all`, at least one a tile), spread over its tiles: the first ones take one more where they do not come
// out even.  Quotient and remainder: all times a tile's number passes 32 bits from about 3 million packed rows on.
struct Share {
    int first, count;
};
constexpr Share share(int all, int tiles, int tile)
{
    const int each = all / tiles, more = all % tiles;
    return {each * tile + (tile < more ? tile : more), each + (tile < more ? 1 : 0)};
}

}  // namespace tree

}  // namespace w2
