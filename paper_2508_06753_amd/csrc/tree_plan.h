// How the attention of drafted tokens (tree_attention.hip) is cut up: no HIP, so that a test can compile it by itself.
#pragma once
#include <stdint.h>

#include <algorithm>

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

constexpr int MAX_CHUNKS = 128;

struct Plan {
    int few;                             // tree_few_kernel, else tree_tile_kernel
    int rt;                              // few: 16-row tiles a wave
    int waves;                           // a workgroup
    int dt;                              // head_dim padded to 64, 128 or 256
    int tiles;                           // row tiles of a request
    uint32_t chunk;                      // keys of a workgroup, a multiple of 128, up to 2^31
    int chunks;                          // of the longest request
};

inline Plan make_plan(int64_t n_requests, int64_t max_rows, int G, int n_kv, int D, int64_t max_len, int64_t total_len)
{
    Plan p;
    const int64_t rows = max_rows * G;
    p.dt = D <= 64 ? 64 : D <= 128 ? 128 : 256;
    p.few = rows <= (p.dt < 256 ? 32 : 16);
    p.rt = p.few && rows <= 16 ? 1 : 2;
    p.waves = !p.few && rows <= 64 ? 2 : 4;
    const int rows_per_wg = p.few ? 16 * p.rt : 32 * p.waves;
    p.tiles = (int)((rows + rows_per_wg - 1) / rows_per_wg);
    if (total_len <= 0 || total_len > n_requests * max_len) total_len = n_requests * max_len;
    // (limits far above the batch's own are allowed, and their product is past 64 bits)
    const __int128 all = (__int128)total_len * n_kv * p.tiles;
    const int64_t tile_rows = std::min<int64_t>(rows, rows_per_wg);
    int64_t chunk;
    if (p.few) {
        // workgroups for eight on every CU, each with so many keys that the parts of its rows, written and read again in 32 bits,
        // stay a tenth of them
        chunk = std::max<int64_t>((int64_t)((all + 2047) / 2048), std::max<int64_t>(128, 20 * tile_rows));
    } else {
        // As many workgroups as local memory has room for at once, however the keys are spread over the requests (each may have
        // a last chunk that is not full): a few more would take as long again (us: 16 requests of 36 rows and up to 4100 keys,
        // about 512 workgroups and up to 128 more: 47, at most 512: 36; 7 of 61 rows and up to 34226 keys, 16 heads: 278 and
        // 220; of four waves two share a CU's SIMDs, and what is left of the last one runs faster: half that margin, 320 and
        // 308 for 2 requests of 320 rows and up to 120000 keys).  Where there are more units than that, parts pass through
        // memory and little is gained, up to 48 keys a row (4 requests of 1000 tokens, 5000 keys, in a second chunk: 136 ->
        // 148; 21 of 166 tokens, 7142 keys, 16 heads: 291 -> 282).  Else two keys a row are enough: workgroups without others
        // beside them wait for memory most of the time (8 requests of 434 rows, 2434 keys, 3 heads: 76 in one chunk, 25 + 6 in
        // ten).
        const int64_t units = n_requests * n_kv * p.tiles, room = p.dt == 64 ? 1024 : p.dt == 128 ? 512 : 256;
        const int64_t rounds = std::max<int64_t>(1, (2 * units + room - 1) / room), free = rounds * room - (p.waves == 2 ? units : units / 2);
        chunk = std::max<int64_t>((int64_t)((all + free - 1) / free), (rounds > 1 ? 48 : 2) * tile_rows);
    }
    chunk = std::max(chunk, (max_len + MAX_CHUNKS - 1) / MAX_CHUNKS);
    if (!p.few) chunk = std::max<int64_t>(256, max_len / std::max<int64_t>(1, (max_len + chunk - 1) / chunk) + 1);    // (of one length)
    if (max_rows * G * n_kv >= (int64_t)1 << 24) chunk = std::max(chunk, max_len);     // (more than a grid of the join counts)
    chunk = (chunk + 127) / 128 * 128;
    // a few short requests: eight waves share a request's keys and no second launch joins chunks (us, one request of 8 heads, 700
    // keys: 9.6 against 6.1 + 3.3 and a launch, 1000 keys: 12.2 against 6.2 + 3.4; 16 requests of 1000: 13.6 against 14.3 + 3.6)
    if (p.few && p.rt == 1 && p.dt < 256 && n_requests * n_kv <= 256 && max_len <= (n_requests * n_kv >= 64 ? 1024 : 768)) {
        p.waves = 8;
        chunk = 1024;
    }
    p.chunk = (uint32_t)std::min<int64_t>(chunk, (int64_t)1 << 31);
    p.chunks = (int)std::max<int64_t>(1, (max_len + p.chunk - 1) / p.chunk);
    return p;
}

// No more parts than there is room for (0: none, a chunk is everything): longer chunks.  max_len < 2^31
inline void fit(Plan& p, int64_t max_len, int64_t room)
{
    if (p.chunks <= room) return;
    const int64_t most = std::max<int64_t>(1, room), each = (max_len + most - 1) / most;
    p.chunk = (uint32_t)std::max<int64_t>(128, (each + 127) / 128 * 128);
    p.chunks = (int)std::max<int64_t>(1, (max_len + p.chunk - 1) / p.chunk);
}

}  // namespace tree

}  // namespace w2
