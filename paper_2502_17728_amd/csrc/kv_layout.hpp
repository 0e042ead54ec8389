// kv_layout.hpp -- the paged key/value cache's layout and the launch rules of what writes and
// reads it.  Host and device code without HIP calls, so that the rules can be tested without a GPU.
//
// A page holds 64 tokens; a block is one key/value head of one page: K codes, V codes, 64 K scales,
// 64 V scales (fp32).  Codes lie in MFMA operand order, 1 KiB fragment chunks of 64 lanes x 16
// bytes, so that a wave loads a chunk with one contiguous instruction and a lane's 16 bytes (E
// elements) are its operand, with no pass through LDS and no exchange between lanes:
//   K chunk (tile, c):  lane (row, g) holds the token of `row`, dimensions 4E c + E g ..+E.
//   V chunk (u, n):     lane (row, g) holds dimension 16 n + row of tokens 4E u + E g ..+E.
// The scores of a K tile leave lane (query, a) with the tokens of rows 4a .. 4a+3.  Token
// 4E u + E a + 8 j + 4 t + i is row 4a + i of tile 2 (E/8 u + j) + t, so the lane's scores of the
// two tiles t = 0, 1 are the tokens 4E u + E a + 8 j ..+8: one operand fragment of the product with V.
#pragma once
#include <algorithm>
#include <stddef.h>
#include <stdint.h>

#if defined(__HIP__)
#define DN_HD __host__ __device__ __forceinline__
#else
#define DN_HD inline
#endif

namespace dn {

constexpr int kKvPage = 64;
constexpr int kKvBf16 = 1, kKvFp8 = 2;  // formats (dn.h: DN_KV_BF16, DN_KV_FP8)
constexpr float kFp8Max = 448.0f;       // largest e4m3
constexpr float kFp8Least = 7.52316384526264e-37f;  // 2^-120: keeps 1 / scale finite

template <int FMT, int D>
struct KvBlock {
    static constexpr int BYTES = FMT == kKvBf16 ? 2 : 1;  // per element
    static constexpr int E = 16 / BYTES;                  // elements of a lane's 16 bytes
    static constexpr int PART = kKvPage * D * BYTES;      // K codes, V codes
    static constexpr int KS = 2 * PART, VS = KS + 4 * kKvPage;
    static constexpr int SIZE = VS + 4 * kKvPage;
    // byte of token o, dimension x, in the K codes and in the V codes
    static DN_HD int k_at(int o, int x) {
        const int tile = (o / (4 * E) * (E / 8) + o % E / 8) * 2 + o % 8 / 4, row = o / E % 4 * 4 + o % 4;
        return (((tile * (D / (4 * E)) + x / (4 * E)) * 4 + x / E % 4) * 16 + row) * 16 + x % E * BYTES;
    }
    static DN_HD int v_at(int o, int x) {
        return (((o / (4 * E) * (D / 16) + x / 16) * 4 + o / E % 4) * 16 + x % 16) * 16 + o % E * BYTES;
    }
};

inline size_t kv_block_bytes(int64_t d, int format) {
    return (size_t)(2 * kKvPage * d * (format == kKvBf16 ? 2 : 1) + 8 * kKvPage);
}

// ------------------------------------------------------------------- attention over the cache
// Work is dealt on the device, where the lengths are.  Of sequence b the n g query rows of one
// key/value head (n new tokens, g query heads) make tiles of `rows`; a tile's keys are cut into
// chunks of `chunk` pages, chunk = ceil(pages of all tiles and heads / target), at least `least`.
// Each (tile, chunk, head) is one workgroup, so all have about the same work whatever the lengths.
// Chunks of a tile that has several leave partial sums, which a second kernel merges.
struct CachePlan {
    int rows;        // query rows per tile: 16 (keys straight to registers) or 64, 128 (through LDS)
    int64_t target;  // workgroups aimed at
    int64_t least;   // pages per chunk at least
    int64_t grid;    // workgroups at most
    int64_t slots;   // partial sums at most
};

// every tile's chunks: at most one more than an even share each, and no more than the table holds
inline CachePlan cache_plan(int64_t T, int64_t B, int64_t heads, int64_t group, int64_t table_width, int rows,
                            bool always_partial) {
    CachePlan p;
    p.rows = rows;
    p.target = rows == 16 ? 768 : rows == 256 ? 256 : 512;
    p.least = rows == 16 ? 8 : 4;
    const int64_t tiles = std::min(T * group, T * group / rows + std::min(B, T));
    const int64_t most = (table_width + p.least - 1) / p.least;  // chunks of one tile
    p.grid = heads * tiles > INT64_MAX / most ? p.target + heads * tiles
                                              : std::min(p.target + heads * tiles, heads * tiles * most);
    // several chunks of a tile are at most twice its even share
    p.slots = always_partial ? p.grid : most < 2 ? 0 : std::min(2 * p.target, p.grid);
    return p;
}

// Tiles of 16 rows while the sequences have no more rows than that on average; keys are then used
// once and go straight to registers.
inline int cache_rows(int64_t T, int64_t B, int64_t group) {
    if (T * group <= 16 * B) return 16;
    return T * group <= 64 * B ? 64 : T * group <= 128 * B ? 128 : 256;
}

inline size_t cache_slot_bytes(int rows, int64_t d) { return (size_t)rows * (size_t)(d + 4) * sizeof(float); }

// Workspace: what each sequence's chunks are (16 bytes each), then the partial sums; behind a
// shared prefix (one sequence of all T tokens) the prefix's own first.
struct CacheWorkspace {
    CachePlan own, prefix;
    size_t info, prefix_slots, own_slots, total;
};
inline CacheWorkspace cache_workspace(int64_t T, int64_t B, int64_t heads, int64_t group, int64_t d, int64_t table_width,
                                      int64_t prefix_pages) {
    CacheWorkspace w;
    w.own = cache_plan(T, B, heads, group, table_width, cache_rows(T, B, group), prefix_pages > 0);
    w.info = 0;
    w.prefix_slots = (size_t)(B + 1) * 16;
    w.prefix_slots = (w.prefix_slots + 255) / 256 * 256;
    w.own_slots = w.prefix_slots;
    w.prefix = CachePlan{};
    if (prefix_pages > 0) {
        w.prefix = cache_plan(T, 1, heads, group, prefix_pages, cache_rows(T, 1, group), true);
        w.own_slots += (size_t)w.prefix.slots * cache_slot_bytes(w.prefix.rows, d);
    }
    w.total = w.own_slots + (size_t)w.own.slots * cache_slot_bytes(w.own.rows, d);
    return w;
}

}  // namespace dn
