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

// ------------------------------------------------------------------- writing
constexpr int kAppendTile = 16;  // tokens of a workgroup at most
// Tokens of a workgroup, which takes one key/value head of them: as few as give its 256 threads an item
// each (two pieces of 8 elements), and 16, which fill V's pieces, once those alone fill the chip.
// Measured at 4 / 8 / 16 tokens, us: 32 query and 8 key/value heads of 128, fp8, 32 tokens 4.6 / 6.0 / 7.3,
// 1000 tokens 9.4 / 9.2 / 9.4, 2048 tokens 16.2 / 16.0 / 13.6, 4096 tokens 28.3 / 26.4 / 23.2; 12 and 12 heads
// of 64, bf16, 1000 tokens 8.7 / 6.6 / 6.0.  (32 tokens: 7.1 for the last, 23.0 for the one before, 16.4 at 2048.)
inline int append_tile(int64_t tokens, int64_t heads, int64_t group, int64_t d) {
    if ((tokens + kAppendTile - 1) / kAppendTile * heads >= 768) return kAppendTile;
    const int64_t items = (group + 2) * d / 16;
    return 4 * items > 128 ? 4 : 8 * items > 128 ? 8 : kAppendTile;
}

// ------------------------------------------------------------------- attention over the cache
// Work is dealt on the device, where the lengths are.  Of sequence b the n g query rows of one
// key/value head (n new tokens, g query heads) make tiles of `rows`.  Two deals:
// - chunks: a tile's keys are cut into equal chunks of at most `per` pages, per = ceil(pages of all
//   tiles and heads / target), at least `least`; each (tile, chunk, head) is a workgroup, which finds
//   itself by a scan of the lengths.  For work whose chunks are short.
// - runs: a kernel before lists, for each of `target` workgroups, an equal stretch of all tiles' keys.
//   It costs a launch; chunks of uneven tiles leave more of the chip idle once they are long.
//   Measured, tiles of 256 rows in chunks / in runs, us, fp8, 32 query over 8 key/value heads of 128: two chunks of
//   1000 tokens against 8191 keys 302 / 250, four of 500 against 4096 153 / 137, two of 512 against 2048 78.7 / 67.1, four
//   ragged ones 272 / 233, 2048 against 16384 496 / 500.  Prompts with nothing cached before them go the other way, of
//   4096 tokens 164 / 191, of 1024 39.1 / 48.5, eight of 1024 131 / 150; the lengths, which would tell, are on the device.
// A tile that is cut leaves partial sums, which a last kernel merges.
struct CachePlan {
    int rows;        // query rows per tile: 16 (keys straight to registers), 64, 128 or 256 (through LDS)
    bool in_runs;
    int64_t target;  // workgroups aimed at
    int64_t least;   // pages per chunk or run at least
    int64_t tiles;   // at most, over all heads
    int64_t grid;    // workgroups launched
    int64_t slots;   // partial sums at most
};

// Tiles of 16 rows while the sequences have no more rows than that on average; keys are then used
// once and go straight to registers.  Measured at rows 16 / 64 / 128 / 256, us: 8 sequences of n tokens
// with 32 query and 8 key/value heads of 128, 4096 keys, fp8: n = 4 21.9 / 26.8 / 32.9 / 53.8, n = 5 28.9 / 27.1 /
// 33.2 / 55.2, n = 16 38.5 / 29.8 / 35.6 / 54.8, n = 17 45.0 / 39.6 / 35.9 / 54.6, n = 64 80.8 / 67.8 / 57.4 / 62.8;
// 128 / 256: n = 96 107 / 100, n = 384 266 / 244.  bf16: n = 4 31.5 / 31.2 / 33.8 / 49.1, n = 5 41.5 / 31.3 / 34.4 / 49.8,
// n = 17 71.8 / 37.6 / 37.5 / 53.5, n = 64 152 / 61.9 / 56.4 / 60.1; n = 96 98 / 92.
// The mean serves calls of like sequences.  Calls that mix a chunk and single tokens, us, against the two as
// calls of their own: 2048 tokens beside 31 single ones, 8192 keys each 538 / 257 + 89 (single tokens in tiles of 256
// rows), 512 beside 31, bf16, 4096 keys 162 / 62 + 87, 512 beside 255, 2048 keys 222 / 54 + 183, 300 beside 7, 4096 keys
// 76 / 61 + 17.
inline int cache_rows(int64_t T, int64_t B, int64_t group) {
    const int64_t rows = (T * group + B - 1) / B;
    return rows <= 16 ? 16 : rows <= 64 ? 64 : rows <= 256 ? 128 : 256;
}

inline CachePlan cache_plan(int64_t T, int64_t B, int64_t heads, int64_t group, int64_t table_width, int rows,
                            bool prefix, bool always_partial) {
    CachePlan p;
    p.rows = rows;
    // A prefix's tiles share the chip with the sequences' own keys, and its partial sums are the more the
    // more it is cut.  Measured, us, fp8, 32 query over 8 key/value heads of 128.  16 rows, 32 sequences of up to 8192
    // keys, 512 / 768 / 1024 / 1536: 76.0 / 75.1 / 77.0 / 79.3.  64 and 128 rows, 256 / 512 / 1024: 8 sequences of 16 tokens, 4096
    // keys 34.5 / 31.0 / 43.1, of 64 70.8 / 53.4 / 64.9, 32 of 16, 1024 keys 31.5 / 28.9 / 37.0.  256 rows, 256 / 512: two chunks of 1000
    // against 8191 keys 247 / 261, 2048 against 16384 498 / 521, four ragged prompts 128 / 137.  Behind a prefix, 128 / 256 /
    // 512: 64 sequences, 8192 keys 44.4 / 33.6 / 41.8, 128 69.7 / 49.6 / 59.3, 16 21.8 / 21.2 / 21.8; 30000 keys 117 / 69 / 62.
    p.target = rows == 16 ? 768 : rows == 256 || prefix ? 256 : 512;
    // 16 rows at 4 / 8 / 16: one sequence of 8192 keys 12.0 / 12.4 / 14.1, four of 2000 11.9 / 11.8 / 14.1, 16 of 4096 30.0 / 30.1 / 27.2,
    // 256 of up to 1000 67.0 / 67.1 / 62.0.  Others at 2 / 4 / 8: two of 16 tokens, 8192 keys 21.3 / 21.5 / 22.8, 64 sequences behind
    // 8192 keys 34.8 / 33.6 / 33.6, behind 2000 29.8 / 26.2 / 28.5.
    p.least = rows == 16 && !prefix ? 8 : 4;
    p.tiles = heads * std::min(T * group, T * group / rows + std::min(B, T));
    const int64_t most = (table_width + p.least - 1) / p.least;  // chunks of one tile
    p.in_runs = rows == 256 && !prefix && !always_partial && most > 1;
    // every tile's chunks: at most one more than an even share each, and no more than the table holds
    p.grid = p.in_runs ? p.target : p.tiles > INT64_MAX / most ? p.target + p.tiles : std::min(p.target + p.tiles, p.tiles * most);
    // several chunks of a tile are at most twice its even share; a run cuts two tiles
    p.slots = always_partial ? p.grid : most < 2 ? 0 : p.in_runs ? 2 * p.target : std::min(2 * p.target, p.grid);
    return p;
}

inline size_t cache_slot_bytes(int rows, int64_t d) { return (size_t)rows * (size_t)(d + 4) * sizeof(float); }

// Workspace: 16 bytes for each sequence and for the shared prefix (one sequence of all T tokens), the
// runs' lists (8 bytes a run and a tile, 24 a piece), then the partial sums.
struct CacheWorkspace {
    CachePlan own, prefix;
    size_t own_info, prefix_info, own_runs, own_parts, prefix_parts, total;
};
inline CacheWorkspace cache_workspace(int64_t T, int64_t B, int64_t heads, int64_t group, int64_t d, int64_t table_width,
                                      int64_t prefix_pages) {
    CacheWorkspace w;
    w.own = cache_plan(T, B, heads, group, table_width, cache_rows(T, B, group), false, prefix_pages > 0);
    w.own_info = 0;
    w.prefix_info = (size_t)B * 16;
    w.own_runs = w.prefix_info + 16;
    w.own_parts = w.own_runs;
    if (w.own.in_runs) w.own_parts += (size_t)(w.own.target + w.own.tiles) * (8 + 24);
    w.own_parts = (w.own_parts + 255) / 256 * 256;
    w.prefix_parts = w.own_parts + (size_t)w.own.slots * cache_slot_bytes(w.own.rows, d);
    w.total = w.prefix_parts;
    w.prefix = CachePlan{};
    if (prefix_pages > 0) {
        // beside tiles of 16 rows the prefix's go without the second half of 256 rows
        const int rows = cache_rows(T, 1, group);
        w.prefix = cache_plan(T, 1, heads, group, prefix_pages, w.own.rows == 16 ? std::min(rows, 128) : rows, true, true);
        w.total += (size_t)w.prefix.slots * cache_slot_bytes(w.prefix.rows, d);
    }
    return w;
}

// ------------------------------------------------------------------- runs
// Long tiles are dealt in equal runs.  The work is laid on a line: sequences, of each its key/value
// heads, of each its tiles, of each its pages.  A tile weighs the query-key pairs of its rows' largest
// query, times `group`, and a start; a sequence's tiles then sum to a closed form.  Every run is an
// equal stretch of the line, so all end together whatever the lengths.  A tile that several runs
// share leaves partial sums, two slots to a run at most: its first tile's and its last's.

// A run's share of a tile: pages [lo, hi), and where its partial sums go (kWhole: it has all pages and
// writes the output; kNone: no pages).
struct Piece {
    int b, head, tile, lo, hi, slot;
};
constexpr int kWhole = -1, kNone = -2;

struct Seq {
    int first, n, len, pages;  // first token, tokens, keys, pages of keys
};

struct Weights {
    int64_t each, more;  // tile t weighs each + (t + 1) more
    DN_HD int64_t before(int64_t t) const { return t * each + more * (t * (t + 1) / 2); }
    DN_HD int64_t of(int64_t t) const { return each + (t + 1) * more; }
};
// A tile's start and end, in keys.  Measured at 128 / 256 / 512 / 1024 / 2048, us, 32 query over 8 key/value heads of
// 128, fp8: two chunks of 1000 tokens against 8191 keys 251 / 246 / 246 / 244 / 245, four of ragged tokens and keys
// (1000 of 9000, 500 of 500, 400 of 4000, 900 of 1500) 305 / 258 / 231 / 239 / 253, a prompt of 4096 220 / 190 / 189 / 195 /
// 209, of 1024 53.7 / 44.5 / 48.4 / 49.5 / 51.2, four ragged ones 147 / 129 / 128 / 138 / 148, two of 512 against 2048
// 66.6 / 66.6 / 67.4 / 66.9 / 68.1; 2048 against 16384 498 to 496 at any.
constexpr int kStart = 512;
DN_HD Weights weights(const Seq& s, int group, int rows) {
    const int behind = s.len - s.n;
    return Weights{(int64_t)((behind > 0 ? behind : 0) + kStart) * group, rows};
}
DN_HD int tiles_of(const Seq& s, int group, int rows) { return (int)(((int64_t)s.n * group + rows - 1) / rows); }

// Row and head numbers: the host refuses calls whose rows (T * group, rounded up to a tile) pass 31 bits, so
// their quotients are 32-bit ones, a third of a 64-bit one's instructions.
DN_HD int quotient32(int64_t a, int b) { return (int)((uint32_t)a / (uint32_t)b); }

// Keys that some query of the tile sees, where each sees those up to its own.
DN_HD int seen_keys(int n, int len, int group, int tile, int rows) {
    const int row = quotient32((int64_t)tile * rows + rows - 1, group), last = row < n - 1 ? row : n - 1;
    const int keys = len - n + last + 1;
    return keys < 0 ? 0 : keys < len ? keys : len;
}

// Where the line cuts a tile that weighs `weight` for `pages`: the page `at` into it, which grows with `at`;
// nobody is left a single page.
struct Cuts {
    int64_t weight;
    int pages;
    double scale;
    DN_HD Cuts(int64_t w, int p) : weight(w), pages(p), scale((double)p / (double)w) {}
    DN_HD int page(int64_t at) const {
        if (at <= 0) return 0;
        if (at >= weight) return pages;
        const int p = (int)((double)at * scale);
        return p < 2 ? 0 : pages - p < 2 ? pages : p;
    }
};

// a / b for 0 <= a, 0 < b: through doubles, which are far shorter than the 64-bit division
DN_HD int64_t quotient(int64_t a, int64_t b) {
    int64_t q = (int64_t)((double)a / (double)b);
    if (q * b > a) --q;
    if ((q + 1) * b <= a) ++q;
    return q;
}

// The line: `target` runs of `per` each, the last one shorter.
struct Line {
    int64_t B, heads, target, total, per;
    int group, rows;
    int64_t tiles_most;
};
DN_HD int64_t run_length(int64_t total, int64_t target, int64_t least, int group) {
    const int64_t even = quotient(total + target - 1, target), short_one = least * kKvPage * group;
    return even > short_one ? even : short_one;
}

// Lists the pieces of one run, which starts in sequence b (its first tile `b_start` on the line and
// number `b_tiles` of all).  Piece (tile + run) of the line: both only grow.  sequence(b) gives the
// lengths, piece(i, ...) and tile(i, first piece, pieces) take what is found; the first piece and
// their number are returned through `first` and `count`.
template <class Sequence, class PieceOut, class TileOut>
DN_HD void deal_run(const Line& line, int64_t run, int64_t b, int64_t b_start, int64_t b_tiles, Sequence&& sequence,
                    PieceOut&& piece_out, TileOut&& tile_out, int& first, int& count) {
    const int64_t per = line.per, x0 = run * per, x1 = x0 + per < line.total ? x0 + per : line.total;
    first = count = 0;
    if (b < 0 || x0 >= x1) return;
    const int group = line.group, rows = line.rows;
    Seq s = sequence(b);
    Weights w = weights(s, group, rows);
    int tiles = tiles_of(s, group, rows);
    const int64_t head_weight = w.before(tiles);
    int head = (int)quotient(x0 - b_start, head_weight);
    const int64_t at = x0 - b_start - head * head_weight;
    int tile = 0, high = tiles - 1;  // the last tile that starts at `at` or before
    while (tile < high) {
        const int mid = (tile + high + 1) >> 1;
        if (w.before(mid) <= at)
            tile = mid;
        else
            high = mid - 1;
    }
    int64_t x = x0 - at + w.before(tile);  // where the tile starts
    int64_t ordinal = b_tiles + (int64_t)head * tiles + tile;
    first = (int)(ordinal + run);
    while (true) {
        const int64_t weight = w.of(tile), piece = ordinal + run;
        const int pages = (seen_keys(s.n, s.len, group, tile, rows) + kKvPage - 1) / kKvPage;
        const Cuts cuts(weight, pages);
        const int lo = cuts.page(x0 - x), hi = cuts.page(x1 - x);
        if (ordinal >= line.tiles_most) break;  // q_start out of order
        const int slot = (int)(2 * run) + (x > x0 ? 1 : 0);
        piece_out(piece, Piece{(int)b, head, tile, lo, hi,
                               lo == 0 && hi == pages && (pages > 0 || x >= x0) ? kWhole : lo < hi ? slot : kNone});
        if (x >= x0) {
            const int64_t last = x + weight <= x1 ? run : quotient(x + weight - 1, per);
            // The tile is divided where some cut leaves pages on both sides: the first one that leaves any
            // before it tells, for cuts only grow.  It is mostly the run's own end, else found by bisection,
            // whatever the tile weighs for its pages (queries before the first key weigh like others and
            // see none).
            int cut = hi;
            if (last > run && cut == 0) {
                int64_t r = run + 2, end = last;
                while (r < end) {
                    const int64_t mid = (r + end) >> 1;
                    if (cuts.page(mid * per - x) == 0)
                        r = mid + 1;
                    else
                        end = mid;
                }
                if (r <= last) cut = cuts.page(r * per - x);
            }
            const bool divided = last > run && cut > 0 && cut < pages;
            tile_out(ordinal, (int)piece, divided ? (int)(last - run) + 1 : 0);
        }
        ++count;
        x += weight;
        if (x >= x1) break;
        ++ordinal;
        if (++tile < tiles) continue;
        tile = 0;
        if (++head < line.heads) continue;
        head = 0;
        do
            if (++b >= line.B) break;
        while ((tiles = tiles_of(s = sequence(b), group, rows)) == 0);
        if (b >= line.B) break;
        w = weights(s, group, rows);
    }
}

}  // namespace dn
