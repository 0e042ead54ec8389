// fp8_rules.hpp -- layout of the 8-bit products' weights, and which kernel takes a call of the 8-bit
// products, of the rows that feed them and of the log probabilities.  Host code without HIP, so
// that the rules can be evaluated (and are tested) without a GPU.
#pragma once
#include <algorithm>
#include <stddef.h>
#include <stdint.h>

namespace dn {

// ------------------------------------------------------------------------------- rows
// Longest rows: 8 pieces of 8 values to each of 1024 threads; fp32 rows, twice the registers, half.
constexpr int64_t kMaxRowBf16 = 65536, kMaxRowF32 = 32768;

struct RowPlan {
    int threads, pieces;  // per row; pieces of 8 values per thread
};
inline RowPlan plan_rows(int64_t M, int64_t K) {
    const int64_t pieces = K / 8;
    const int threads = pieces <= 128 ? 64 : (pieces <= 1024 && M >= 256) ? 256 : pieces <= 256 ? 256 : 1024;
    int per = 1;
    while ((int64_t)threads * per < pieces) per *= 2;
    return RowPlan{threads, per};
}

// ------------------------------------------------------------------------------- weights
struct Fp8Layout {
    int64_t kchunks, blocks;  // 64-byte chunks along K (K padded to 128), blocks of 16 packed columns
    size_t scales, bias, total;
};
inline Fp8Layout fp8_layout(int64_t K, int64_t N, int gated) {
    Fp8Layout l;
    l.kchunks = (K + 127) / 128 * 2;
    l.blocks = (N + 15) / 16 * (gated ? 2 : 1);
    l.scales = (size_t)l.blocks * l.kchunks * 1024;
    l.bias = l.scales + (size_t)l.blocks * 64;
    l.total = l.bias + (size_t)l.blocks * 64;
    return l;
}

// ------------------------------------------------------------------------------- products
enum class Fp8Kernel { kRing };
struct Fp8Plan {
    Fp8Kernel kernel;
    int bm, bn;      // tile
    int64_t splits;  // of K
};
constexpr int64_t kMaxSplits = 16;

inline Fp8Plan plan_fp8(int64_t M, int64_t K, int64_t blocks, int64_t splits_that_fit) {
    Fp8Plan p{Fp8Kernel::kRing, 64, 64, 1};
    const int64_t tiles = (M + 63) / 64 * ((blocks + 3) / 4), stages = (K + 127) / 128;
    p.splits = std::max<int64_t>(1, std::min({256 / tiles, stages / 8, kMaxSplits, splits_that_fit}));
    return p;
}
// fp32 partial sums of one split
inline size_t fp8_partial_bytes(int64_t M, int64_t blocks) { return (size_t)M * blocks * 64; }
inline size_t fp8_workspace(int64_t M, int64_t K, int64_t blocks) {
    const Fp8Plan p = plan_fp8(M, K, blocks, kMaxSplits);
    return p.splits > 1 ? p.splits * fp8_partial_bytes(M, blocks) : 0;
}

// ------------------------------------------------------------------------------- log probabilities
constexpr int64_t kMaxTop = 64, kMaxSegments = 64;

// Workgroups to a row.
inline int64_t logprob_segments(int64_t T, int64_t V) {
    const int64_t by_chip = (1024 + T - 1) / T, by_row = V / 4096;
    return std::max<int64_t>(1, std::min({by_chip, by_row, kMaxSegments}));
}
// A segment leaves its maximum, denominator and entropy sum (16 bytes) and `top` ranked keys of 8 bytes.
inline size_t logprob_workspace(int64_t T, int64_t V, int64_t top) {
    const int64_t s = logprob_segments(T, V);
    return s > 1 ? (size_t)T * s * (16 + 8 * top) : 0;
}

}  // namespace dn
