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
// Which kernel takes a call, by estimated time: rounds of workgroups (256 CUs, `per_cu` of them on each), each a
// fixed 1.5 us (first copies, epilogue) and its stages of 128 codes at `stage_us`; never less than W from HBM at 6.2 TB/s.
// Stage times were fitted to calls of one round, us: 64 x 64 tiles 0.235 (two on a CU 0.36 the pair), 64 x 128 0.315,
// 128 x 128 0.46, 256 x 128 0.84, 256 x 256 1.42.  Measured, us, best first:
//   64 rows 4096 -> 12288    64 x 64 11.4, 64 x 128 12.9, 128 x 128 17
//   128 rows 4096 -> 12288   64 x 128 13.2, 64 x 64 14.3, 128 x 128 16.9
//   256 rows 4096 -> 12288   128 x 128 18.2, 64 x 128 24.3
//   512 rows 4096 -> 12288   256 x 128 28.8, 128 x 128 35.5, 256 x 256 42.4
//   1024 rows 4096 -> 12288  256 x 256 48.9, 256 x 128 56.6, 128 x 128 59.8
//   2048 rows 14336 -> 4096  256 x 128 101, 128 x 128 124, 256 x 256 (128 tiles) 128
// K is split where that fills the chip: 100 rows 14336 -> 4096 16.9 us with 8 splits, 17.1 with 4, 19.0 with 2, 26.9 without; the join
// costs a launch and the traffic of the fp32 sums.
constexpr int kFp8Tiles = 5;
struct Fp8Tile {
    int bm, bn, threads, per_cu;
    double stage_us, pair_us;  // one workgroup on a CU, all of per_cu
};
constexpr Fp8Tile kFp8Tile[kFp8Tiles] = {{64, 64, 128, 2, 0.235, 0.36},
                                         {64, 128, 256, 1, 0.315, 0.315},
                                         {128, 128, 256, 1, 0.46, 0.46},
                                         {256, 128, 512, 1, 0.84, 0.84},
                                         {256, 256, 512, 1, 1.42, 1.42}};
constexpr int64_t kMaxSplits = 16;

// tile >= 0: that tile, K in `splits` parts.  tile < 0: streamed (rf 1) or ring (rf 2) kernel, 16 rf rows x nc column blocks.
struct Fp8Plan {
    int tile, rf, nc;
    int64_t splits;
    double us;
};

// fp32 partial sums of one split
inline size_t fp8_partial_bytes(int64_t M, int64_t blocks) { return (size_t)M * blocks * 64; }

// f32: codes widened to bf16, whose products take twice as long; the largest tile has no registers for it.
inline Fp8Plan plan_fp8(int64_t M, int64_t K, int64_t blocks, int gated, int f32, int64_t splits_that_fit) {
    const int64_t stages = (K + 127) / 128;
    const double w_us = (double)blocks * 16 * (double)K / 6.2e6, slow = f32 ? 1.8 : 1.0;
    Fp8Plan best{-1, 0, 0, 1, 0};
    // Up to 64 rows: W streamed into registers (rf 1) or rings of the waves' own (rf 2).  Per step of 128 codes 0.02 us and
    // 0.072 us per column block, or 0.045 and 0.068.  16 rows 4096 -> 4096 5.7 us, 32 rows 6.4, 64 rows 7.2, in tiles 10.4.
    // (5 blocks, which would suit widths of about 20480, are not built.)
    for (int rf = 1; rf <= 2 && M <= 64; ++rf) {
        const int64_t rows = (M + 16 * rf - 1) / (16 * rf);
        static constexpr int kNc[7] = {1, 2, 3, 4, 6, 7, 8};
        for (int nc : kNc) {
            // (7 blocks streamed never win with fp32 outputs: the ring's step is the shorter one, and W's share of HBM does not hide it)
            if ((gated && nc % 2) || (rf == 2 && nc == 8) || (f32 && rf == 1 && nc == 7)) continue;
            const int64_t wgs = rows * ((blocks + nc - 1) / nc);
            const double step = rf == 1 ? 0.02 + 0.072 * nc : 0.045 + 0.068 * nc;
            const double us = 2.7 + std::max(w_us, (double)((wgs + 255) / 256) * (double)stages * step * (f32 ? 1.15 : 1.0));
            if (best.rf == 0 || us < best.us) best = Fp8Plan{-1, rf, nc, 1, us};
        }
    }
    if (M <= 16) return best;
    for (int i = 0; i < (f32 ? kFp8Tiles - 1 : kFp8Tiles); ++i) {
        const Fp8Tile& t = kFp8Tile[i];
        const int64_t tiles = (M + t.bm - 1) / t.bm * ((blocks * 16 + t.bn - 1) / t.bn);
        for (int64_t splits = 1; splits <= std::min(kMaxSplits, splits_that_fit); splits *= 2) {
            if (splits > 1 && (tiles * splits > 512 || stages / splits < 8)) break;
            const int64_t wgs = tiles * splits, per_round = 256 * t.per_cu;
            const double stage = (wgs <= 256 ? t.stage_us : t.pair_us) * slow;
            const int64_t each = (stages + splits - 1) / splits;
            double us = 3.0 + std::max(w_us, (double)((wgs + per_round - 1) / per_round) * (1.5 + (double)each * stage));
            if (splits > 1) us += 3.5 + (double)splits * (double)fp8_partial_bytes(M, blocks) * 2.0 / 6e6;
            if (best.us == 0 || us < best.us) best = Fp8Plan{i, 0, 0, splits, us};
        }
    }
    return best;
}
// Workgroups of the call, and threads to each.
inline int64_t fp8_workgroups(const Fp8Plan& p, int64_t M, int64_t blocks) {
    if (p.tile < 0) return (M + 16 * p.rf - 1) / (16 * p.rf) * ((blocks + p.nc - 1) / p.nc);
    const Fp8Tile& t = kFp8Tile[p.tile];
    return (M + t.bm - 1) / t.bm * ((blocks * 16 + t.bn - 1) / t.bn) * p.splits;
}
inline int fp8_threads(const Fp8Plan& p) {
    return p.tile >= 0 ? kFp8Tile[p.tile].threads : p.rf == 2 && p.nc > 2 ? 256 : 512;
}

// Whether the outputs are stored with the non-temporal hint: those of the 256-row tiles, where rows are whole 64-byte pieces.  They
// then reach HBM beside the products that follow, instead of being written back when these need the cache; broken pieces would go
// there one part at a time.  us with the hint and without: 4096 x 4096 -> 12288 162, 164, -> 2 x 14336 379, 387 (with the
// quantisation of its rows behind it 409, 418), 501 rows of it 52, 53 (58, 58); 6244 x 1088 -> 11712 104, 112, -> 11744 107, 113, -> 11728
// 136, 115, -> 11704 148, 117; in fp32 -> 11712 203, 205, -> 11704 217, 208.
inline bool fp8_streams_out(const Fp8Plan& p, int64_t N, int f32, uintptr_t out) {
    return p.tile >= 0 && kFp8Tile[p.tile].bm >= 256 && N * (f32 ? 4 : 2) % 64 == 0 && out % 64 == 0;
}

inline size_t fp8_workspace(int64_t M, int64_t K, int64_t blocks, int gated) {
    const int64_t splits = std::max(plan_fp8(M, K, blocks, gated, 0, kMaxSplits).splits, plan_fp8(M, K, blocks, gated, 1, kMaxSplits).splits);
    return splits > 1 ? splits * fp8_partial_bytes(M, blocks) : 0;
}

// ------------------------------------------------------------------------------- log probabilities
constexpr int64_t kMaxTop = 64, kMaxSegments = 16;

// Threads to a workgroup and workgroups to a row.  Each wave ranks what it reads by itself, so ranked rows take as few
// waves as fill the chip, and rows without ranks few only if they are short.  Measured, us, with 512, 256, 128 and 64 threads,
// bf16 with 20 alternatives: 300 x 131072 34.6, 37.2, 57.4, -; 1000 x 100003 50.3, 45.9, 49.7, 67.3; 2000 x 8192 28.3, 21.2, 18.0, 18.3;
// 4000 x 32008 90.8, 67.2, 59.1, 53.7; 8000 x 32008 177, 130, 110, 115; 16000 x 8192 195, 120, 88, 68; without alternatives:
// 16000 x 8192 58, 49, 44, 44; 16000 x 1000 -, 28, 20, 12; fp32 4000 x 32008 87.8, 91.2, 96.9, 94.0.
// The rule was fitted to these and asks neither for the type nor for `top`, which costs up to a fifth elsewhere: fp32 with 20
// 4000 x 32008 116, 100, 108, 100, 16000 x 8192 204, 136, 111, 104; bf16 4000 x 32008 with 64 193, 117, 93, 76, with 5 70, 54, 52, 48.
// Fewer than 256 rows get a workgroup to each 16384 tokens while there is about one to a CU; a second kernel then joins
// them: 32 x 131072 17.2 (8 segments; 16: 18.7, 4: 21.0), 1 x 32000 12.4 (2; 1: 13.6), 200 x 32000 16.8 (1; 2: 19.0).
struct LogprobPlan {
    int threads;
    int64_t segments;
};
inline LogprobPlan plan_logprobs(int64_t T, int64_t V, int64_t top) {
    if (T >= 256) {
        const bool shorter = V < 16384;
        if (T < 512) return LogprobPlan{512, 1};
        if (!top) return LogprobPlan{!shorter ? 512 : T >= 2000 && V < 8192 ? 64 : 128, 1};
        return LogprobPlan{T < 2000 ? 256 : shorter && T >= 4000 ? 64 : 128, 1};
    }
    return LogprobPlan{512, std::max<int64_t>(1, std::min({256 / T, (V + 8192) / 16384, kMaxSegments}))};
}
// A segment leaves its maximum, denominator and entropy sum (16 bytes) and `top` ranked keys of 8 bytes.
inline size_t logprob_workspace(int64_t T, int64_t V, int64_t top) {
    const int64_t s = plan_logprobs(T, V, top).segments;
    return s > 1 ? (size_t)T * s * (16 + 8 * top) : 0;
}

}  // namespace dn
