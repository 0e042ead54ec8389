// attention_cache.hip -- deferred Softmax -> P.V of ragged sequences over the paged key/value cache:
//
//   out = sum_j 2^(s_j - m) v_j V_j / sum_j 2^(s_j - m),   s_j = scale log2(e) k_j (q . K_j),
//
// K_j, V_j the codes of token j and k_j, v_j their scales: a scale is one number per key, so it
// multiplies the key's score (k_j) and numerator (v_j) and no code is scaled by itself.  Both
// products are taken transposed, as in attention.hip: a lane keeps one query, and the numerators
// go from the scores' accumulators straight into the second product (kv_layout.hpp).
//
// Scores, maximum, sums and partial sums are fp32.  Numerators enter the product with V as bf16, the matrix
// cores' operand: in tiles of 16 rows, which wait for memory, as two parts, the rounded value and what
// rounding left (2^-16 relative); in larger tiles, where the products and the operations beside them
// set the time, as the rounded value alone (2^-8 relative at most, the size of the output's own
// rounding).  The row sums take the numerators before that.  Measured, error in the 2-norm against
// 64 bits: 1.6e-3 to 1.8e-3 in two parts, the error of the exact result rounded once, and 2.1e-3 to 2.4e-3 in
// one.  Time in one part / in two, us: 32 sequences of one token against 4196 to 8192 keys, fp8, 73.1 / 73.7, against
// 4096, bf16, 90.0 / 90.1; 8 sequences of 16 tokens against 4096 keys, fp8, 31.0 / 33.4, of 64 53.3 / 63.3; two chunks of 1000
// against 8191 225 / 334; 2048 tokens against 16384, bf16, 477 / 656.  Queries see keys up to
// their own: query i of n sees keys 0 .. kv_len - n + i.  A masked key weighs exactly 0 whatever
// its slot holds: its numerator is selected away, and V codes past kv_len are zeroed before the
// product (codes below are finite: rows with NaN or infinities are held as a NaN scale).
#include <type_traits>

#include "dn_device.hpp"
#include "dn_launch.hpp"
#include "kv_layout.hpp"

namespace dn {
namespace ca {

struct Args {
    const __bf16* Q;
    int64_t q_stride;
    const char* pool;
    int64_t pages;
    int heads, group;
    const int32_t* table;    // [B][width]
    int64_t width;
    const int32_t* q_start;  // [B + 1]; null: one sequence of all T tokens
    const int32_t* kv_len;   // [B]; null: `prefix` keys, all of them visible to every query
    int64_t prefix;
    int64_t T, B;
    int64_t target, least, slots;
    int always_partial;
    float sl2;  // scale * log2(e)
    int4* info;    // [B]: first slot, pages per chunk, chunks of the longest tile, first tile
    // dealt in runs (else null, 0): of each run and of each tile its first piece and their number
    int2* run_pieces;
    int2* tile_pieces;
    Piece* pieces;
    int64_t tiles_most;
    float* parts;  // [slots][rows][d + 4]: sums, l, m
    __bf16* out;   // [T][heads * group][d]
};

__device__ __forceinline__ Seq sequence(const Args& a, int64_t b) {
    Seq s;
    if (!a.q_start) {
        s.first = 0;
        s.n = (int)a.T;
    } else {
        const int lo = min(max(a.q_start[b], 0), (int)a.T), hi = min(max(a.q_start[b + 1], 0), (int)a.T);
        s.first = lo;
        s.n = max(hi - lo, 0);
    }
    s.len = a.kv_len ? (int)min((int64_t)max(a.kv_len[b], 0), a.width * kKvPage) : (int)a.prefix;
    s.pages = (s.len + kKvPage - 1) / kKvPage;
    return s;
}

struct Item {
    int b, tile, chunk, head;
    int per;   // pages per chunk
    int slot;  // of this item, where its tile has several chunks
    int first, n, len;  // of its sequence
};

// inclusive scan over the wave, on the data-parallel lane moves (no LDS)
template <int CTRL, int ROWS>
__device__ __forceinline__ int lane_move(int v) {
    return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_scan(int v) {
    v += lane_move<0x111, 0xf>(v);  // row_shr:1
    v += lane_move<0x112, 0xf>(v);  // row_shr:2
    v += lane_move<0x114, 0xf>(v);  // row_shr:4
    v += lane_move<0x118, 0xf>(v);  // row_shr:8
    v += lane_move<0x142, 0xa>(v);  // row_bcast:15 into rows 1 and 3
    v += lane_move<0x143, 0xc>(v);  // row_bcast:31 into rows 2 and 3
    return v;
}

// Which item this workgroup takes: false where there is none left.  Sequences in order, of each its
// tiles from the last (which sees the most keys) to the first, of each its chunks, of each the heads
// (consecutive workgroups go to different XCDs: with 8 heads one XCD reads one head's keys).  Every
// wave works it out for itself, 64 sequences at a time, one to a lane.
__device__ __forceinline__ bool find_item(const Args& a, int id, int rows, Item& it) {
    const int lane = threadIdx.x & 63;
    int64_t cost = 0;
    for (int64_t b = lane; b < a.B; b += 64) {
        const Seq s = sequence(a, b);
        cost += (int64_t)(int)(((int64_t)s.n * a.group + rows - 1) / rows) * s.pages;
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) cost += __shfl_xor(cost, o);
    cost = cost * a.heads + a.target - 1;
    const int even = cost >> 32 ? (int)(cost / a.target) : (int)((uint32_t)cost / (uint32_t)a.target);
    const int per = max((int)a.least, even);
    int items_before = 0, slots_before = 0;
    for (int64_t b0 = 0; b0 < a.B; b0 += 64) {
        const int64_t b = b0 + lane;
        // lanes past the last sequence read it again, and count nothing
        const Seq s = sequence(a, min(b, a.B - 1));
        int tiles = (int)(((int64_t)s.n * a.group + rows - 1) / rows), chunks = max(1, (s.pages + per - 1) / per);
        const int items = b < a.B ? tiles * chunks * a.heads : 0, parts = a.always_partial || chunks > 1 ? items : 0;
        const int to = items_before + wave_scan(items), from = to - items;
        const int slots_to = slots_before + wave_scan(parts);
        const uint64_t here = __ballot(id >= from && id < to);
        if (here) {
            const int l = __builtin_ctzll(here);
            const int at = id - __builtin_amdgcn_readlane(from, l), slot = __builtin_amdgcn_readlane(slots_to - parts, l);
            chunks = __builtin_amdgcn_readlane(chunks, l);
            tiles = __builtin_amdgcn_readlane(tiles, l);
            it.b = (int)b0 + l;
            const int rest = at / a.heads;
            it.head = at - rest * a.heads;
            it.chunk = rest % chunks;
            it.tile = tiles - 1 - rest / chunks;
            it.per = per;
            // slots go by tile, chunk and head, whatever order the items have
            it.slot = slot + (it.tile * chunks + it.chunk) * a.heads + it.head;
            it.first = __builtin_amdgcn_readlane(s.first, l);
            it.n = __builtin_amdgcn_readlane(s.n, l);
            it.len = __builtin_amdgcn_readlane(s.len, l);
            // a store that is known to be global: a flat one would make every later wait a full one
            if (at == 0 && threadIdx.x == 0)
                *(__attribute__((address_space(1))) u32x4*)(uintptr_t)(a.info + it.b) =
                    u32x4{(uint32_t)slot, (uint32_t)per, (uint32_t)chunks, 0u};
            return true;
        }
        items_before = __builtin_amdgcn_readlane(to, 63);
        slots_before = __builtin_amdgcn_readlane(slots_to, 63);
        if (id < items_before) return false;  // counts past 31 bits (q_start out of order)
    }
    return false;
}

// Keys that some query of the tile sees.
__device__ __forceinline__ int tile_keys(const Args& a, int n, int len, int tile, int rows) {
    return a.kv_len ? seen_keys(n, len, a.group, tile, rows) : len;
}
__device__ __forceinline__ int tile_chunks(int keys, int per) {
    return max(1, ((keys + kKvPage - 1) / kKvPage + per - 1) / per);
}

// The pages of one of a tile's chunks, which are as equal as they can be.
__device__ __forceinline__ void chunk_pages(int keys, int chunks, int chunk, int& lo, int& hi) {
    const int pages = (keys + kKvPage - 1) / kKvPage, each = pages / chunks, more = pages - each * chunks;
    lo = chunk * each + min(chunk, more);
    hi = lo + each + (chunk < more ? 1 : 0);
}

// ----------------------------------------------------------------------------- runs
// Lists every run's pieces, a run to a thread (kv_layout.hpp: deal_run).
__global__ __launch_bounds__(64) void plan_kernel(const Args a, int rows) {
    const int lane = threadIdx.x;
    const int64_t run = (int64_t)blockIdx.x * 64 + lane;
    int64_t total = 0;
    for (int64_t b = lane; b < a.B; b += 64) {
        const Seq s = sequence(a, b);
        total += weights(s, a.group, rows).before(tiles_of(s, a.group, rows)) * a.heads;
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) total += __shfl_xor(total, o);
    const Line line{a.B, a.heads, a.target, total, run_length(total, a.target, a.least, a.group), a.group, rows, a.tiles_most};
    const int64_t x0 = run * line.per;
    // the sequence in which the run starts: 64 sequences at a time, one to a lane
    int64_t start = 0, tile_start = 0, b = -1, b_start = 0, b_tiles = 0;
    for (int64_t b0 = 0; b0 < a.B; b0 += 64) {
        int64_t sum = 0, tiles = 0;
        if (b0 + lane < a.B) {
            const Seq s = sequence(a, b0 + lane);
            tiles = tiles_of(s, a.group, rows);
            sum = weights(s, a.group, rows).before(tiles) * a.heads;
            tiles *= a.heads;
        }
        int64_t to = sum, tiles_to = tiles;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t y = __shfl_up(to, o), z = __shfl_up(tiles_to, o);
            to += lane >= o ? y : 0;
            tiles_to += lane >= o ? z : 0;
        }
        to += start;
        tiles_to += tile_start;
        if (blockIdx.x == 0 && b0 + lane < a.B) a.info[b0 + lane] = int4{0, 0, 0, (int)(tiles_to - tiles)};
        int low = 0, high = 64;  // the first lane whose sequence ends past x0
#pragma unroll
        for (int i = 0; i < 6; ++i) {
            const int mid = (low + high) >> 1;
            if (__shfl(to, mid - 1) <= x0)
                low = mid;
            else
                high = mid;
        }
        const int64_t to_l = __shfl(to, low & 63), sum_l = __shfl(sum, low & 63);
        const int64_t tiles_to_l = __shfl(tiles_to, low & 63), tiles_l = __shfl(tiles, low & 63);
        if (b < 0 && to_l > x0) {
            b = b0 + low;
            b_start = to_l - sum_l;
            b_tiles = tiles_to_l - tiles_l;
        }
        start = __shfl(to, 63);
        tile_start = __shfl(tiles_to, 63);
    }
    if (run >= a.target) return;
    int2 list;
    deal_run(
        line, run, b, b_start, b_tiles, [&](int64_t at) { return sequence(a, at); },
        [&](int64_t at, const Piece& p) { a.pieces[at] = p; },
        [&](int64_t at, int first, int pieces) { a.tile_pieces[at] = int2{first, pieces}; }, list.x, list.y);
    a.run_pieces[run] = list;
}

// The table's page, kept inside the pool whatever the table holds.
__device__ __forceinline__ int page_at(const Args& a, int b, int64_t at) {
    const int32_t p = a.table[(int64_t)b * a.width + at];
    return (uint64_t)(int64_t)p < (uint64_t)a.pages ? p : 0;
}

// A fragment chunk's 16 bytes as operands of E / 8 products.
template <int FMT>
__device__ __forceinline__ u32x4 frag(const u32x4& c, int j);
template <>
__device__ __forceinline__ u32x4 frag<kKvBf16>(const u32x4& c, int) { return c; }
__device__ __forceinline__ uint32_t fp8_pair(uint32_t w, bool hi) {
    const bf16x2_t v = hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)
                          : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
    return __builtin_bit_cast(uint32_t, v);
}
template <>
__device__ __forceinline__ u32x4 frag<kKvFp8>(const u32x4& c, int j) {
    const uint32_t lo = j ? c.z : c.x, hi = j ? c.w : c.y;
    return u32x4{fp8_pair(lo, false), fp8_pair(lo, true), fp8_pair(hi, false), fp8_pair(hi, true)};
}

// All ones over the first `keep` tokens of a lane's 16 bytes of V, zeros over the others.  Words, not
// lane masks: those would fill the scalar registers.
template <int FMT>
__device__ __forceinline__ u32x4 keep_tokens(int keep) {
    constexpr int PER = FMT == kKvBf16 ? 2 : 4, BITS = 32 / PER;  // tokens in a word
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int left = min(max(keep - j * PER, 0), PER);
        w[j] = left == PER ? ~0u : (1u << (left * BITS)) - 1u;
    }
    return u32x4{w[0], w[1], w[2], w[3]};
}

// Partial sums relative to m, brought to a larger reference.  A reference is never -inf (kLowest, no
// key yet), so no difference of two infinities arises but where a score is +inf: NaN, as it should be.
constexpr float kLowest = -3.402823466e38f;
__device__ __forceinline__ float weight(float m, float mn) { return __builtin_amdgcn_exp2f(m - mn); }

// Softmax state of one 16-query block: the reference maximum, raised only when a score exceeds it by
// more than 8 (numerators stay below 2^8), and the lane's share of the sum.
struct State {
    float m, l;
};

// Scores of TILES key tiles (16 each, of one unit) -> numerators as operands, in PARTS.  s holds q . K; kk the
// lane's K scales (of each tile's four keys) times scale log2(e), vs its V scales; lim: the last key
// that this lane's query sees.
template <int TILES, int D, bool MASK, int PARTS>
__device__ __forceinline__ void softmax_unit(const f32x4 (&s)[TILES], const f32x4 (&kk)[TILES], const f32x4 (&vs)[TILES],
                                             const int (&key0)[TILES], int lim, State& st, f32x4 (&acc)[D / 16],
                                             u32x4 (&pf)[PARTS][TILES / 2]) {
    f32x4 x[TILES];
    float top = -__builtin_inff();
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[t][i] = __builtin_fmaf(s[t][i], kk[t][i], -st.m);
            if (MASK) x[t][i] = key0[t] + i <= lim ? x[t][i] : -__builtin_inff();
            top = fmaxf(top, x[t][i]);
        }
    if (__any(top > 8.f)) {
        float high = kLowest;
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[t][i] = s[t][i] * kk[t][i];
                if (MASK) x[t][i] = key0[t] + i <= lim ? x[t][i] : -__builtin_inff();
                high = fmaxf(high, x[t][i]);
            }
        const float mn = fmaxf(max_lane_groups(high), st.m), w = weight(st.m, mn);
        st.m = mn;
        st.l *= w;
#pragma unroll
        for (int n = 0; n < D / 16; ++n) acc[n] *= w;
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[t][i] -= mn;
    }
#pragma unroll
    for (int t = 0; t < TILES; t += 2) {
        float p[8];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(x[t + h][i]);
                // a masked key's scale may be anything: its numerator is 0 whatever it holds
                const bool on = !MASK || key0[t + h] + i <= lim;
                st.l += on ? e : 0.f;
                p[4 * h + i] = on ? e * vs[t + h][i] : 0.f;
            }
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = pack_bf16(p[2 * i], p[2 * i + 1]);
                p[2 * i] -= bf_lo(w[i]);
                p[2 * i + 1] -= bf_hi(w[i]);
            }
            pf[part][t / 2] = u32x4{w[0], w[1], w[2], w[3]};
        }
    }
}

// ----------------------------------------------------------------------------- few rows
// Tiles of 16 rows.  Bound by HBM: each wave takes pages of the chunk in turn, its codes straight to
// registers (V of a unit and K of the next in flight while the unit's scores are worked on), and
// the four waves' sums meet in LDS at the end.  Measured, 32 sequences against 4196 to 8192 keys, 32 query over
// 8 key/value heads of 128, fp8 (418 MB): 72 us, 5.8 TB/s; the call with its merge 75 us.  fp8 takes 217
// registers, so two workgroups to a CU; held to 168 for three it spills (157 us, with numerators in one part).
constexpr int kDecodeRows = 16, kDecodeParts = 2;
template <int FMT, int D>
constexpr int decode_lds = 4 * kDecodeRows * (D + 4) * 4 + 8 * kDecodeRows * 4;

template <int FMT, int D>
__device__ __forceinline__ void decode_item(const Args& a, int id, char* lds) {
    using B = KvBlock<FMT, D>;
    constexpr int E = B::E, R = kDecodeRows, UNITS = kKvPage / (4 * E), TILES = E / 4, KC = D / (4 * E), NB = D / 16;
    constexpr int LOADS = NB;  // chunks of K, and of V, in a unit
    static_assert(TILES * KC == LOADS, "");
    constexpr int PITCH = D + 4;
    float(*sums)[R][PITCH] = reinterpret_cast<float(*)[R][PITCH]>(lds);
    float(*ml)[2][R] = reinterpret_cast<float(*)[2][R]>(lds + 4 * R * PITCH * 4);

    Item it;
    if (!find_item(a, id, R, it)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q = lane & 15, G = lane >> 4;
    const int keys = tile_keys(a, it.n, it.len, it.tile, R), chunks = tile_chunks(keys, it.per);
    if (it.chunk >= chunks) return;
    const bool partial = a.always_partial || chunks > 1;
    if (partial && (it.slot < 0 || it.slot >= a.slots)) return;

    // this lane's query
    const int64_t row = (int64_t)it.tile * R + q;
    const int rows_here = (int)min((int64_t)R, (int64_t)it.n * a.group - (int64_t)it.tile * R);
    const int64_t rr = q < rows_here ? row : row - q;
    const int qi = quotient32(rr, a.group), qh = it.head * a.group + ((int)rr - qi * a.group);
    const __bf16* qp = a.Q + (int64_t)(it.first + qi) * a.q_stride + (int64_t)qh * D;
    u32x4 qf[D / 32];
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int j = 0; j < E / 8; ++j) qf[c * (E / 8) + j] = ld16(qp + 4 * E * c + E * G + 8 * j);
    const int lim = a.kv_len ? it.len - it.n + qi : it.len - 1;
    // the first query of the tile sees the fewest keys
    const int lim_min = a.kv_len ? it.len - it.n + quotient32((int64_t)it.tile * R, a.group) : it.len - 1;

    f32x4 acc[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    State st{kLowest, 0.f};

    int page_lo, page_hi;
    chunk_pages(keys, chunks, it.chunk, page_lo, page_hi);
    const int count = page_hi - page_lo > wave ? (page_hi - page_lo - wave + 3) / 4 : 0;  // pages of this wave
    const int64_t page_bytes = (int64_t)a.heads * B::SIZE;
    const char* head_base = a.pool + (int64_t)it.head * B::SIZE;
    // page ids of the next 64 pages of this wave, one to a lane
    int ids = 0;
    auto block_of = [&](int k) __attribute__((always_inline)) {
        if (k % 64 == 0) ids = k + lane < count ? page_at(a, it.b, page_lo + wave + 4 * (k + lane)) : 0;
        return head_base + (int64_t)__builtin_amdgcn_readlane(ids, k % 64) * page_bytes;
    };
    u32x4 kf[LOADS], vf[LOADS];
    f32x4 ks[TILES];
    const int total = count * UNITS;
    const char* block = nullptr;
    auto scales = [&](int at, int u, int t) __attribute__((always_inline)) {
        return *reinterpret_cast<const f32x4*>(block + at + 4 * (4 * E * u + E * G + 4 * t));
    };
    auto fetch_k = [&](int un) __attribute__((always_inline)) {
        const int u = un % UNITS;
        if (u == 0) block = block_of(un / UNITS);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) kf[i] = ld16_stream(block + (u * LOADS + i) * kChunkBytes + lane * 16);
#pragma unroll
        for (int t = 0; t < TILES; ++t) ks[t] = scales(B::KS, u, t);
    };
    if (total > 0) fetch_k(0);
    // MORE is a constant: where the next loads were conditional the compiler's waits for V would have to
    // cover the path without them, and so wait for them too
    auto step = [&](int un, auto mask_tag, auto more_tag) __attribute__((always_inline)) {
        constexpr bool MASK = decltype(mask_tag)::value, MORE = decltype(more_tag)::value;
        const int u = un % UNITS, page = page_lo + wave + 4 * (un / UNITS);
        f32x4 vs[TILES], s[TILES], kk[TILES];
        int key0[TILES];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) vf[i] = ld16_stream(block + B::PART + (u * LOADS + i) * kChunkBytes + lane * 16);
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            vs[t] = scales(B::VS, u, t);
            key0[t] = page * kKvPage + 4 * E * u + E * G + 4 * t;
        }
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < KC; ++c)
#pragma unroll
                for (int j = 0; j < E / 8; ++j)
                    s[t] = mfma_chunk<__bf16>(frag<FMT>(kf[t * KC + c], j), qf[c * (E / 8) + j], s[t]);
            kk[t] = ks[t] * a.sl2;
        }
        if constexpr (MORE) fetch_k(un + 1);
        u32x4 pf[kDecodeParts][TILES / 2];
        softmax_unit<TILES, D, MASK>(s, kk, vs, key0, lim, st, acc, pf);
        if constexpr (MASK) {
            const u32x4 keep = keep_tokens<FMT>(it.len - (page * kKvPage + 4 * E * u + E * G));
#pragma unroll
            for (int i = 0; i < LOADS; ++i) vf[i] &= keep;
        }
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int j = 0; j < E / 8; ++j)
#pragma unroll
                for (int part = 0; part < kDecodeParts; ++part)
                    acc[n] = mfma_chunk<__bf16>(frag<FMT>(vf[n], j), pf[part][j], acc[n]);
    };
    // pages that every query of the tile sees whole, then those that a mask cuts, then the last unit
    const std::true_type yes{};
    const std::false_type no{};
    const int whole_pages = (lim_min + 1) / kKvPage - page_lo;
    const int whole = min((whole_pages > wave ? (whole_pages - wave + 3) / 4 : 0) * UNITS, total - 1);
    for (int un = 0; un < whole; ++un) step(un, no, yes);
    for (int un = max(whole, 0); un < total - 1; ++un) step(un, yes, yes);
    if (total > 0) step(total - 1, yes, no);

    // the four waves' sums
    const float l = sum_lane_groups(st.l);
    if (G == 0) {
        ml[wave][0][q] = st.m;
        ml[wave][1][q] = l;
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) *reinterpret_cast<f32x4*>(&sums[wave][q][16 * n + 4 * G]) = acc[n];
    __syncthreads();
    constexpr int PER = 8;  // outputs of a thread at a time
    for (int i = threadIdx.x; i < rows_here * (D / PER); i += 256) {
        const int r = i / (D / PER), x = i % (D / PER) * PER;
        float m = kLowest, w[4], lt = 0.f, o[PER];
#pragma unroll
        for (int v = 0; v < 4; ++v) m = fmaxf(m, ml[v][0][r]);
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] = 0.f;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            w[v] = weight(ml[v][0][r], m);
            lt += w[v] * ml[v][1][r];
#pragma unroll
            for (int e = 0; e < PER; ++e) o[e] += w[v] * sums[v][r][x + e];
        }
        const int64_t ro = (int64_t)it.tile * R + r;
        if (partial) {
            float* part = a.parts + ((int64_t)it.slot * R + r) * (int64_t)(D + 4);
            *reinterpret_cast<f32x4*>(part + x) = f32x4{o[0], o[1], o[2], o[3]};
            *reinterpret_cast<f32x4*>(part + x + 4) = f32x4{o[4], o[5], o[6], o[7]};
            if (x == 0) *reinterpret_cast<f32x4*>(part + D) = f32x4{lt, m, 0.f, 0.f};
        } else {
            const int i_q = quotient32(ro, a.group);
            const bool none = a.kv_len && it.len - it.n + i_q < 0;  // no key at all: zero
            const float inv = none ? 0.f : 1.0f / lt;
            uint32_t pk[PER / 2];
#pragma unroll
            for (int e = 0; e < PER / 2; ++e) pk[e] = none ? 0u : pack_bf16(o[2 * e] * inv, o[2 * e + 1] * inv);
            const int64_t oh = (int64_t)(it.first + i_q) * a.heads * a.group + it.head * a.group + ((int)ro - i_q * a.group);
            *reinterpret_cast<u32x4*>(a.out + oh * D + x) = u32x4{pk[0], pk[1], pk[2], pk[3]};
        }
    }
}

// ----------------------------------------------------------------------------- many rows
// The lane's row: its sums into the tile's slot, or divided into the output.
template <int D>
__device__ __forceinline__ void store_rows(const Args& a, const Item& it, int rows, int64_t row, int64_t rows_all,
                                           int slot, int lim, const State& st, const f32x4 (&acc)[D / 16]) {
    const int G = (threadIdx.x & 63) >> 4;
    const float l = sum_lane_groups(st.l);
    if (row >= rows_all) return;
    if (slot >= 0) {
        float* part = a.parts + ((int64_t)slot * rows + (row - (int64_t)it.tile * rows)) * (int64_t)(D + 4);
#pragma unroll
        for (int n = 0; n < D / 16; ++n) *reinterpret_cast<f32x4*>(part + 16 * n + 4 * G) = acc[n];
        if (G == 0) *reinterpret_cast<f32x4*>(part + D) = f32x4{l, st.m, 0.f, 0.f};
        return;
    }
    const int qi = quotient32(row, a.group);
    const bool none = lim < 0;  // no key at all: zero
    const float inv = 1.0f / l;
    const int64_t oh = (int64_t)(it.first + qi) * a.heads * a.group + it.head * a.group + ((int)row - qi * a.group);
#pragma unroll
    for (int n = 0; n < D / 16; ++n) {
        const uint2 v = {pack_bf16(acc[n][0] * inv, acc[n][1] * inv), pack_bf16(acc[n][2] * inv, acc[n][3] * inv)};
        *reinterpret_cast<uint2*>(a.out + oh * D + 16 * n + 4 * G) = none ? uint2{0, 0} : v;
    }
}

// Tiles of 4 waves x QW x 16 rows.  Bound by the matrix cores and the exponentials beside them: a
// page goes through LDS as bf16 operands (two slots, the next one filled while a page is worked on)
// and serves the tile's four waves.  bf16 codes are copied there directly; e4m3 codes go through
// registers and are widened once for all waves.  Measured, 8 sequences of 16 / 64 new tokens against 4096 keys, 32
// query over 8 key/value heads of 128, fp8: 30 / 57 us a call.
template <int D>
constexpr int tile_lds = 2 * (2 * kKvPage * D * 2 + 8 * kKvPage);

template <int FMT, int D, int QW>
__device__ __forceinline__ void tile_item(const Args& a, int id, char* smem) {
    using B = KvBlock<FMT, D>;
    constexpr int E = B::E, J = E / 8, R = 64 * QW, TILES = 4, KC = D / (4 * E), NB = D / 16;
    constexpr int FRAGS = 2 * kKvPage * D * 2 / kChunkBytes;  // operands of a page, 1 KiB each: K's, then V's
    constexpr int CHUNKS = FRAGS / J;                         // of 1 KiB in the cache
    constexpr int SCALES = FRAGS * kChunkBytes;               // then K's and V's scales
    constexpr int STEP = SCALES + 8 * kKvPage;
    static_assert(2 * STEP == tile_lds<D>, "");

    Item it;
    if (!find_item(a, id, R, it)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int q = lane & 15, G = lane >> 4;
    const int keys = tile_keys(a, it.n, it.len, it.tile, R), chunks = tile_chunks(keys, it.per);
    if (it.chunk >= chunks) return;
    const bool partial = a.always_partial || chunks > 1;
    if (partial && (it.slot < 0 || it.slot >= a.slots)) return;

    const int64_t rows_all = (int64_t)it.n * a.group;
    const int64_t row0 = (int64_t)it.tile * R + wave * QW * 16;  // the wave's first row
    u32x4 qf[QW][D / 32];
    int lim[QW];
#pragma unroll
    for (int f = 0; f < QW; ++f) {
        const int64_t row = min(row0 + f * 16 + q, rows_all - 1);
        const int qi = quotient32(row, a.group), qh = it.head * a.group + ((int)row - qi * a.group);
        const __bf16* qp = a.Q + (int64_t)(it.first + qi) * a.q_stride + (int64_t)qh * D;
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int j = 0; j < E / 8; ++j) qf[f][c * (E / 8) + j] = ld16(qp + 4 * E * c + E * G + 8 * j);
        lim[f] = a.kv_len ? it.len - it.n + qi : it.len - 1;
    }

    f32x4 acc[QW][NB];
    State st[QW];
#pragma unroll
    for (int f = 0; f < QW; ++f) {
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[f][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        st[f] = State{kLowest, 0.f};
    }

    int page_lo, page_hi;
    chunk_pages(keys, chunks, it.chunk, page_lo, page_hi);
    const int count = page_hi - page_lo;
    const int64_t page_bytes = (int64_t)a.heads * B::SIZE;
    const char* head_base = a.pool + (int64_t)it.head * B::SIZE;
    const uint32_t lds0 = lds_addr32(smem);
    int ids = 0;
    u32x4 raw[CHUNKS / 4];
    auto fetch = [&](int k) __attribute__((always_inline)) {
        if (k % 64 == 0) ids = k + lane < count ? page_at(a, it.b, page_lo + k + lane) : 0;
        const char* block = head_base + (int64_t)__builtin_amdgcn_readlane(ids, k % 64) * page_bytes;
        const uint64_t src = uniform_u64(block);
        const uint32_t dst = lds0 + (uint32_t)(k & 1) * STEP;
#pragma unroll
        for (int i = 0; i < CHUNKS / 4; ++i) {
            const uint32_t at = (uint32_t)(wave + 4 * i) * kChunkBytes;
            if constexpr (J == 1)
                g2lds16_async_sb(src, at + lane * 16, dst + at);
            else
                raw[i] = ld16(block + at + lane * 16);
        }
        // the scales: half a KiB, the first 32 lanes of one wave
        if (wave == 0 && lane < 32) g2lds16_async_sb(src, (uint32_t)B::KS + lane * 16, dst + (uint32_t)SCALES);
    };
    auto land = [&](int k) __attribute__((always_inline)) {
        if constexpr (J > 1) {
            char* slot = smem + (k & 1) * STEP;
#pragma unroll
            for (int i = 0; i < CHUNKS / 4; ++i)
#pragma unroll
                for (int j = 0; j < J; ++j)
                    *reinterpret_cast<u32x4*>(slot + ((wave + 4 * i) * J + j) * kChunkBytes + lane * 16) =
                        frag<FMT>(raw[i], j);
        }
        wait_vm();
        __syncthreads();
    };
    if (count > 0) {
        fetch(0);
        land(0);
    }
    // Operands are read from LDS one group of products ahead, in an order fixed by scheduling groups.
    auto read = [&](const char* slot, int first, u32x4(&fr)[KC * J]) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < KC * J; ++c) fr[c] = lds_ld16(lds_ptr((char*)slot + (first + c) * kChunkBytes + lane * 16));
    };
    constexpr int G4 = KC * J, VG = FRAGS / 2 / G4;  // operands of a group; groups of V
    auto step = [&](int k, auto tag) __attribute__((always_inline)) {
        constexpr bool MASK = decltype(tag)::value;
        const char* slot = smem + (k & 1) * STEP;
        const int base = (page_lo + k) * kKvPage;
        f32x4 s[QW][TILES], kk[TILES], vs[TILES];
        int key0[TILES];
        u32x4 fr[2][G4];
        read(slot, 0, fr[0]);
        if (k + 1 < count) fetch(k + 1);
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            read(slot, (t + 1) * G4, fr[(t + 1) & 1]);  // after the last tile of K: V's first group
#pragma unroll
            for (int f = 0; f < QW; ++f) s[f][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < G4; ++c)
#pragma unroll
                for (int f = 0; f < QW; ++f) s[f][t] = mfma_chunk<__bf16>(fr[t & 1][c], qf[f][c], s[f][t]);
        }
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const int o = t * 4 / E * 4 * E + E * G + t * 4 % E;  // tile t's first token of lane group G
            kk[t] = *reinterpret_cast<const f32x4*>(slot + SCALES + 4 * o) * a.sl2;
            vs[t] = *reinterpret_cast<const f32x4*>(slot + SCALES + 4 * kKvPage + 4 * o);
            key0[t] = base + o;
        }
        u32x4 pf[QW][1][TILES / 2];
#pragma unroll
        for (int f = 0; f < QW; ++f) softmax_unit<TILES, D, MASK>(s[f], kk, vs, key0, lim[f], st[f], acc[f], pf[f]);
        u32x4 keep[TILES / 2];
        if constexpr (MASK) {
#pragma unroll
            for (int c = 0; c < TILES / 2; ++c)
                keep[c] = keep_tokens<kKvBf16>(it.len - (base + 4 * E * (c / J) + E * G + 8 * (c % J)));
        }
#pragma unroll
        for (int v = 0; v < VG; ++v) {
            if (v + 1 < VG) read(slot, (TILES + v + 1) * G4, fr[(v + 1) & 1]);
#pragma unroll
            for (int c = 0; c < G4; ++c) {
                const int at = v * G4 + c, n = at / J % NB, u = at / J / NB, j = at % J;
                if constexpr (MASK) fr[v & 1][c] &= keep[u * J + j];
#pragma unroll
                for (int f = 0; f < QW; ++f) acc[f][n] = mfma_chunk<__bf16>(fr[v & 1][c], pf[f][0][u * J + j], acc[f][n]);
            }
        }
        if (k + 1 < count) land(k + 1);  // page k + 1 has landed, and every wave is done with page k
    };
    // pages that every query of the tile sees whole, then those that a mask cuts
    const int64_t tile_row = (int64_t)it.tile * R;
    const int lim_min = a.kv_len ? it.len - it.n + quotient32(tile_row, a.group) : it.len - 1;
    const int whole = min(max((lim_min + 1) / kKvPage - page_lo, 0), count);
    for (int k = 0; k < whole; ++k) step(k, std::false_type{});
    for (int k = whole; k < count; ++k) step(k, std::true_type{});

#pragma unroll
    for (int f = 0; f < QW; ++f)
        store_rows<D>(a, it, R, row0 + f * 16 + q, rows_all, partial ? it.slot : kWhole, lim[f], st[f], acc[f]);
}

// Items of `rows` query rows: 16, 64 or 128.
template <int FMT, int D, int ROWS>
__device__ __forceinline__ void item(const Args& a, int id, char* lds) {
    if constexpr (ROWS == kDecodeRows)
        decode_item<FMT, D>(a, id, lds);
    else
        tile_item<FMT, D, ROWS / 64>(a, id, lds);
}
template <int FMT, int D, int ROWS>
constexpr int item_lds = ROWS == kDecodeRows ? decode_lds<FMT, D> : tile_lds<D>;

template <int FMT, int D, int ROWS>
__global__ __launch_bounds__(256, 2) void cache_kernel(const Args a) {
    __shared__ __attribute__((aligned(1024))) char lds[item_lds<FMT, D, ROWS>];
    item<FMT, D, ROWS>(a, blockIdx.x, lds);
}

// The shared prefix in tiles of ROWS rows and each sequence's own keys in tiles of 16, side by side in
// one launch: either alone leaves most of the chip idle.  Bound by the prefix's serial page steps (8 pages a
// workgroup).  Measured, 64 sequences behind 8192 keys, 32 query over 8 key/value heads of 128, fp8: 32 us a call with
// its merge; one launch after the other took 48.
template <int FMT, int D, int ROWS>
__global__ __launch_bounds__(256, 2) void shared_kernel(const Args prefix, const Args own, int prefix_items) {
    constexpr int LDS = item_lds<FMT, D, ROWS> > decode_lds<FMT, D> ? item_lds<FMT, D, ROWS> : decode_lds<FMT, D>;
    __shared__ __attribute__((aligned(1024))) char lds[LDS];
    if ((int)blockIdx.x < prefix_items)
        item<FMT, D, ROWS>(prefix, blockIdx.x, lds);
    else
        decode_item<FMT, D>(own, blockIdx.x - prefix_items, lds);
}

// Tiles of 8 waves x 32 rows, two waves to a SIMD.  A page is an exponential phase (mask, maximum,
// numerators: VALU) and a matrix phase (its product with V, the scores of the next page); the two
// halves of the workgroup run one phase apart, separated by barriers, so that on every SIMD one
// wave's exponentials run beside the other's products: left alone the two fall into step.  The half
// that runs behind (late) fills the rings, one page ahead: stage k is K of page k + 1 and V of page k.
// With phases counted from the first scores of the early half (-1), early waves work on page k in 2k
// and 2k + 1, late ones in 2k + 1 and 2k + 2; stage k lands by the end of 2k in slots last read in 2k - 2.
// Bound by the VALU beside the matrix cores (53 % and 41 % busy, fp8).  Measured, 32 query over 8 key/value heads of
// 128: one 2048-token chunk against 16384 keys 1050 TFLOP/s (bf16), 820 to 870 (fp8, which the late waves widen);
// two ragged chunks of 1000 against 8191 keys, fp8, 225 us a call, 825 TFLOP/s.
template <int FMT, int D>
__global__ __launch_bounds__(512) void wide_kernel(const Args a) {
    using B = KvBlock<FMT, D>;
    constexpr int E = B::E, J = E / 8, QW = 2, R = 256, TILES = 4, NB = D / 16, DC = D / 32;
    constexpr int PAGE_K = kKvPage * D * 2;                // bf16 operands of a page's K, and of its V
    constexpr int FRAGS = PAGE_K / kChunkBytes;
    constexpr int CHUNKS = FRAGS / J;                      // of 1 KiB in the cache
    constexpr int PER = CHUNKS / 4;                        // of a late wave
    constexpr int VRING = 2 * PAGE_K, SRING = 4 * PAGE_K;  // K, V: two slots each; scales: four
    constexpr int SCALES = 8 * kKvPage;
    __shared__ __attribute__((aligned(1024))) char smem[SRING + 4 * SCALES];

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    Item it;
    int page_lo, count, slot;
    int2 list = {0, 1};
    if (a.pieces) {
        // give each XCD a stretch of the line: its workgroups then share keys in one L2
        list = a.run_pieces[xcd_contiguous(blockIdx.x, gridDim.x)];
        list.x = __builtin_amdgcn_readfirstlane(list.x);
        list.y = __builtin_amdgcn_readfirstlane(list.y);
    }
    for (; list.y > 0; ++list.x, --list.y) {
    if (a.pieces) {
        const Piece p = a.pieces[list.x];
        it.b = __builtin_amdgcn_readfirstlane(p.b);
        it.head = __builtin_amdgcn_readfirstlane(p.head);
        it.tile = __builtin_amdgcn_readfirstlane(p.tile);
        page_lo = __builtin_amdgcn_readfirstlane(p.lo);
        count = __builtin_amdgcn_readfirstlane(p.hi) - page_lo;
        slot = __builtin_amdgcn_readfirstlane(p.slot);
        const Seq s = sequence(a, it.b);
        it.first = __builtin_amdgcn_readfirstlane(s.first);
        it.n = __builtin_amdgcn_readfirstlane(s.n);
        it.len = __builtin_amdgcn_readfirstlane(s.len);
    } else {
        if (!find_item(a, blockIdx.x, R, it)) return;
        const int keys = tile_keys(a, it.n, it.len, it.tile, R), chunks = tile_chunks(keys, it.per);
        if (it.chunk >= chunks) return;
        int page_hi;
        chunk_pages(keys, chunks, it.chunk, page_lo, page_hi);
        count = page_hi - page_lo;
        slot = a.always_partial || chunks > 1 ? it.slot : kWhole;
    }
    if (slot == kNone || slot >= a.slots) continue;

    int lane = tid & 63;
    asm volatile("" : "+v"(lane));
    const int q = lane & 15, G = lane >> 4;
    const int64_t rows_all = (int64_t)it.n * a.group;
    const int64_t tile_row = (int64_t)it.tile * R, row0 = tile_row + wave * QW * 16;  // the wave's first row
    u32x4 qf[QW][DC];
    int lim[QW];
#pragma unroll
    for (int f = 0; f < QW; ++f) {
        const int64_t row = min(row0 + f * 16 + q, rows_all - 1);
        const int qi = quotient32(row, a.group), qh = it.head * a.group + ((int)row - qi * a.group);
        const __bf16* qp = a.Q + (int64_t)(it.first + qi) * a.q_stride + (int64_t)qh * D;
#pragma unroll
        for (int c = 0; c < DC; ++c) qf[f][c] = ld16(qp + 4 * E * (c / J) + E * G + 8 * (c % J));
        lim[f] = a.kv_len ? it.len - it.n + qi : it.len - 1;
    }
    f32x4 acc[QW][NB], s[QW][TILES];
    State st[QW];
#pragma unroll
    for (int f = 0; f < QW; ++f) {
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[f][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        st[f] = State{kLowest, 0.f};
    }

    const int64_t page_bytes = (int64_t)a.heads * B::SIZE;
    const char* head_base = a.pool + (int64_t)it.head * B::SIZE;
    const uint32_t lds0 = lds_addr32(smem);
    const bool late = wave >= 4;
    const int w4 = wave & 3;
    int ids = 0;
    u32x4 raw[2][PER];
    auto block_of = [&](int k) __attribute__((always_inline)) {
        return head_base + (int64_t)__builtin_amdgcn_readlane(ids, k % 64) * page_bytes;
    };
    // One page's K (which = 0) or V: bf16 codes on their way into the ring, e4m3 codes into registers.
    auto fetch = [&](int which, int k) __attribute__((always_inline)) {
        const char* block = block_of(k) + which * B::PART;
        const uint64_t src = uniform_u64(block);
        const uint32_t dst = lds0 + which * VRING + (uint32_t)(k & 1) * PAGE_K;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t at = (uint32_t)(w4 + 4 * i) * kChunkBytes;
            if constexpr (J == 1)
                g2lds16_async_sb(src, at + lane * 16, dst + at);
            else
                raw[which][i] = ld16(block + at + lane * 16);
        }
        if (which == 0 && w4 == 0 && lane < 32)
            g2lds16_async_sb(src, (uint32_t)B::KS + lane * 16, lds0 + SRING + (uint32_t)(k & 3) * SCALES);
    };
    // A late wave's e4m3 codes into the rings: V of page k + 1 and K of page k + 2 (where there is none,
    // what lies in the registers goes into a slot that is not read again).
    auto put = [&](int k, bool v = true) __attribute__((always_inline)) {
        if constexpr (J > 1) {
#pragma unroll
            for (int which = 1; which >= 0; --which) {
                char* dst = smem + which * VRING + ((which ? k + 1 : k + 2) & 1) * PAGE_K;
                if (which && !v) continue;
#pragma unroll
                for (int i = 0; i < PER; ++i)
#pragma unroll
                    for (int j = 0; j < J; ++j)
                        *reinterpret_cast<u32x4*>(dst + ((w4 + 4 * i) * J + j) * kChunkBytes + lane * 16) =
                            frag<FMT>(raw[which][i], j);
            }
        }
    };
    // the page table's next 64 entries from the 64-page boundary that page k crosses
    auto table = [&](int k) __attribute__((always_inline)) {
        if (k % 64 == 0) ids = k + lane < count ? page_at(a, it.b, page_lo + k + lane) : 0;
    };
    auto stage = [&](int k) __attribute__((always_inline)) {  // V of page k before the table moves on to page k + 1's
        fetch(1, k);
        if (k + 1 < count) {
            table(k + 1);
            fetch(0, k + 1);
        }
    };
    auto meet = [&]() __attribute__((always_inline)) {
        wait_lgkm0();
        block_barrier();
    };
    auto read = [&](const char* slot, int first, u32x4(&fr)[DC]) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < DC; ++c) fr[c] = lds_ld16(lds_ptr((char*)slot + (first + c) * kChunkBytes + lane * 16));
    };
    constexpr int VG = FRAGS / DC;  // groups of V operands
    u32x4 pf[QW][1][TILES / 2];
    // The product of page k's numerators with V, then the scores of page k + 1.  Operands are read
    // from LDS one group of DC ahead of their products, in an order fixed by scheduling groups: left
    // to itself the compiler reads each beside its use and waits for it.
    auto matrix = [&](int k, auto pv_tag, auto qk_tag, auto mask_tag) __attribute__((always_inline)) {
        constexpr bool PV = decltype(pv_tag)::value, QK = decltype(qk_tag)::value, MASK = decltype(mask_tag)::value;
        constexpr int V0 = PV ? VG : 0, GROUPS = V0 + (QK ? TILES : 0);
        const char* vb = smem + VRING + (k & 1) * PAGE_K;
        const char* kb = smem + ((k + 1) & 1) * PAGE_K;
        u32x4 fr[2][DC];
        auto group = [&](int i) __attribute__((always_inline)) {
            if (i < V0)
                read(vb, i * DC, fr[i & 1]);
            else
                read(kb, (i - V0) * DC, fr[i & 1]);
        };
        u32x4 keep[TILES / 2];
        if constexpr (MASK && PV) {
#pragma unroll
            for (int c = 0; c < TILES / 2; ++c)
                keep[c] = keep_tokens<kKvBf16>(it.len - ((page_lo + k) * kKvPage + 4 * E * (c / J) + E * G + 8 * (c % J)));
        }
        if constexpr (QK) {
#pragma unroll
            for (int f = 0; f < QW; ++f)
#pragma unroll
                for (int t = 0; t < TILES; ++t) s[f][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        group(0);
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) {
            if (i + 1 < GROUPS) group(i + 1);
#pragma unroll
            for (int c = 0; c < DC; ++c) {
                if (i < V0) {
                    const int at = i * DC + c, n = at / J % NB, u = at / J / NB, j = at % J;
                    if constexpr (MASK && PV) fr[i & 1][c] &= keep[u * J + j];
#pragma unroll
                    for (int f = 0; f < QW; ++f) acc[f][n] = mfma_chunk<__bf16>(fr[i & 1][c], pf[f][0][u * J + j], acc[f][n]);
                } else {
                    const int t = i - V0;
#pragma unroll
                    for (int f = 0; f < QW; ++f) s[f][t] = mfma_chunk<__bf16>(fr[i & 1][c], qf[f][c], s[f][t]);
                }
            }
        }
        if constexpr (!MASK) {
            __builtin_amdgcn_sched_group_barrier(kSgDsRead, DC, 0);
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) {
                if (i + 1 < GROUPS) __builtin_amdgcn_sched_group_barrier(kSgDsRead, DC, 0);
                __builtin_amdgcn_sched_group_barrier(kSgMfma, DC * QW, 0);
            }
        }
    };
    auto exponentials = [&](int k, auto mask_tag) __attribute__((always_inline)) {
        constexpr bool MASK = decltype(mask_tag)::value;
        const char* scales = smem + SRING + (k & 3) * SCALES;
        f32x4 kk[TILES], vs[TILES];
        int key0[TILES];
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const int o = t * 4 / E * 4 * E + E * G + t * 4 % E;  // tile t's first token of lane group G
            kk[t] = *reinterpret_cast<const f32x4*>(scales + 4 * o) * a.sl2;
            vs[t] = *reinterpret_cast<const f32x4*>(scales + 4 * kKvPage + 4 * o);
            key0[t] = (page_lo + k) * kKvPage + o;
        }
#pragma unroll
        for (int f = 0; f < QW; ++f) softmax_unit<TILES, D, MASK>(s[f], kk, vs, key0, lim[f], st[f], acc[f], pf[f]);
    };
    const std::true_type yes{};
    const std::false_type no{};
    auto page = [&](int k, auto mask_tag, auto late_tag) __attribute__((always_inline)) {
        constexpr bool LATE = decltype(late_tag)::value;
        const bool more = k + 1 < count;
        if (LATE && J == 1 && more) stage(k + 1);
        exponentials(k, mask_tag);
        meet();
        __builtin_amdgcn_s_setprio(1);  // the products first: the other wave's exponentials fill the gaps
        if (more)
            matrix(k, yes, yes, mask_tag);
        else
            matrix(k, yes, no, mask_tag);
        __builtin_amdgcn_s_setprio(0);
        if (LATE && more) {
            put(k);
            wait_vm();  // stage k + 1
            if (J > 1 && k + 2 < count) stage(k + 2);
        }
        if (!LATE || more) meet();
    };
    // pages that every query of the tile sees whole, then those that a mask cuts
    const int lim_min = a.kv_len ? it.len - it.n + quotient32(tile_row, a.group) : it.len - 1;
    const int whole = min(max((lim_min + 1) / kKvPage - page_lo, 0), count);
    if (count > 0) {
        if (late) {
            table(0);
            fetch(0, 0);
            put(-2, false);
            wait_vm();
            meet();
            stage(0);  // phase -1
            meet();
            matrix(-1, no, yes, no);
            put(-1);
            wait_vm();
            if (J > 1 && count > 1) stage(1);
            meet();
            for (int k = 0; k < whole; ++k) page(k, no, yes);
            for (int k = whole; k < count; ++k) page(k, yes, yes);
        } else {
            meet();
            matrix(-1, no, yes, no);
            meet();
            for (int k = 0; k < whole; ++k) page(k, no, no);
            for (int k = whole; k < count; ++k) page(k, yes, no);
        }
    }

    // the lane's rows anew: what an address needs of them would else be held through the pages
    int rows_at = wave * QW * 16 + q;
    asm volatile("" : "+v"(rows_at));
#pragma unroll
    for (int f = 0; f < QW; ++f)
        store_rows<D>(a, it, R, tile_row + rows_at + f * 16, rows_all, slot, lim[f], st[f], acc[f]);
    __syncthreads();  // before the next piece's pages
    }
}

// ----------------------------------------------------------------------------- merge
struct Set {
    const int4* info;
    const float* parts;
    const Piece* pieces;  // of runs; null: chunks
    int64_t slots;
    int rows;
};

// Output rows (token, query head): D / (4 NV) threads over a row's dimensions (NV vectors each), NS such groups
// over its partial sums, the other threads over rows.  Bound by reading the partial sums, or over
// few rows by loads that wait for one another (5 us of 1024 rows of 2 to 4 parts).  `shared` (parts
// null: none) holds the partial sums over the prefix, `own` those over the sequence's own keys;
// without a prefix rows whose tile has one chunk are already written.
template <int D, int NS, int NV>
__global__ __launch_bounds__(256) void merge_kernel(const Args a, const Set own, const Set shared) {
    constexpr int NX = D / (4 * NV), STEP = 4 * NX, ROWS = 256 / (NX * NS);
    static_assert(NS == 1 || NV == 1, "");
    __shared__ __attribute__((aligned(16))) float red[NS > 1 ? ROWS : 1][NS][D + 4];
    const int tid = threadIdx.x, heads = a.heads * a.group;
    const int in = tid / (NX * NS), g = tid / NX % NS, x = tid % NX * 4;
    const int64_t row_id = (int64_t)blockIdx.x * ROWS + in, token = quotient32(row_id, heads);
    const bool is_row = token < a.T;
    // the token's sequence: the one of its own number where each has one token, else a search
    int b = -1;
    if (is_row) {
        const int64_t guess = min(token, a.B - 1);
        if (a.q_start[guess] <= token && token < a.q_start[guess + 1]) {
            b = (int)guess;
        } else {
            int low = 0, high = (int)a.B - 1;  // the last that starts at the token or before
            while (low < high) {
                const int mid = (low + high + 1) >> 1;
                if (a.q_start[mid] <= token)
                    low = mid;
                else
                    high = mid - 1;
            }
            if (a.q_start[low] <= token && token < a.q_start[low + 1]) b = low;
        }
    }
    bool write = is_row && b >= 0;
    const int hq = (int)(row_id - token * heads), h = quotient32(hq, a.group), r = hq - h * a.group;
    const Set* sets[2] = {&own, &shared};
    float m = kLowest, l = 0.f;
    f32x4 o[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) o[v] = f32x4{0.f, 0.f, 0.f, 0.f};
    bool none = false;
    if (write) {
        const Seq s = sequence(a, b);
        none = !shared.parts && s.len - s.n + (int)(token - s.first) < 0;  // no key at all: zero
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const Set& set = *sets[w];
            if (!set.parts) continue;
            const int4 plan = set.info[w ? 0 : b];
            const int row = (int)(w ? token : token - s.first) * a.group + r;
            const int tile = row >> (31 - __builtin_clz(set.rows)), in_tile = row & (set.rows - 1);  // powers of two
            int count, first;
            if (set.pieces) {
                const int64_t ordinal = plan.w + (int64_t)h * tiles_of(s, a.group, set.rows) + tile;
                int2 list = {0, 0};
                if (ordinal >= 0 && ordinal < a.tiles_most) list = a.tile_pieces[ordinal];
                first = list.x;
                count = list.y;
                if (!shared.parts && count == 0) write = false;
            } else {
                const int chunks = w ? plan.z : tile_chunks(tile_keys(a, s.n, s.len, tile, set.rows), max(plan.y, 1));
                if (!shared.parts && chunks == 1) write = false;
                first = plan.x + tile * plan.z * a.heads + h;
                count = chunks;
            }
            if (!write) break;
            // q_start out of order can leave a sequence no workgroup: what it reads here is then no list
            const int64_t most = set.pieces ? a.tiles_most + a.target : set.slots;
            if (first < 0 || count > most || first > most - count) count = 0;
            for (int c = g; c < count; c += NS) {
                const int slot = set.pieces ? set.pieces[first + c].slot : first + c * a.heads;
                if (slot < 0 || slot >= set.slots) continue;  // a run with none of its pages; q_start out of order
                const float* part = set.parts + ((int64_t)slot * set.rows + in_tile) * (D + 4);
                f32x4 p[NV];
#pragma unroll
                for (int v = 0; v < NV; ++v) p[v] = *reinterpret_cast<const f32x4*>(part + x + v * STEP);
                const f32x4 t = *reinterpret_cast<const f32x4*>(part + D);
                const float mn = fmaxf(m, t[1]), wo = weight(m, mn), wn = weight(t[1], mn);
                l = wo * l + wn * t[0];
#pragma unroll
                for (int v = 0; v < NV; ++v) o[v] = o[v] * wo + p[v] * wn;
                m = mn;
            }
        }
    }
    if constexpr (NS > 1) {
        *reinterpret_cast<f32x4*>(&red[in][g][x]) = o[0];
        if (x == 0) {
            red[in][g][D] = l;
            red[in][g][D + 1] = m;
        }
        __syncthreads();
        if (g) return;
#pragma unroll
        for (int v = 1; v < NS; ++v) {
            const float mv = red[in][v][D + 1], mn = fmaxf(m, mv), wo = weight(m, mn), wn = weight(mv, mn);
            l = wo * l + wn * red[in][v][D];
            o[0] = o[0] * wo + *reinterpret_cast<const f32x4*>(&red[in][v][x]) * wn;
            m = mn;
        }
    }
    if (!write) return;
    const float inv = 1.0f / l;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const uint2 w = {pack_bf16(o[v][0] * inv, o[v][1] * inv), pack_bf16(o[v][2] * inv, o[v][3] * inv)};
        *reinterpret_cast<uint2*>(a.out + row_id * D + x + v * STEP) = none ? uint2{0, 0} : w;
    }
}

template <int D>
hipError_t launch_merge(const Args& a, const Set& own, const Set& shared, hipStream_t s) {
    // A workgroup to each row until the rows fill the chip.  Measured, with one part at a time / a workgroup's
    // worth at a time (the whole call, us, fp8, 32 and 8 heads of 128): 32 rows of 65536 keys 68.5 / 34.3, 512 of
    // 4096 32.8 / 31.2, 1024 of 2048 32.3 / 32.1, 2048 of 1024 30.9 / 33.0, 32768 of 16384 293 / 328.  A shared
    // prefix leaves each row more parts: 2048 rows behind 8192 keys 39.6 / 32.7.
    // Past that a row's lookups are VALU work that fewer threads a row spread over more dimensions: 1 / 2 / 4
    // vectors a thread, us: two chunks of 1000 against 8191 keys 231.6 / 226.8 / 225.0 (the merge 21.6 / 15.8 / 14.9),
    // four of 500 against 4096 170 / 164 / 163; 4096 rows behind 8192 keys, which have many parts, 53.3 / 51.4 / 54.2.
    const int64_t rows = a.T * a.heads * a.group;
    constexpr int MOST = 256 / (D / 4);
    if (rows <= (shared.parts ? 2048 : 1024))
        merge_kernel<D, MOST, 1><<<dim3((unsigned)rows), 256, 0, s>>>(a, own, shared);
    else if (shared.parts)
        merge_kernel<D, 1, 2><<<dim3((unsigned)((rows + 2 * MOST - 1) / (2 * MOST))), 256, 0, s>>>(a, own, shared);
    else
        merge_kernel<D, 1, 4><<<dim3((unsigned)((rows + 4 * MOST - 1) / (4 * MOST))), 256, 0, s>>>(a, own, shared);
    return hipGetLastError();
}

template <int FMT, int D>
hipError_t launch(const Args& a, int rows, int64_t grid, hipStream_t s) {
    const dim3 g((unsigned)grid);
    if (rows == 16)
        cache_kernel<FMT, D, 16><<<g, 256, 0, s>>>(a);
    else if (rows == 64)
        cache_kernel<FMT, D, 64><<<g, 256, 0, s>>>(a);
    else if (rows == 128)
        cache_kernel<FMT, D, 128><<<g, 256, 0, s>>>(a);
    else
        wide_kernel<FMT, D><<<g, 512, 0, s>>>(a);
    return hipGetLastError();
}
template <int FMT, int D>
hipError_t launch_shared(const Args& prefix, int rows, int64_t prefix_grid, const Args& own, int64_t grid, hipStream_t s) {
    const dim3 g((unsigned)(prefix_grid + grid));
    if (rows == 16)
        shared_kernel<FMT, D, 16><<<g, 256, 0, s>>>(prefix, own, (int)prefix_grid);
    else if (rows == 64)
        shared_kernel<FMT, D, 64><<<g, 256, 0, s>>>(prefix, own, (int)prefix_grid);
    else
        shared_kernel<FMT, D, 128><<<g, 256, 0, s>>>(prefix, own, (int)prefix_grid);
    return hipGetLastError();
}
// calls f with the cache's format and d as constants
template <class F>
hipError_t with_format(const KvPool& c, F&& f) {
    using std::integral_constant;
    const integral_constant<int, 64> d64{};
    const integral_constant<int, 128> d128{};
    if (c.format == kKvBf16) return c.d == 64 ? f(integral_constant<int, kKvBf16>{}, d64) : f(integral_constant<int, kKvBf16>{}, d128);
    return c.d == 64 ? f(integral_constant<int, kKvFp8>{}, d64) : f(integral_constant<int, kKvFp8>{}, d128);
}

}  // namespace ca

hipError_t launch_attention_cache(const AttentionCacheCall& c, hipStream_t s) {
    const int64_t prefix_pages = (c.prefix + kKvPage - 1) / kKvPage, group = c.q_heads / c.pool.heads;
    const CacheWorkspace w = cache_workspace(c.T, c.B, c.pool.heads, group, c.pool.d, c.width, prefix_pages);
    char* ws = (char*)c.workspace;
    ca::Args a{};
    a.Q = (const __bf16*)c.Q;
    a.q_stride = c.q_stride;
    a.pool = (const char*)c.pool.data;
    a.pages = c.pool.pages;
    a.heads = (int)c.pool.heads;
    a.group = (int)group;
    a.T = c.T;
    a.sl2 = c.scale * 1.4426950408889634f;
    a.out = (__bf16*)c.out;
    auto planned = [&](const CachePlan& p, size_t info, size_t parts, size_t runs) {
        a.target = p.target;
        a.least = p.least;
        a.slots = p.slots;
        a.info = (int4*)(ws + info);
        a.parts = (float*)(ws + parts);
        a.run_pieces = p.in_runs ? (int2*)(ws + runs) : nullptr;
        a.tile_pieces = p.in_runs ? a.run_pieces + p.target : nullptr;
        a.pieces = p.in_runs ? (Piece*)(a.tile_pieces + p.tiles) : nullptr;
        a.tiles_most = p.tiles;
        return ca::Set{a.info, a.parts, a.pieces, p.slots, p.rows};
    };
    ca::Set shared{};
    ca::Args prefix{};
    if (prefix_pages > 0) {
        a.table = c.prefix_table;
        a.width = prefix_pages;
        a.prefix = c.prefix;
        a.B = 1;
        a.always_partial = 1;
        shared = planned(w.prefix, w.prefix_info, w.prefix_parts, 0);
        prefix = a;
    }
    a.table = c.table;
    a.width = c.width;
    a.q_start = c.q_start;
    a.kv_len = c.kv_len;
    a.B = c.B;
    const ca::Set own = planned(w.own, w.own_info, w.own_parts, w.own_runs);
    hipError_t e = hipSuccess;
    if (a.pieces) {
        ca::plan_kernel<<<dim3((unsigned)((w.own.target + 63) / 64)), 64, 0, s>>>(a, w.own.rows);
        e = hipGetLastError();
    }
    if (e == hipSuccess)
        e = ca::with_format(c.pool, [&](auto fmt, auto d) {
            constexpr int F = decltype(fmt)::value, D = decltype(d)::value;
            if (prefix_pages > 0 && w.own.rows == 16)
                return ca::launch_shared<F, D>(prefix, w.prefix.rows, w.prefix.grid, a, w.own.grid, s);
            if (prefix_pages > 0) {
                const hipError_t first = ca::launch<F, D>(prefix, w.prefix.rows, w.prefix.grid, s);
                if (first != hipSuccess) return first;
            }
            return ca::launch<F, D>(a, w.own.rows, w.own.grid, s);
        });
    if (e != hipSuccess || w.own.slots == 0) return e;
    return c.pool.d == 64 ? ca::launch_merge<64>(a, own, shared, s) : ca::launch_merge<128>(a, own, shared, s);
}

}  // namespace dn
