// attention_cache.hip -- deferred Softmax -> P.V of ragged sequences over the paged key/value cache:
//
//   out = sum_j 2^(s_j - m) v_j V_j / sum_j 2^(s_j - m),   s_j = scale log2(e) k_j (q . K_j),
//
// K_j, V_j the codes of token j and k_j, v_j their scales: a scale is one number per key, so it
// multiplies the key's score (k_j) and numerator (v_j) and no code is scaled by itself.  Both
// products are taken transposed, as in attention.hip: a lane keeps one query, and the numerators
// go from the scores' accumulators straight into the second product (kv_layout.hpp).
//
// Numerators are rounded to bf16, the matrix cores' operand (2^-8 relative at most, the size of the
// output's own rounding); scores, maximum, sums and partial sums are fp32.  Queries see keys up to
// their own: query i of n sees keys 0 .. kv_len - n + i.  A masked key weighs exactly 0 whatever
// its slot holds: its numerator is selected away, and V codes past kv_len are zeroed before the
// product (codes below are finite: rows with NaN or infinities are held as a NaN scale).
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
    int4* info;    // [B]: first slot, pages per chunk, chunks of the longest tile, 0
    float* parts;  // [slots][rows][d + 4]: sums, l, m
    __bf16* out;   // [T][heads * group][d]
};

struct Seq {
    int first, n, len, pages;  // first token, tokens, keys, pages of keys
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
    int per;       // pages per chunk
    int64_t slot;  // of this item, where its tile has several chunks
    Seq s;
};

// exclusive scan over the 256 threads of a workgroup; total in every thread
__device__ __forceinline__ int64_t scan256(int64_t v, int64_t* lds, int64_t& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int64_t t = lds[w];
        before += w < wave ? t : 0;
        total += t;
    }
    return before + x - v;
}

// Which item this workgroup takes: false where there is none left.  Sequences in order, of each its
// tiles from the last (which sees the most keys) to the first, of each its chunks, of each the heads
// (consecutive workgroups go to different XCDs: with 8 heads one XCD reads one head's keys).
__device__ __forceinline__ bool find_item(const Args& a, int rows, Item& it) {
    __shared__ int64_t lds[4];
    __shared__ Item found;
    const int64_t id = blockIdx.x;
    const int tid = threadIdx.x;
    int64_t cost = 0, total;
    Seq mine{};
    for (int64_t b = tid; b < a.B; b += 256) {
        mine = sequence(a, b);
        const int64_t tiles = ((int64_t)mine.n * a.group + rows - 1) / rows;
        cost += tiles * mine.pages * a.heads;
    }
    scan256(cost, lds, total);
    const int64_t per = max(a.least, (total + a.target - 1) / a.target);
    int64_t items_before = 0, slots_before = 0;
    if (tid == 0) found.b = -1;
    for (int64_t b0 = 0; b0 < a.B; b0 += 256) {
        const int64_t b = b0 + tid;
        int64_t items = 0, parts = 0, chunks = 1;
        if (b < a.B) {
            if (a.B > 256) mine = sequence(a, b);
            const int64_t tiles = ((int64_t)mine.n * a.group + rows - 1) / rows;
            chunks = max((int64_t)1, (mine.pages + per - 1) / per);
            items = tiles * chunks * a.heads;
            parts = a.always_partial || chunks > 1 ? items : 0;
        }
        int64_t items_total, parts_total;
        const int64_t ib = items_before + scan256(items, lds, items_total);
        const int64_t pb = slots_before + scan256(parts, lds, parts_total);
        if (items > 0 && id >= ib && id < ib + items) {
            const int64_t at = id - ib, rest = at / a.heads;
            const int64_t tiles = items / (chunks * a.heads);
            found.b = (int)b;
            found.head = (int)(at - rest * a.heads);
            found.chunk = (int)(rest % chunks);
            found.tile = (int)(tiles - 1 - rest / chunks);
            found.per = (int)per;
            // slots go by tile, chunk and head, whatever order the items have
            found.slot = pb + ((int64_t)found.tile * chunks + found.chunk) * a.heads + found.head;
            found.s = mine;
            if (at == 0 && a.info) a.info[b] = int4{(int)pb, (int)per, (int)chunks, 0};
        }
        items_before += items_total;
        slots_before += parts_total;
        if (id < items_before) break;
    }
    __syncthreads();
    it = found;
    return it.b >= 0;
}

// Keys that some query of the tile sees.
__device__ __forceinline__ int tile_keys(const Args& a, const Seq& s, int tile, int rows) {
    if (!a.kv_len) return s.len;
    const int last = (int)min((int64_t)s.n - 1, ((int64_t)tile * rows + rows - 1) / a.group);
    return min(s.len, max(s.len - s.n + last + 1, 0));
}
__device__ __forceinline__ int tile_chunks(int keys, int per) {
    return max(1, ((keys + kKvPage - 1) / kKvPage + per - 1) / per);
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

// Zeroes the codes of a V chunk's tokens from the `keep`-th of the lane's on.
template <int FMT>
__device__ __forceinline__ u32x4 keep_tokens(u32x4 c, int keep) {
    constexpr int PER = FMT == kKvBf16 ? 2 : 4, BITS = 32 / PER;  // tokens in a word
    uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int left = keep - j * PER;
        w[j] = left >= PER ? w[j] : left <= 0 ? 0u : w[j] & ((1u << (left * BITS)) - 1u);
    }
    return u32x4{w[0], w[1], w[2], w[3]};
}

__device__ __forceinline__ float weight(float m, float mn) {
    return m != -__builtin_inff() ? __builtin_amdgcn_exp2f(m - mn) : 0.f;
}

// Softmax state of one 16-query block: the reference maximum, raised only when a unit exceeds it by
// more than 2^8 (numerators stay below 256), and the lane's share of the sum.
struct State {
    float m, l;
};

// Scores of TILES key tiles (16 each, of one unit) -> numerators as operands.  s holds q . K; ks, vs
// the lane's scales of each tile's four keys; lim: the last unit key that this lane's query sees.
template <int TILES, int D, bool MASK>
__device__ __forceinline__ void softmax_unit(const f32x4 (&s)[TILES], const float4 (&ks)[TILES], const float4 (&vs)[TILES],
                                             const int (&key0)[TILES], int lim, float sl2, State& st, f32x4 (&acc)[D / 16],
                                             u32x4 (&pf)[TILES / 2]) {
    float x[TILES][4];
    float top = -__builtin_inff();
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const float k4[4] = {ks[t].x, ks[t].y, ks[t].z, ks[t].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[t][i] = s[t][i] * (k4[i] * sl2);
            if (MASK) x[t][i] = key0[t] + i <= lim ? x[t][i] : -__builtin_inff();
            top = fmaxf(top, x[t][i]);
        }
    }
    top = max_lane_groups(top);
    if (__any(top > st.m + 8.f)) {
        const float mn = fmaxf(top, st.m), w = weight(st.m, mn);
        st.m = mn;
        st.l *= w;
#pragma unroll
        for (int n = 0; n < D / 16; ++n) acc[n] *= w;
    }
    const float m = st.m == -__builtin_inff() ? 0.f : st.m;
#pragma unroll
    for (int t = 0; t < TILES; t += 2) {
        float p[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float v4[4] = {vs[t + h].x, vs[t + h].y, vs[t + h].z, vs[t + h].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(x[t + h][i] - m);
                const bool on = !MASK || key0[t + h] + i <= lim;
                st.l += on ? e : 0.f;
                p[4 * h + i] = on ? e * v4[i] : 0.f;
            }
        }
        pf[t / 2] = u32x4{pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])};
    }
}

// ----------------------------------------------------------------------------- few rows
// Tiles of 16 rows.  Bound by HBM: each wave takes pages of the chunk in turn, its codes straight to
// registers (V of a unit and K of the next in flight while the unit's scores are worked on), and
// the four waves' sums meet in LDS at the end.
template <int FMT, int D>
__global__ __launch_bounds__(256) void decode_kernel(const Args a) {
    using B = KvBlock<FMT, D>;
    constexpr int E = B::E, R = 16, UNITS = kKvPage / (4 * E), TILES = E / 4, KC = D / (4 * E), NB = D / 16;
    constexpr int LOADS = NB;  // chunks of K, and of V, in a unit
    static_assert(TILES * KC == LOADS, "");
    constexpr int PITCH = D + 4;
    __shared__ __attribute__((aligned(16))) float sums[4][R][PITCH];
    __shared__ float ml[4][2][R];

    Item it;
    if (!find_item(a, R, it)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q = lane & 15, G = lane >> 4;
    const int keys = tile_keys(a, it.s, it.tile, R), chunks = tile_chunks(keys, it.per);
    if (it.chunk >= chunks) return;
    const bool partial = a.always_partial || chunks > 1;
    if (partial && it.slot >= a.slots) return;

    // this lane's query
    const int64_t row = (int64_t)it.tile * R + q;
    const int rows_here = (int)min((int64_t)R, (int64_t)it.s.n * a.group - (int64_t)it.tile * R);
    const int64_t rr = q < rows_here ? row : row - q;
    const int qi = (int)(rr / a.group), qh = it.head * a.group + (int)(rr % a.group);
    const __bf16* qp = a.Q + (int64_t)(it.s.first + qi) * a.q_stride + (int64_t)qh * D;
    u32x4 qf[D / 32];
#pragma unroll
    for (int c = 0; c < KC; ++c)
#pragma unroll
        for (int j = 0; j < E / 8; ++j) qf[c * (E / 8) + j] = ld16(qp + 4 * E * c + E * G + 8 * j);
    const int lim = a.kv_len ? it.s.len - it.s.n + qi : it.s.len - 1;
    // the first query of the tile sees the fewest keys
    const int lim_min = a.kv_len ? it.s.len - it.s.n + (int)((int64_t)it.tile * R / a.group) : it.s.len - 1;

    f32x4 acc[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    State st{-__builtin_inff(), 0.f};

    const int page_lo = it.chunk * it.per, page_hi = min(page_lo + it.per, (keys + kKvPage - 1) / kKvPage);
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
    const int total = count * UNITS;
    const char* block = nullptr;
    if (total > 0) {
        block = block_of(0);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) kf[i] = ld16_stream(block + i * kChunkBytes + lane * 16);
    }
    for (int un = 0; un < total; ++un) {
        const int u = un % UNITS, page = page_lo + wave + 4 * (un / UNITS);
        float4 ks[TILES], vs[TILES];
        int key0[TILES];
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const int o = 4 * E * u + E * G + 4 * t;
            ks[t] = *reinterpret_cast<const float4*>(block + B::KS + 4 * o);
            vs[t] = *reinterpret_cast<const float4*>(block + B::VS + 4 * o);
            key0[t] = page * kKvPage + o;
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) vf[i] = ld16_stream(block + B::PART + (u * LOADS + i) * kChunkBytes + lane * 16);
        f32x4 s[TILES];
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < KC; ++c)
#pragma unroll
                for (int j = 0; j < E / 8; ++j)
                    s[t] = mfma_chunk<__bf16>(frag<FMT>(kf[t * KC + c], j), qf[c * (E / 8) + j], s[t]);
        }
        if (un + 1 < total) {
            const int nu = (un + 1) % UNITS;
            if (nu == 0) block = block_of((un + 1) / UNITS);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) kf[i] = ld16_stream(block + (nu * LOADS + i) * kChunkBytes + lane * 16);
        }
        u32x4 pf[TILES / 2];
        const int end = page * kKvPage + 4 * E * (u + 1);  // first key past the unit
        if (end - 1 > lim_min) {
            softmax_unit<TILES, D, true>(s, ks, vs, key0, lim, a.sl2, st, acc, pf);
            if (end > it.s.len) {
                const int keep = min(max(it.s.len - (page * kKvPage + 4 * E * u + E * G), 0), E);
#pragma unroll
                for (int i = 0; i < LOADS; ++i) vf[i] = keep_tokens<FMT>(vf[i], keep);
            }
        } else {
            softmax_unit<TILES, D, false>(s, ks, vs, key0, lim, a.sl2, st, acc, pf);
        }
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int j = 0; j < E / 8; ++j) acc[n] = mfma_chunk<__bf16>(frag<FMT>(vf[n], j), pf[j], acc[n]);
    }

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
        float m = -__builtin_inff(), w[4], lt = 0.f, o[PER];
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
            float* part = a.parts + (it.slot * R + r) * (int64_t)(D + 4);
            *reinterpret_cast<f32x4*>(part + x) = f32x4{o[0], o[1], o[2], o[3]};
            *reinterpret_cast<f32x4*>(part + x + 4) = f32x4{o[4], o[5], o[6], o[7]};
            if (x == 0) *reinterpret_cast<f32x4*>(part + D) = f32x4{lt, m, 0.f, 0.f};
        } else {
            const int i_q = (int)(ro / a.group);
            const bool none = a.kv_len && it.s.len - it.s.n + i_q < 0;  // no key at all: zero
            const float inv = none ? 0.f : 1.0f / lt;
            uint32_t pk[PER / 2];
#pragma unroll
            for (int e = 0; e < PER / 2; ++e) pk[e] = none ? 0u : pack_bf16(o[2 * e] * inv, o[2 * e + 1] * inv);
            const int64_t oh = (int64_t)(it.s.first + i_q) * a.heads * a.group + it.head * a.group + ro % a.group;
            *reinterpret_cast<u32x4*>(a.out + oh * D + x) = u32x4{pk[0], pk[1], pk[2], pk[3]};
        }
    }
}

// ----------------------------------------------------------------------------- many rows
// Tiles of 4 waves x QW x 16 rows.  Bound by the matrix cores: a page's codes go through LDS (two
// slots, copied while the page before is worked on) and serve the tile's four waves.
template <int FMT, int D, int QW>
__global__ __launch_bounds__(256, 2) void tile_kernel(const Args a) {
    using B = KvBlock<FMT, D>;
    constexpr int E = B::E, R = 64 * QW, TILES = 4, KC = D / (4 * E), NB = D / 16;
    constexpr int CHUNKS = 2 * B::PART / kChunkBytes;           // K and V codes
    constexpr int SLOT = 2 * B::PART + 8 * kKvPage;             // and the scales
    __shared__ __attribute__((aligned(1024))) char smem[2 * ((SLOT + 1023) / 1024 * 1024)];
    constexpr int STEP = (SLOT + 1023) / 1024 * 1024;

    Item it;
    if (!find_item(a, R, it)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int q = lane & 15, G = lane >> 4;
    const int keys = tile_keys(a, it.s, it.tile, R), chunks = tile_chunks(keys, it.per);
    if (it.chunk >= chunks) return;
    const bool partial = a.always_partial || chunks > 1;
    if (partial && it.slot >= a.slots) return;

    const int64_t rows_all = (int64_t)it.s.n * a.group;
    const int64_t row0 = (int64_t)it.tile * R + wave * QW * 16;  // the wave's first row
    u32x4 qf[QW][D / 32];
    int lim[QW], lim_min;
#pragma unroll
    for (int f = 0; f < QW; ++f) {
        const int64_t row = min(row0 + f * 16 + q, rows_all - 1);
        const int qi = (int)(row / a.group), qh = it.head * a.group + (int)(row % a.group);
        const __bf16* qp = a.Q + (int64_t)(it.s.first + qi) * a.q_stride + (int64_t)qh * D;
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int j = 0; j < E / 8; ++j) qf[f][c * (E / 8) + j] = ld16(qp + 4 * E * c + E * G + 8 * j);
        lim[f] = a.kv_len ? it.s.len - it.s.n + qi : it.s.len - 1;
    }
    lim_min = a.kv_len ? it.s.len - it.s.n + (int)(min(row0, rows_all - 1) / a.group) : it.s.len - 1;

    f32x4 acc[QW][NB];
    State st[QW];
#pragma unroll
    for (int f = 0; f < QW; ++f) {
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[f][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        st[f] = State{-__builtin_inff(), 0.f};
    }

    const int page_lo = it.chunk * it.per, page_hi = min(page_lo + it.per, (keys + kKvPage - 1) / kKvPage);
    const int count = page_hi - page_lo;
    const int64_t page_bytes = (int64_t)a.heads * B::SIZE;
    const char* head_base = a.pool + (int64_t)it.head * B::SIZE;
    const uint32_t lds0 = lds_addr32(smem);
    int ids = 0;
    auto issue = [&](int k) __attribute__((always_inline)) {
        if (k % 64 == 0) ids = k + lane < count ? page_at(a, it.b, page_lo + k + lane) : 0;
        const uint64_t src = uniform_u64(head_base + (int64_t)__builtin_amdgcn_readlane(ids, k % 64) * page_bytes);
        const uint32_t dst = lds0 + (uint32_t)(k & 1) * STEP;
#pragma unroll
        for (int i = 0; i < CHUNKS / 4; ++i) {
            const uint32_t at = (uint32_t)(wave + 4 * i) * kChunkBytes;
            g2lds16_async_sb(src, at + lane * 16, dst + at);
        }
        // the scales: half a KiB, the first 32 lanes of one wave
        if (wave == 0 && lane < 32) g2lds16_async_sb(src, (uint32_t)B::KS + lane * 16, dst + (uint32_t)B::KS);
    };
    if (count > 0) issue(0);
    for (int k = 0; k < count; ++k) {
        wait_vm();
        __syncthreads();  // page k has landed, and every wave is done with page k - 1
        if (k + 1 < count) issue(k + 1);
        const char* slot = smem + (k & 1) * STEP;
        const int base = (page_lo + k) * kKvPage;
        f32x4 s[QW][TILES];
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
#pragma unroll
            for (int f = 0; f < QW; ++f) s[f][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                const u32x4 kf = lds_ld16(lds_ptr((char*)slot + (t * KC + c) * kChunkBytes + lane * 16));
#pragma unroll
                for (int j = 0; j < E / 8; ++j) {
                    const u32x4 b = frag<FMT>(kf, j);
#pragma unroll
                    for (int f = 0; f < QW; ++f) s[f][t] = mfma_chunk<__bf16>(b, qf[f][c * (E / 8) + j], s[f][t]);
                }
            }
        }
        float4 ks[TILES], vs[TILES];
        int key0[TILES];
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const int o = t * 4 / E * 4 * E + E * G + t * 4 % E;  // tile t's first token of lane group G
            ks[t] = *reinterpret_cast<const float4*>(slot + B::KS + 4 * o);
            vs[t] = *reinterpret_cast<const float4*>(slot + B::VS + 4 * o);
            key0[t] = base + o;
        }
        u32x4 pf[QW][TILES / 2];
        const bool masked = base + kKvPage - 1 > lim_min;
#pragma unroll
        for (int f = 0; f < QW; ++f) {
            if (masked)
                softmax_unit<TILES, D, true>(s[f], ks, vs, key0, lim[f], a.sl2, st[f], acc[f], pf[f]);
            else
                softmax_unit<TILES, D, false>(s[f], ks, vs, key0, lim[f], a.sl2, st[f], acc[f], pf[f]);
        }
        const bool cut = base + kKvPage > it.s.len;
#pragma unroll
        for (int u = 0; u < kKvPage / (4 * E); ++u) {
            const int keep = min(max(it.s.len - (base + 4 * E * u + E * G), 0), E);
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                u32x4 vf = lds_ld16(lds_ptr((char*)slot + B::PART + (u * NB + n) * kChunkBytes + lane * 16));
                if (cut) vf = keep_tokens<FMT>(vf, keep);
#pragma unroll
                for (int j = 0; j < E / 8; ++j) {
                    const u32x4 b = frag<FMT>(vf, j);
#pragma unroll
                    for (int f = 0; f < QW; ++f) acc[f][n] = mfma_chunk<__bf16>(b, pf[f][u * (E / 8) + j], acc[f][n]);
                }
            }
        }
    }

#pragma unroll
    for (int f = 0; f < QW; ++f) {
        const int64_t row = row0 + f * 16 + q;
        const float l = sum_lane_groups(st[f].l);
        if (row >= rows_all) continue;
        if (partial) {
            float* part = a.parts + (it.slot * R + (row - (int64_t)it.tile * R)) * (int64_t)(D + 4);
#pragma unroll
            for (int n = 0; n < NB; ++n) *reinterpret_cast<f32x4*>(part + 16 * n + 4 * G) = acc[f][n];
            if (G == 0) *reinterpret_cast<f32x4*>(part + D) = f32x4{l, st[f].m, 0.f, 0.f};
        } else {
            const int qi = (int)(row / a.group);
            const bool none = lim[f] < 0;
            const float inv = 1.0f / l;
            const int64_t oh = (int64_t)(it.s.first + qi) * a.heads * a.group + it.head * a.group + row % a.group;
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const uint2 v = {pack_bf16(acc[f][n][0] * inv, acc[f][n][1] * inv),
                                 pack_bf16(acc[f][n][2] * inv, acc[f][n][3] * inv)};
                *reinterpret_cast<uint2*>(a.out + oh * D + 16 * n + 4 * G) = none ? uint2{0, 0} : v;
            }
        }
    }
}

// ----------------------------------------------------------------------------- merge
struct Set {
    const int4* info;
    const float* parts;
    int64_t slots;
    int rows;
};

// Partial sums of a row: the first one's slot, the next ones `heads` slots further each.  0 where the
// plan that a sequence's workgroups left does not fit the workspace (q_start out of order).
__device__ __forceinline__ int parts_of(const Set& set, const int4& plan, int tile, int chunks, int heads, int h,
                                        int64_t& first) {
    first = plan.x + (int64_t)tile * plan.z * heads + h;
    return first >= 0 && first + (int64_t)(chunks - 1) * heads < set.slots ? chunks : 0;
}

// One output row per workgroup: D / 4 threads over its dimensions, the others over its partial sums.
// `shared` (parts null: none) holds the partial sums over the prefix, `own` those over the
// sequence's own keys; without a prefix rows whose tile has one chunk are already written.
template <int D>
__global__ __launch_bounds__(256) void merge_kernel(const Args a, const Set own, const Set shared) {
    constexpr int NX = D / 4, NS = 256 / NX;
    __shared__ int found;
    __shared__ __attribute__((aligned(16))) float red[NS][D + 4];
    __shared__ float red_m[NS];
    const int tid = threadIdx.x;
    const int hq = blockIdx.x % (a.heads * a.group);
    const int64_t token = blockIdx.x / (a.heads * a.group);
    if (tid == 0) found = -1;
    __syncthreads();
    for (int64_t b = tid; b < a.B; b += 256)
        if (a.q_start[b] <= token && token < a.q_start[b + 1]) found = (int)b;
    __syncthreads();
    const int b = found;
    if (b < 0) return;
    const Seq s = sequence(a, b);
    const int h = hq / a.group, r = hq % a.group;
    int64_t first[2] = {0, 0};
    int count[2] = {0, 0}, at[2] = {0, 0}, lim_keys;
    const float* base[2] = {own.parts, shared.parts};
    {
        const int4 info = own.info[b];
        const int64_t row = (token - s.first) * a.group + r;
        const int tile = (int)(row / own.rows);
        const int chunks = tile_chunks(tile_keys(a, s, tile, own.rows), max(info.y, 1));
        lim_keys = s.len - s.n + (int)(token - s.first) + 1;
        if (!shared.parts && chunks == 1) return;
        at[0] = (int)(row % own.rows);
        count[0] = parts_of(own, info, tile, chunks, a.heads, h, first[0]);
    }
    if (shared.parts) {
        const int4 info = shared.info[0];
        const int64_t row = token * a.group + r;
        const int tile = (int)(row / shared.rows);
        at[1] = (int)(row % shared.rows);
        count[1] = parts_of(shared, info, tile, info.z, a.heads, h, first[1]);
    }
    const int x = tid % NX * 4, g = tid / NX;
    float m = -__builtin_inff(), l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const int rows = w ? shared.rows : own.rows;
        for (int c = g; c < count[w]; c += NS) {
            const float* part = base[w] + ((first[w] + (int64_t)c * a.heads) * rows + at[w]) * (int64_t)(D + 4);
            const f32x4 v = *reinterpret_cast<const f32x4*>(part + x), t = *reinterpret_cast<const f32x4*>(part + D);
            const float mn = fmaxf(m, t[1]), wo = weight(m, mn), wn = weight(t[1], mn);
            l = wo * l + wn * t[0];
            o = o * wo + v * wn;
            m = mn;
        }
    }
    *reinterpret_cast<f32x4*>(&red[g][x]) = o;
    if (x == 0) {
        red[g][D] = l;
        red_m[g] = m;
    }
    __syncthreads();
    if (g) return;
    float mt = -__builtin_inff(), lt = 0.f;
#pragma unroll
    for (int v = 0; v < NS; ++v) mt = fmaxf(mt, red_m[v]);
    f32x4 ot = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < NS; ++v) {
        const float w = weight(red_m[v], mt);
        lt += w * red[v][D];
        ot += *reinterpret_cast<const f32x4*>(&red[v][x]) * w;
    }
    const bool none = !shared.parts && lim_keys <= 0;
    const float inv = 1.0f / lt;
    const uint2 v = {pack_bf16(ot[0] * inv, ot[1] * inv), pack_bf16(ot[2] * inv, ot[3] * inv)};
    *reinterpret_cast<uint2*>(a.out + (token * a.heads * a.group + hq) * D + x) = none ? uint2{0, 0} : v;
}

template <int FMT, int D>
hipError_t launch(const Args& a, int rows, int64_t grid, hipStream_t s) {
    const dim3 g((unsigned)grid);
    if (rows == 16)
        decode_kernel<FMT, D><<<g, 256, 0, s>>>(a);
    else if (rows == 64)
        tile_kernel<FMT, D, 1><<<g, 256, 0, s>>>(a);
    else
        tile_kernel<FMT, D, 2><<<g, 256, 0, s>>>(a);
    return hipGetLastError();
}
hipError_t launch_any(const KvPool& c, const Args& a, int rows, int64_t grid, hipStream_t s) {
    if (c.format == kKvBf16)
        return c.d == 64 ? launch<kKvBf16, 64>(a, rows, grid, s) : launch<kKvBf16, 128>(a, rows, grid, s);
    return c.d == 64 ? launch<kKvFp8, 64>(a, rows, grid, s) : launch<kKvFp8, 128>(a, rows, grid, s);
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
    ca::Args own = a, pre = a;
    ca::Set shared{};
    if (prefix_pages > 0) {
        pre.table = c.prefix_table;
        pre.width = prefix_pages;
        pre.prefix = c.prefix;
        pre.B = 1;
        pre.target = w.prefix.target;
        pre.least = w.prefix.least;
        pre.slots = w.prefix.slots;
        pre.always_partial = 1;
        pre.info = (int4*)ws + c.B;
        pre.parts = (float*)(ws + w.prefix_slots);
        const hipError_t e = ca::launch_any(c.pool, pre, w.prefix.rows, w.prefix.grid, s);
        if (e != hipSuccess) return e;
        shared = ca::Set{pre.info, pre.parts, pre.slots, w.prefix.rows};
    }
    own.table = c.table;
    own.width = c.width;
    own.q_start = c.q_start;
    own.kv_len = c.kv_len;
    own.B = c.B;
    own.target = w.own.target;
    own.least = w.own.least;
    own.slots = w.own.slots;
    own.always_partial = prefix_pages > 0;
    own.info = (int4*)ws;
    own.parts = (float*)(ws + w.own_slots);
    const hipError_t e = ca::launch_any(c.pool, own, w.own.rows, w.own.grid, s);
    if (e != hipSuccess || (w.own.slots == 0 && prefix_pages == 0)) return e;
    const ca::Set set{own.info, own.parts, own.slots, w.own.rows};
    const dim3 g((unsigned)(c.T * c.q_heads));
    if (c.pool.d == 64)
        ca::merge_kernel<64><<<g, 256, 0, s>>>(own, set, shared);
    else
        ca::merge_kernel<128><<<g, 256, 0, s>>>(own, set, shared);
    return hipGetLastError();
}

}  // namespace dn
