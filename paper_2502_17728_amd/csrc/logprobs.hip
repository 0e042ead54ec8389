// logprobs.hip -- log probabilities of given tokens, entropy and the likeliest tokens of each row of
// logits, in one pass.
//
// With m the row's maximum and d = scale (x - m): l = sum e^d, s = sum e^d d, and then
//     ln p_i = d_i - ln l,     entropy = ln l - s / l,
// so the normalization (Eq. (7) with the max subtraction of its footnote) is applied to the tokens
// asked for alone, after the pass.  Each lane keeps its own (m, l, s); on a larger m' they become
// f l and f (s + d' l) with d' = scale (m - m'), f = e^d'.  Exponents are to base 2 inside.
//
// The likeliest tokens are 64-bit keys: the logit's bits in an order that integers share, then the
// complement of the token's id, so that the larger key is the likelier token and, among equals, the
// lower id.  A wave puts the groups of 8 tokens whose largest may belong to the likeliest aside, in
// LDS; every few dozen groups their tokens are filtered, and a search by bits over the keys (one
// ballot a bit) finds a bound that `top` of them reach and drops the rest.  The first bound comes so from the
// lanes' maxima of the first 512 tokens; a row of random order is searched about five times.  The waves'
// keys are then cut together, and only what is left, about `top` keys, is put in order.
//
// Bound by HBM where fp32 is read (4000 x 32001 88 us, 5.8 TB/s), by the VALU in bf16 (1000 x 100003 34 us without ranks,
// 46 with 20, 47.5 on other logits each time; HBM 29), by launches and the serial ranking for short inputs (1 x 8192 6.4 us,
// 32 x 131072 12.7 and a join).
#include "dn_device.hpp"
#include "dn_launch.hpp"
#include "fp8_rules.hpp"

namespace dn {

constexpr float kLowest = -3.402823466e38f;
// 2^-200 is 0 in fp32; keeps 0 * -inf out of the sums.  (x - m may pass fp32's range: with a scale of 2^-96 or more, which calls have,
// such a token's power is below e^(-2^32).)
constexpr float kLeastExponent = -200.f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kBuffer = 128;                 // keys of a wave's list
constexpr int kMostKept = 72;                // of which a cut leaves at most: `top` (at most 64) and 8 more
constexpr int kFlush = 32, kGroups = kFlush + 64;  // groups put aside: looked at past kFlush, and 64 more fit

struct LpArgs {
    const void* logits;
    int64_t stride, T, V, n;
    float scale;
    int top;
    int segments;
    const int32_t* targets;
    float *logprobs, *entropy, *top_logprobs;
    int32_t* top_ids;
    float* part_sums;              // [T][segments][4]
    unsigned long long* part_top;  // [T][segments][top]
};

// ------------------------------------------------------------------------------- sums
struct Sums {
    float m, l, s;
};
__device__ __forceinline__ float exponent(float x, float m, float c) { return (x - m) * c; }  // c = scale log2 e

__device__ __forceinline__ void raise(Sums& a, float m, float c) {
    const float d = exponent(a.m, m, c), f = __builtin_amdgcn_exp2f(d);
    a.s = f * __builtin_fmaf(__builtin_fmaxf(d, kLeastExponent), a.l, a.s);
    a.l *= f;
    a.m = m;
}
__device__ __forceinline__ void join(Sums& a, Sums b, float c) {
    const float m = __builtin_fmaxf(a.m, b.m);
    raise(a, m, c);
    raise(b, m, c);
    a.l += b.l;
    a.s += b.s;
}
// Reductions over the wave's 64 lanes without LDS: pairs, quads, halves of a row of 16, then rows.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false);
}
template <class F>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t v, F f) {
    v = f(v, dpp<0xB1>(v));   // lane ^ 1
    v = f(v, dpp<0x4E>(v));   // lane ^ 2
    v = f(v, dpp<0x141>(v));  // the row's halves mirrored
    v = f(v, dpp<0x140>(v));  // the row mirrored
    const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = f(p[0], p[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return f(q[0], q[1]);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    return wave_reduce(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ float wave_maxf(float v) {
    return __uint_as_float(wave_reduce(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__builtin_fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }));
}
__device__ __forceinline__ float wave_addf(float v) {
    return __uint_as_float(wave_reduce(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}
__device__ __forceinline__ Sums wave_join(Sums a, float c) {
    raise(a, wave_maxf(a.m), c);
    a.l = wave_addf(a.l);
    a.s = wave_addf(a.s);
    return a;
}

// ------------------------------------------------------------------------------- ranks
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);  // -0 ranks as +0
    return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(unsigned long long key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ uint32_t id_of(unsigned long long key) { return ~(uint32_t)key; }

__device__ __forceinline__ void lds_in_order() { asm volatile("" ::: "memory"); }  // a wave's LDS instructions are served in order

__device__ __forceinline__ int lanes_below(unsigned long long mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

__device__ __forceinline__ uint32_t wave_min(uint32_t v) {
    return wave_reduce(v, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}

// A t of which count(t) >= top, where count(lo) >= top and no value is above hi: the largest whose bits below `least` are
// zero, or a smaller one with count(t) <= enough.
template <class F>
__device__ __forceinline__ uint32_t search(uint32_t lo, uint32_t hi, int least, int top, int enough, F count) {
    if (lo >= hi) return lo;
    int bit = 31 - __builtin_clz(lo ^ hi);
    uint32_t t = lo & ~((2u << bit) - 1);  // what lo and hi share
    for (; bit >= least; --bit) {
        const uint32_t next = t | (1u << bit);
        const int n = count(next);
        if (n >= top) {
            t = next;
            if (n <= enough) break;
        }
    }
    return t > lo ? t : lo;
}

// A wave's part of LDS
struct WaveRanks {
    unsigned long long keys[kBuffer];
    float values[kGroups * 8];
    uint32_t first[kGroups];
};

// A wave's likeliest tokens so far: n keys, none below `floor`, and groups of 8 tokens that have not been looked at.
// A further token counts if the order of its logit is `bar` or more, which is to say the logit `least` or more.
struct Ranked {
    DN_LDS WaveRanks* m;
    int n, groups, top;
    uint32_t floor, bar;
    float least;

    __device__ __forceinline__ void set_bar(uint32_t b) {
        bar = b;
        // orders up to that of -inf belong to NaNs of either sign: every number counts
        least = b <= 0x007fffffu ? -__builtin_inff() : value_of((unsigned long long)b << 32);
    }

    // From the lanes' maxima of the first tokens (NaN where a lane has none, or NaNs among them): at least `top` tokens are not below
    // what `top` of these reach, and the rest need not be kept.
    __device__ __forceinline__ void start(float most) {
        const uint32_t o = most == most ? order_of(most) : 0;
        floor = search(wave_min(o), wave_max(o), 16, top, top + 1, [&](uint32_t t) { return __popcll(__ballot(o >= t)); });
        set_bar(floor);
    }

    // Sorts the keys and cuts them to `top`, by counting the larger ones.
    __device__ __forceinline__ void rank(int lane) {
        lds_in_order();
        DN_LDS unsigned long long* k = m->keys;
        const unsigned long long a = lane < n ? k[lane] : 0, b = 64 + lane < n ? k[64 + lane] : 0;
        if (lane >= n && lane < n + 8) k[lane] = 0;  // whole groups of 8 below
        if (64 + lane >= n && 64 + lane < n + 8) k[64 + lane] = 0;
        lds_in_order();
        typedef unsigned long long u64x2 __attribute__((ext_vector_type(2)));
        int ra = 0, rb = 0;
        for (int i = 0; i < n; i += 8) {
            u64x2 o[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = *reinterpret_cast<DN_LDS u64x2*>(k + i + 2 * j);
#pragma unroll
            for (int j = 0; j < 8; ++j) ra += o[j / 2][j & 1] > a;
            if (n > 64) {
#pragma unroll
                for (int j = 0; j < 8; ++j) rb += o[j / 2][j & 1] > b;
            }
        }
        lds_in_order();
        if (lane < n && ra < top) k[ra] = a;
        if (64 + lane < n && rb < top) k[rb] = b;
        lds_in_order();
        if (n >= top) {
            n = top;
            floor = (uint32_t)__builtin_amdgcn_readfirstlane((int)(k[top - 1] >> 32));
            set_bar(floor);
        }
    }

    // The list takes chunk() further tokens after a cut, which leaves kept() keys at most: for the largest `top` a few
    // more than `top`, so that a cut needs no order (64 of 256 x 32000 logits 44 -> 30 us).
    __device__ __forceinline__ int chunk() const { return top > 56 ? kBuffer - kMostKept : 64; }
    __device__ __forceinline__ int kept() const { return kBuffer - chunk(); }

    // Drops keys that `top` others are above.
    __device__ __forceinline__ void cut(int lane) {
        lds_in_order();
        const unsigned long long a = lane < n ? m->keys[lane] : 0, b = 64 + lane < n ? m->keys[64 + lane] : 0;
        const uint32_t ha = (uint32_t)(a >> 32), hb = (uint32_t)(b >> 32);
        floor = search(floor, wave_max(ha > hb ? ha : hb), 8, top, top + 8,
                       [&](uint32_t t) { return __popcll(__ballot(ha >= t)) + __popcll(__ballot(hb >= t)); });
        const bool ka = a != 0 && ha >= floor, kb = b != 0 && hb >= floor;
        const unsigned long long ma = __ballot(ka), mb = __ballot(kb);
        if (ka) m->keys[lanes_below(ma)] = a;
        if (kb) m->keys[__popcll(ma) + lanes_below(mb)] = b;
        n = __popcll(ma) + __popcll(mb);
        lds_in_order();
        set_bar(floor);
        if (n > kept()) rank(lane);  // many equals
    }

    // The tokens of the groups put aside.  Later groups hold higher ids: of those, a logit that only equals the last
    // of `top` keys does not count.
    __device__ __forceinline__ void flush(int V, int lane) {
        lds_in_order();
        const int step = chunk();
        for (int i = 0; i < groups * 8; i += step) {
            const int at = i + lane, g = at >> 3;
            const bool there = lane < step && at < groups * 8;
            const float x = there ? m->values[at] : 0.f;
            const uint32_t id = there ? m->first[g] + (at & 7) : 0, o = order_of(x);
            bool keep = there && x == x && (int)id >= 0 && (int)id < V && o >= bar;
            unsigned long long mask = __ballot(keep);
            if (n + __popcll(mask) > kBuffer) {
                cut(lane);
                keep = keep && o >= bar;
                mask = __ballot(keep);
            }
            if (keep) m->keys[n + lanes_below(mask)] = ((unsigned long long)o << 32) | (uint32_t)~id;
            n += __popcll(mask);
        }
        groups = 0;
        if (n >= top) {
            cut(lane);
            if (floor != 0xffffffffu) set_bar(floor + 1);
        }
    }

    // f[0 .. 7] are tokens at, at + 1, .. (from V on they are none), `most` the largest of them, or NaN if one of them is: then the
    // group is put aside whatever its numbers are.  (Rows of nothing but NaNs, 1000 x 100003, take 118 us instead of 44 with
    // a look for their groups' numbers here, and all other rows 46.0 instead of 47.4.)
    __device__ __forceinline__ void add(const float* f, float most, int at, int V, int lane) {
        const bool keep = !(most < least);
        const unsigned long long mask = __ballot(keep);
        if (!mask) return;
        if (keep) {
            const int g = groups + lanes_below(mask);
            *reinterpret_cast<DN_LDS f32x4*>(&m->values[g * 8]) = f32x4{f[0], f[1], f[2], f[3]};
            *reinterpret_cast<DN_LDS f32x4*>(&m->values[g * 8 + 4]) = f32x4{f[4], f[5], f[6], f[7]};
            m->first[g] = (uint32_t)at;
        }
        groups += __popcll(mask);
        if (groups > kFlush) flush(V, lane);
    }
};

// The `top` largest of `total` keys (at most 64 CHUNKS; zeros are none) in order, by one wave: lane i gets the i-th,
// 0 where there are fewer.  At least `top` keys have order `lo` or more, if that is not 1.  `m` is scratch.
template <int CHUNKS>
__device__ __forceinline__ unsigned long long top_of_(const DN_LDS unsigned long long* keys, int total, int top, uint32_t lo_bound,
                                                      DN_LDS WaveRanks* m, int lane) {
    uint32_t hi[CHUNKS], lo[CHUNKS], most = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const unsigned long long k = c * 64 + lane < total ? keys[c * 64 + lane] : 0;
        hi[c] = (uint32_t)(k >> 32);
        lo[c] = (uint32_t)k;
        most = hi[c] > most ? hi[c] : most;
    }
    auto count = [&](uint32_t t) {
        int n = 0;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) n += __popcll(__ballot(hi[c] >= t));
        return n;
    };
    uint32_t t = lo_bound;
    const int all = count(t);
    int left = all;
    if (all > 64) {  // then at least `top` (at most 64)
        t = search(t, wave_max(most), 0, top, 64, count);
        left = count(t);
    }
    uint32_t last = 0;  // of the keys with order t, those whose lower half is `last` or more
    if (left > kBuffer) {
        const int above = t == 0xffffffffu ? 0 : count(t + 1);
        last = search(0, 0xffffffffu, 0, top - above, top - above, [&](uint32_t l) {
            int n = 0;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) n += __popcll(__ballot(hi[c] == t && lo[c] >= l));
            return n;
        });
    }
    Ranked r{m, 0, 0, top, 0, 0, 0.f};
    lds_in_order();
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const bool keep = hi[c] > t || (hi[c] == t && lo[c] >= last);
        const unsigned long long mask = __ballot(keep);
        if (keep) m->keys[r.n + lanes_below(mask)] = ((unsigned long long)hi[c] << 32) | lo[c];
        r.n += __popcll(mask);
    }
    r.rank(lane);
    return lane < r.n ? m->keys[lane] : 0;
}
__device__ __forceinline__ unsigned long long top_of(const DN_LDS unsigned long long* keys, int total, int top, uint32_t lo,
                                                     DN_LDS WaveRanks* m, int lane) {
    if (total <= 128) return top_of_<2>(keys, total, top, lo, m, lane);
    if (total <= 256) return top_of_<4>(keys, total, top, lo, m, lane);
    if (total <= 512) return top_of_<8>(keys, total, top, lo, m, lane);
    return top_of_<16>(keys, total, top, lo, m, lane);
}

// ------------------------------------------------------------------------------- results
// scale (x - m), also where x - m alone has no room in fp32 (halves are exact)
__device__ __forceinline__ float distance(float x, float m, float scale) { return (0.5f * x - 0.5f * m) * scale * 2.f; }

// A lane's first given token and its logit, read before the pass over the row.
struct Given {
    int32_t t;
    float x;
    template <class T>
    __device__ __forceinline__ void load(const LpArgs& p, int64_t row, const T* logits, int64_t i) {
        t = i < p.n ? p.targets[row * p.n + i] : -1;
        x = t >= 0 && t < p.V ? to_f32<T>(logits[t]) : 0.f;
    }
    __device__ __forceinline__ float logprob(const LpArgs& p, const Sums& a, float log_l) const {
        return t < 0 ? 0.f : t < p.V ? distance(x, a.m, p.scale) - log_l : __builtin_nanf("");
    }
};

template <class T>
__device__ __forceinline__ void finish(const LpArgs& p, int64_t row, const T* x, const Sums& a, unsigned long long key,
                                       Given given, int lane) {
    const float log_l = kLn2 * __builtin_amdgcn_logf(a.l);
    for (int64_t i = lane; i < p.n; i += kWave) {
        if (i >= kWave) given.load(p, row, x, i);
        p.logprobs[row * p.n + i] = given.logprob(p, a, log_l);
    }
    if (p.entropy && lane == 0) p.entropy[row] = log_l - kLn2 * (a.s / a.l);
    if (lane < p.top) {
        p.top_logprobs[row * p.top + lane] = key ? distance(value_of(key), a.m, p.scale) - log_l : __builtin_nanf("");
        p.top_ids[row * p.top + lane] = key ? (int32_t)id_of(key) : -1;
    }
}

// 8 values as they lie in memory: a load that is not widened at once is not waited for at once.
#define DN_GLOBAL __attribute__((address_space(1)))
__device__ __forceinline__ u32x4 global_ld16(const DN_GLOBAL char* p) { return *reinterpret_cast<const DN_GLOBAL u32x4*>(p); }
template <class T>
struct Piece;
template <>
struct Piece<__bf16> {
    u32x4 w;
    __device__ __forceinline__ void load(const DN_GLOBAL char* p) { w = global_ld16(p); }
    __device__ __forceinline__ void get(float* f) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[2 * e] = bf_lo(w[e]);
            f[2 * e + 1] = bf_hi(w[e]);
        }
    }
};
template <>
struct Piece<float> {
    u32x4 a, b;
    __device__ __forceinline__ void load(const DN_GLOBAL char* p) {
        a = global_ld16(p);
        b = global_ld16(p + 16);
    }
    __device__ __forceinline__ void get(float* f) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[e] = __uint_as_float(a[e]);
            f[4 + e] = __uint_as_float(b[e]);
        }
    }
};
// What a row without a whole piece loads, in vain.
__device__ const u32x4 kNoPiece[2] = {};

// The largest of 8 values by three-operand instructions (the two-operand ones take twice as many), NaN if one of them is: the
// other kind of maximum, v_max3, drops what stands beside a signalling NaN.
__device__ __forceinline__ float max8(const float* f) {
    float a, b, c, d;
    asm("v_maximum3_f32 %0, %1, %2, %3" : "=v"(a) : "v"(f[0]), "v"(f[1]), "v"(f[2]));
    asm("v_maximum3_f32 %0, %1, %2, %3" : "=v"(b) : "v"(f[3]), "v"(f[4]), "v"(f[5]));
    asm("v_maximum3_f32 %0, %1, %2, %3" : "=v"(c) : "v"(a), "v"(f[6]), "v"(f[7]));
    asm("v_maximum3_f32 %0, %1, %2, %2" : "=v"(d) : "v"(b), "v"(c));
    return d;
}

// A workgroup of NT threads takes a row, or one of its segments; loads run two steps of 8 NT tokens ahead.
template <class T, bool TOP, int NT>
__global__ __launch_bounds__(NT) void logprobs_kernel(LpArgs p) {
    constexpr int NW = NT / kWave;
    __shared__ float sums[NW][3];
    __shared__ int counts[NW];
    __shared__ uint32_t floors[NW];
    __shared__ unsigned long long pool[TOP ? NW * kMostKept : 1];
    __shared__ __attribute__((aligned(16))) WaveRanks ranks[TOP ? NW : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = blockIdx.x / (unsigned)p.segments;
    const int seg = (int)(blockIdx.x % (unsigned)p.segments);
    const T* x = reinterpret_cast<const T*>(p.logits) + row * p.stride;
    const int V = (int)p.V;
    const float c = p.scale * kLog2eF;
    // the row in pieces of 8 values that start at aligned addresses: the first piece may begin before it
    const int shift = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
    const int pieces = (int)((p.V + shift + 7) / 8), per = (pieces + p.segments - 1) / p.segments;
    const int end = min(pieces, (seg + 1) * per);
    // pieces that lie in the row whole; the others' values are read one by one
    const int whole0 = shift ? 1 : 0, whole1 = (V + shift) / 8 - 1;
    const bool any_whole = whole1 >= whole0;
    const DN_GLOBAL char* base = (const DN_GLOBAL char*)(any_whole ? (const void*)(x - shift) : (const void*)kNoPiece);
    const int from0 = any_whole ? whole0 : 0, from1 = any_whole ? whole1 : 0, whole_end = min(end - 1, whole1);

    Sums a{kLowest, 0.f, 0.f};
    Ranked ranked{(DN_LDS WaveRanks*)&ranks[TOP ? wave : 0], 0, 0, p.top, 0, 0, 0.f};
    int v0 = seg * per + wave * kWave;
    Given given{-1, 0.f};
    if (wave == 0 && p.segments == 1 && p.n) given.load(p, row, x, lane);
    bool first = true;
    Piece<T> q[2];
    // without conditions, so that the loads in flight can be counted: past the row's last whole piece this one again
    auto load = [&](int from, Piece<T>& to) {
        const uint32_t v = (uint32_t)max(min(from + lane, from1), from0);
        to.load(base + (size_t)(v * (uint32_t)(8 * sizeof(T))));  // below 2^32: V is below 2^30
    };
    auto take = [&](Piece<T>& piece) {
        const int v = v0 + lane;
        float f[8];
        piece.get(f);
        load(v0 + 2 * NT, piece);
        bool there = true;
        if (v0 < whole0 || v0 + kWave - 1 > whole_end) {
            if (v < whole0 || v > whole_end) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at = v * 8 - shift + e;
                    f[e] = v < end && at >= 0 && at < V ? to_f32<T>(x[at]) : -__builtin_inff();
                }
            }
            there = v < end;
        }
        float most = max8(f);
        // seldom: one maximum for the wave.  (A NaN raises nothing: the row's sums are NaN by then.)
        if (__any(most > a.m)) raise(a, wave_maxf(__builtin_fmaxf(a.m, most)), c);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = exponent(f[e], a.m, c), w = __builtin_amdgcn_exp2f(d);
            a.l += w;
            a.s = __builtin_fmaf(w, __builtin_fmaxf(d, kLeastExponent), a.s);
        }
        if constexpr (TOP) {
            if (first) ranked.start(there ? most : __builtin_nanf(""));
            first = false;
            ranked.add(f, most, there ? v * 8 - shift : V, V, lane);  // v * 8 - shift < 2^31: V is
        }
        v0 += NT;
    };
    load(v0, q[0]);
    __builtin_amdgcn_sched_barrier(0);  // in this order: the first is waited for alone
    load(v0 + NT, q[1]);
    __builtin_amdgcn_sched_barrier(0);
    while (v0 < end) {
        take(q[0]);
        take(q[1]);  // possibly past the end, where it changes nothing
    }
    a = wave_join(a, c);
    if (TOP && ranked.groups) ranked.flush(V, lane);
    if (TOP && ranked.n > ranked.kept()) ranked.cut(lane);
    if (lane == 0) {
        sums[wave][0] = a.m;
        sums[wave][1] = a.l;
        sums[wave][2] = a.s;
        counts[wave] = ranked.n;
        floors[wave] = ranked.n >= p.top ? ranked.floor : 1;
    }
    __syncthreads();
    int total = 0;
    uint32_t floor = 1;
    if constexpr (TOP) {  // the waves' keys side by side
        int mine = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (w == wave) mine = total;
            total += counts[w];
            floor = floors[w] > floor ? floors[w] : floor;
        }
        floor = __builtin_amdgcn_readfirstlane(floor);
        for (int i = lane; i < ranked.n; i += kWave) pool[mine + i] = ranked.m->keys[i];
        __syncthreads();
    }
    if (wave != 0) return;
    a = Sums{kLowest, 0.f, 0.f};
    if (lane < NW) a = Sums{sums[lane][0], sums[lane][1], sums[lane][2]};
    a = wave_join(a, c);
    const unsigned long long key = TOP ? top_of((DN_LDS unsigned long long*)pool, __builtin_amdgcn_readfirstlane(total), p.top, floor, ranked.m, lane) : 0;
    if (p.segments == 1) {
        finish<T>(p, row, x, a, key, given, lane);
    } else {
        if (lane == 0) *reinterpret_cast<f32x4*>(p.part_sums + (int64_t)blockIdx.x * 4) = f32x4{a.m, a.l, a.s, 0.f};
        if (TOP && lane < p.top) p.part_top[(int64_t)blockIdx.x * p.top + lane] = key;
    }
}

// Joins a row's segments: one wave.
template <class T>
__global__ __launch_bounds__(kWave) void logprobs_join_kernel(LpArgs p) {
    __shared__ unsigned long long pool[kMaxSegments * kMaxTop];
    __shared__ __attribute__((aligned(16))) WaveRanks ranks;
    const int lane = threadIdx.x, total = p.segments * p.top;
    const int64_t row = blockIdx.x;
    const T* x = reinterpret_cast<const T*>(p.logits) + row * p.stride;
    Given given{-1, 0.f};
    if (p.n) given.load(p, row, x, lane);
    for (int i = lane; i < total; i += kWave) pool[i] = p.part_top[row * total + i];
    Sums a{kLowest, 0.f, 0.f};
    if (lane < p.segments) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(p.part_sums + (row * p.segments + lane) * 4);
        a = Sums{v[0], v[1], v[2]};
    }
    lds_in_order();
    a = wave_join(a, p.scale * kLog2eF);
    unsigned long long key = 0;
    if (p.top) {
        // a segment's last key has `top` keys at or above it (0 where a segment has fewer)
        const uint32_t last = lane < p.segments ? (uint32_t)(pool[lane * p.top + p.top - 1] >> 32) : 0, most = wave_max(last);
        key = top_of((DN_LDS unsigned long long*)pool, total, p.top, most > 1 ? most : 1, (DN_LDS WaveRanks*)&ranks, lane);
    }
    finish<T>(p, row, x, a, key, given, lane);
}

template <class T, bool TOP>
static void launch_logprobs(const LpArgs& p, int threads, hipStream_t s) {
    const dim3 grid((unsigned)(p.T * p.segments));
    switch (threads) {
        case 64: logprobs_kernel<T, TOP, 64><<<grid, 64, 0, s>>>(p); break;
        case 128: logprobs_kernel<T, TOP, 128><<<grid, 128, 0, s>>>(p); break;
        case 256:  // ranked rows alone
            if constexpr (TOP) logprobs_kernel<T, TOP, 256><<<grid, 256, 0, s>>>(p);
            break;
        default: logprobs_kernel<T, TOP, 512><<<grid, 512, 0, s>>>(p);
    }
    if (p.segments > 1) logprobs_join_kernel<T><<<dim3((unsigned)p.T), kWave, 0, s>>>(p);
}

hipError_t launch_token_logprobs(const void* logits, int64_t stride, int64_t T, int64_t V, int dtype, float scale,
                                 const int32_t* targets, int64_t n, int64_t top, float* logprobs, float* entropy,
                                 float* top_logprobs, int32_t* top_ids, void* workspace, hipStream_t s) {
    const LogprobPlan plan = plan_logprobs(T, V, top);
    float* sums = reinterpret_cast<float*>(workspace);
    const LpArgs p{logits, stride, T, V, n, scale, (int)top, (int)plan.segments, targets, logprobs, entropy, top_logprobs,
                   top_ids, sums, reinterpret_cast<unsigned long long*>(sums + (plan.segments > 1 ? T * plan.segments * 4 : 0))};
    if (dtype == 0)
        top ? launch_logprobs<float, true>(p, plan.threads, s) : launch_logprobs<float, false>(p, plan.threads, s);
    else
        top ? launch_logprobs<__bf16, true>(p, plan.threads, s) : launch_logprobs<__bf16, false>(p, plan.threads, s);
    return hipGetLastError();
}

}  // namespace dn
