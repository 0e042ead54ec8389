// logprobs.hip -- log probabilities of given tokens, entropy and the likeliest tokens of each row of
// logits, in one pass.
//
// With m the row's maximum and d = scale (x - m): l = sum e^d, s = sum e^d d, and then
//     ln p_i = d_i - ln l,     entropy = ln l - s / l,
// so the normalization (Eq. (7) with the max subtraction of its footnote) is applied to the tokens
// asked for alone, after the pass.  Each lane keeps its own (m, l, s); on a larger m' they become
// f l and f (s + d' l) with d' = scale (m - m'), f = e^d'.  Exponents are to base 2 inside.
//
// The likeliest tokens are a sorted list per wave, one entry to a lane, as 64-bit keys: the logit's
// bits in an order that integers share, then the complement of the token's id, so that the larger
// key is the likelier token and, among equals, the lower id.
//
// Bound by HBM for long inputs (one read of the logits), by launches and the serial ranking for short.
#include "dn_device.hpp"
#include "dn_launch.hpp"
#include "fp8_rules.hpp"

namespace dn {

constexpr float kLowest = -3.402823466e38f;
constexpr float kLeastExponent = -200.f;  // 2^-200 is 0 in fp32; keeps 0 * -inf out of the sums
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kLpThreads = 256, kLpWaves = kLpThreads / kWave;

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
__device__ __forceinline__ Sums wave_join(Sums a, float c) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1)
        join(a, Sums{__shfl_xor(a.m, o), __shfl_xor(a.l, o), __shfl_xor(a.s, o)}, c);
    return a;
}

// ------------------------------------------------------------------------------- ranks
__device__ __forceinline__ unsigned long long key_of(float x, uint32_t id) {
    const uint32_t u = __float_as_uint(x + 0.f);  // -0 ranks as +0
    const uint32_t o = u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
    return ((unsigned long long)o << 32) | (uint32_t)~id;
}
__device__ __forceinline__ float value_of(unsigned long long key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ uint32_t id_of(unsigned long long key) { return ~(uint32_t)key; }

__device__ __forceinline__ unsigned long long lane_key(unsigned long long k, int lane) {
    return ((unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32) |
           (uint32_t)__builtin_amdgcn_readlane((int)k, lane);
}

// A wave's ranked list: lane i holds the i-th largest key so far, 0 where there is none yet.
struct Ranked {
    unsigned long long key;
    float last;        // the value and id that a token has to beat
    uint32_t last_id;
    __device__ __forceinline__ void clear() {
        key = 0;
        last = -__builtin_inff();
        last_id = 0xffffffffu;
    }
    __device__ __forceinline__ bool beats(float x, uint32_t id) const { return x > last || (x == last && id < last_id); }
    __device__ __forceinline__ void insert(unsigned long long k, int lane, int top) {
        const int pos = __popcll(__ballot(key > k));
        const unsigned long long up = __shfl_up(key, 1);
        key = lane < pos ? key : lane == pos ? k : up;
        const unsigned long long e = lane_key(key, top - 1);
        if (e != 0) {
            last = value_of(e);
            last_id = id_of(e);
        }
    }
};

// Joins `lists` (at most 64) sorted lists of `top` keys: lane i of the calling wave gets the i-th key.
__device__ __forceinline__ unsigned long long join_lists(const unsigned long long* keys, int lists, int top, int lane) {
    int at = 0;
    unsigned long long head = lane < lists ? keys[(int64_t)lane * top] : 0, mine = 0;
    for (int r = 0; r < top; ++r) {
        unsigned long long best = head;
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) {
            const unsigned long long other = __shfl_xor(best, o);
            best = other > best ? other : best;
        }
        if (lane == r) mine = best;
        if (best == 0) break;
        if (head == best) {
            ++at;
            head = at < top ? keys[(int64_t)lane * top + at] : 0;
        }
    }
    return mine;
}

// ------------------------------------------------------------------------------- results
template <class T>
__device__ __forceinline__ void finish(const LpArgs& p, int64_t row, const T* x, const Sums& a, unsigned long long key,
                                       int thread, int threads) {
    const float log_l = kLn2 * __builtin_amdgcn_logf(a.l);
    for (int64_t i = thread; i < p.n; i += threads) {
        const int32_t t = p.targets[row * p.n + i];
        float v = 0.f;
        if (t >= 0) v = t < p.V ? (to_f32<T>(x[t]) - a.m) * p.scale - log_l : __builtin_nanf("");
        p.logprobs[row * p.n + i] = v;
    }
    if (p.entropy && thread == 0) p.entropy[row] = log_l - kLn2 * (a.s / a.l);
    if (thread < p.top) {
        p.top_logprobs[row * p.top + thread] = key ? (value_of(key) - a.m) * p.scale - log_l : __builtin_nanf("");
        p.top_ids[row * p.top + thread] = key ? (int32_t)id_of(key) : -1;
    }
}

// 8 values from x[at] on, -inf outside [0, V); x + at is aligned to 16 bytes.
template <class T>
__device__ __forceinline__ void load8(const T* x, int64_t at, int64_t V, float* f);
template <>
__device__ __forceinline__ void load8<__bf16>(const __bf16* x, int64_t at, int64_t V, float* f) {
    if (at >= 0 && at + 8 <= V) {
        const u32x4 w = ld16_stream(x + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[2 * e] = bf_lo(w[e]);
            f[2 * e + 1] = bf_hi(w[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = at + e >= 0 && at + e < V ? (float)x[at + e] : -__builtin_inff();
    }
}
template <>
__device__ __forceinline__ void load8<float>(const float* x, int64_t at, int64_t V, float* f) {
    if (at >= 0 && at + 8 <= V) {
        const u32x4 a = ld16_stream(x + at), b = ld16_stream(x + at + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[e] = __uint_as_float(a[e]);
            f[4 + e] = __uint_as_float(b[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = at + e >= 0 && at + e < V ? x[at + e] : -__builtin_inff();
    }
}

template <class T, bool TOP>
__global__ __launch_bounds__(kLpThreads) void logprobs_kernel(LpArgs p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.x / p.segments;
    const int seg = (int)(blockIdx.x % p.segments);
    const T* x = reinterpret_cast<const T*>(p.logits) + row * p.stride;
    const int64_t V = p.V;
    const float c = p.scale * kLog2eF;
    // the row in pieces of 8 values that start at aligned addresses: the first piece may begin before it
    const int shift = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
    const int64_t pieces = (V + shift + 7) / 8, per = (pieces + p.segments - 1) / p.segments;
    const int64_t end = min(pieces, (seg + 1) * per);

    Sums a{kLowest, 0.f, 0.f};
    Ranked ranked;
    ranked.clear();
    for (int64_t v0 = seg * per + wave * kWave; v0 < end; v0 += kLpThreads) {
        const int64_t at = (v0 + lane) * 8 - shift;
        const int64_t limit = v0 + lane < end ? V : 0;  // past the segment: nothing
        float f[8];
        load8<T>(x, at, limit, f);
        const float most = __builtin_fmaxf(__builtin_fmaxf(__builtin_fmaxf(f[0], f[1]), __builtin_fmaxf(f[2], f[3])),
                                           __builtin_fmaxf(__builtin_fmaxf(f[4], f[5]), __builtin_fmaxf(f[6], f[7])));
        if (__any(most > a.m)) raise(a, __builtin_fmaxf(a.m, most), c);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = exponent(f[e], a.m, c), w = __builtin_amdgcn_exp2f(d);
            a.l += w;
            a.s = __builtin_fmaf(w, __builtin_fmaxf(d, kLeastExponent), a.s);
        }
        if constexpr (TOP) {
            const uint32_t first = (uint32_t)max(at, (int64_t)0);
            if (__any(at < limit && ranked.beats(most, first))) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int64_t id = at + e;
                    unsigned long long left = __ballot(id >= 0 && id < limit && ranked.beats(f[e], (uint32_t)id));
                    while (left) {
                        const int b = __builtin_ctzll(left);
                        const float xv = __uint_as_float(__builtin_amdgcn_readlane((int)__float_as_uint(f[e]), b));
                        const uint32_t xi = (uint32_t)__builtin_amdgcn_readlane((int)id, b);
                        ranked.insert(key_of(xv, xi), lane, p.top);
                        left &= left - 1;
                        left &= __ballot(ranked.beats(f[e], (uint32_t)id));
                    }
                }
            }
        }
    }
    a = wave_join(a, c);
    __shared__ float sums[kLpWaves][3];
    __shared__ unsigned long long keys[TOP ? kLpWaves * kMaxTop : 1];
    if (lane == 0) {
        sums[wave][0] = a.m;
        sums[wave][1] = a.l;
        sums[wave][2] = a.s;
    }
    if (TOP && lane < p.top) keys[wave * p.top + lane] = ranked.key;
    __syncthreads();
    if (wave != 0) return;
    a = Sums{sums[0][0], sums[0][1], sums[0][2]};
#pragma unroll
    for (int w = 1; w < kLpWaves; ++w) join(a, Sums{sums[w][0], sums[w][1], sums[w][2]}, c);
    const unsigned long long key = TOP ? join_lists(keys, kLpWaves, p.top, lane) : 0;
    if (p.segments == 1) {
        finish<T>(p, row, x, a, key, lane, kWave);
    } else {
        if (lane == 0) *reinterpret_cast<f32x4*>(p.part_sums + (int64_t)blockIdx.x * 4) = f32x4{a.m, a.l, a.s, 0.f};
        if (TOP && lane < p.top) p.part_top[(int64_t)blockIdx.x * p.top + lane] = key;
    }
}

// One wave joins a row's segments (at most 64, one to a lane).
template <class T>
__global__ __launch_bounds__(kWave) void logprobs_join_kernel(LpArgs p) {
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    Sums a{kLowest, 0.f, 0.f};
    if (lane < p.segments) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(p.part_sums + (row * p.segments + lane) * 4);
        a = Sums{v[0], v[1], v[2]};
    }
    a = wave_join(a, p.scale * kLog2eF);
    const unsigned long long key =
        p.top ? join_lists(p.part_top + row * p.segments * p.top, p.segments, p.top, lane) : 0;
    finish<T>(p, row, reinterpret_cast<const T*>(p.logits) + row * p.stride, a, key, lane, kWave);
}

hipError_t launch_token_logprobs(const void* logits, int64_t stride, int64_t T, int64_t V, int dtype, float scale,
                                 const int32_t* targets, int64_t n, int64_t top, float* logprobs, float* entropy,
                                 float* top_logprobs, int32_t* top_ids, void* workspace, int64_t segments, hipStream_t s) {
    float* sums = reinterpret_cast<float*>(workspace);
    const LpArgs p{logits, stride, T, V, n, scale, (int)top, (int)segments, targets, logprobs, entropy, top_logprobs, top_ids,
                   sums, reinterpret_cast<unsigned long long*>(sums + (segments > 1 ? T * segments * 4 : 0))};
    const dim3 grid((unsigned)(T * segments));
    if (dtype == 0) {
        if (top)
            logprobs_kernel<float, true><<<grid, kLpThreads, 0, s>>>(p);
        else
            logprobs_kernel<float, false><<<grid, kLpThreads, 0, s>>>(p);
        if (segments > 1) logprobs_join_kernel<float><<<dim3((unsigned)T), kWave, 0, s>>>(p);
    } else {
        if (top)
            logprobs_kernel<__bf16, true><<<grid, kLpThreads, 0, s>>>(p);
        else
            logprobs_kernel<__bf16, false><<<grid, kLpThreads, 0, s>>>(p);
        if (segments > 1) logprobs_join_kernel<__bf16><<<dim3((unsigned)T), kWave, 0, s>>>(p);
    }
    return hipGetLastError();
}

}  // namespace dn
