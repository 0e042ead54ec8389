// kv_cache.hip -- rotary positions, and writing and reading back the paged key/value cache.
//
// Rotation: dimensions (p, q) of a head form pairs, (2i, 2i + 1) or (i, i + rot/2); position n turns
// each by its angle, y_p = x_p cos - x_q sin, y_q = x_q cos + x_p sin.  The transpose (the gradient)
// is the rotation by the opposite angle.  cos and sin come from a table of fp32 pairs, each rounded
// once from fp64, so that angles stay exact at long positions and no call evaluates them again.
//
// All kernels here are bound by HBM (or, over a few tokens, by launch and load latency): every
// element is read once, in 16-byte pieces, and written once.
#include "dn_device.hpp"
#include "dn_launch.hpp"
#include "kv_layout.hpp"

namespace dn {
namespace kv {

__global__ __launch_bounds__(256) void rotary_table_kernel(const double* __restrict__ inv_freq, int half,
                                                           int64_t count, double amplitude, float* __restrict__ table) {
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= count) return;
    const int64_t pos = at / half;
    double s, c;
    sincos((double)pos * inv_freq[at - pos * half], &s, &c);
    table[2 * at] = (float)(c * amplitude);
    table[2 * at + 1] = (float)(s * amplitude);
}

// A thread's part of one head: two 16-byte pieces whose elements pair up.
template <class T>
struct Pieces {
    static constexpr int N = elem<T>::per16;
    float a[N], b[N];
};
template <class T>
__device__ __forceinline__ void widen(const u32x4& v, float* f);
template <>
__device__ __forceinline__ void widen<__bf16>(const u32x4& v, float* f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f[2 * j] = bf_lo(w[j]);
        f[2 * j + 1] = bf_hi(w[j]);
    }
}
template <>
__device__ __forceinline__ void widen<float>(const u32x4& v, float* f) {
    f[0] = __uint_as_float(v.x);
    f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z);
    f[3] = __uint_as_float(v.w);
}
template <class T>
__device__ __forceinline__ u32x4 narrow(const float* f);
template <>
__device__ __forceinline__ u32x4 narrow<__bf16>(const float* f) {
    return u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
}
template <>
__device__ __forceinline__ u32x4 narrow<float>(const float* f) {
    return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
}

// Where the two pieces of item p lie in a head: pairs first (rot / 2N items), then the rest as it is.
template <int N>
__device__ __forceinline__ void piece_dims(int p, int rot, bool interleaved, int& xa, int& xb) {
    const int turned = rot / (2 * N);
    if (interleaved || p >= turned) {
        xa = 2 * N * p;
        xb = xa + N;
    } else {
        xa = N * p;
        xb = xa + rot / 2;
    }
}

// Turns the pieces by row `cs` of the table (cos, sin pairs); null: a position outside the table, NaN.
template <class T>
__device__ __forceinline__ void turn(Pieces<T>& v, int p, const float* cs, bool interleaved, float sign) {
    constexpr int N = Pieces<T>::N;
    float c[N], s[N];
    if (cs) {
        const float4* row = reinterpret_cast<const float4*>(cs + 2 * N * p);
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
            const float4 t = row[j];
            c[2 * j] = t.x;
            s[2 * j] = t.y * sign;
            c[2 * j + 1] = t.z;
            s[2 * j + 1] = t.w * sign;
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) c[j] = s[j] = __builtin_nanf("");
    }
    if (interleaved) {  // pairs lie side by side: a holds the first N/2, b the others
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
            const float a0 = v.a[2 * j], a1 = v.a[2 * j + 1], b0 = v.b[2 * j], b1 = v.b[2 * j + 1];
            v.a[2 * j] = a0 * c[j] - a1 * s[j];
            v.a[2 * j + 1] = a1 * c[j] + a0 * s[j];
            v.b[2 * j] = b0 * c[N / 2 + j] - b1 * s[N / 2 + j];
            v.b[2 * j + 1] = b1 * c[N / 2 + j] + b0 * s[N / 2 + j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float a = v.a[j], b = v.b[j];
            v.a[j] = a * c[j] - b * s[j];
            v.b[j] = b * c[j] + a * s[j];
        }
    }
}

// One item (two pieces) per thread, items of a head, then heads, then tokens: consecutive threads
// read consecutive memory, and the heads of a token find its table row in L1.  Measured, 8192 tokens x 40 heads
// of 128, bf16, rows of 6144: 33 us a call on changing tensors, 5.2 TB/s, a copy's rate.
template <class T>
__global__ __launch_bounds__(256) void rotary_kernel(const T* x, int64_t x_stride, const int32_t* __restrict__ positions,
                                                     const float* __restrict__ table, int64_t rows, int64_t tokens,
                                                     uint32_t per_token, uint32_t per_head, int d, int rot, int interleaved,
                                                     float sign, T* out, int64_t out_stride) {
    constexpr int N = Pieces<T>::N;
    const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t token = item / per_token;
    if (token >= tokens) return;
    const uint32_t in = (uint32_t)(item - token * per_token), head = in / per_head;
    const int p = (int)(in - head * per_head);
    int xa, xb;
    piece_dims<N>(p, rot, interleaved, xa, xb);
    const T* src = x + token * x_stride + (int64_t)head * d;
    T* dst = out + token * out_stride + (int64_t)head * d;
    u32x4 ra = ld16(src + xa), rb = ld16(src + xb);
    if (p < rot / (2 * N)) {
        const int64_t pos = positions[token];
        Pieces<T> v;
        widen<T>(ra, v.a);
        widen<T>(rb, v.b);
        turn<T>(v, p, (uint64_t)pos < (uint64_t)rows ? table + pos * rot : nullptr, interleaved, sign);
        ra = narrow<T>(v.a);
        rb = narrow<T>(v.b);
    }
    *reinterpret_cast<u32x4*>(dst + xa) = ra;
    *reinterpret_cast<u32x4*>(dst + xb) = rb;
}

// ----------------------------------------------------------------------------- codes
// Scale of a row from the largest |x| among its threads' bits; NaN where one of its elements is held as no
// finite number (bits at or past infinity's, in bf16 at or past those that round to it, halfway above its
// largest): the row's codes are then 0 and it reads back as NaN, and no masked product with it can spread.
template <int FMT>
__device__ __forceinline__ float row_scale(uint32_t top, float& inv) {
    if (top >= (FMT == kKvBf16 ? 0x7f7f8000u : 0x7f800000u)) {
        inv = 0.f;
        return __builtin_nanf("");
    }
    if constexpr (FMT == kKvBf16) {
        inv = 1.f;
        return 1.f;
    }
    const float scale = fmaxf(__uint_as_float(top) * (1.0f / kFp8Max), kFp8Least);
    inv = 1.0f / scale;
    return scale;
}
__device__ __forceinline__ uint32_t pack_fp8(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// 8 elements as codes: 16 bytes of bf16 (inv is 1, or 0 for rows of NaN) or 8 of e4m3
template <int FMT>
struct Codes;
template <>
struct Codes<kKvBf16> {
    typedef u32x4 type;
    static __device__ __forceinline__ type of(const float* f, float inv) {
        return inv == 0.f ? u32x4{0, 0, 0, 0} : narrow<__bf16>(f);
    }
};
template <>
struct Codes<kKvFp8> {
    typedef uint2 type;
    static __device__ __forceinline__ type of(const float* f, float inv) {
        if (inv == 0.f) return uint2{0, 0};
        return uint2{pack_fp8(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv),
                     pack_fp8(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv)};
    }
};

struct AppendArgs {
    const __bf16* qkv;
    int64_t stride;
    const int32_t* slots;
    const int32_t* positions;
    const float* table;
    int64_t rows, tokens, total_slots;
    int heads, group, rot, interleaved, tile;
    char* pool;
    __bf16* q_out;
};

// One key/value head of `tile` tokens: its query heads are turned and written, K is turned, K and V
// are put into codes, staged in LDS and written out in the order in which a block holds them.  K's
// 16-byte pieces hold one token; V's hold E consecutive tokens of one dimension and go out whole
// where E tokens of the call fill one, else element by element.  Measured, 4096 tokens of 32 query and 8
// key/value heads of 128, fp8 (95 MB): 24 us, 3.9 TB/s.
template <int FMT, int D>
__global__ __launch_bounds__(256) void append_kernel(const AppendArgs a) {
    using B = KvBlock<FMT, D>;
    constexpr int E = B::E, N = 8, ITEMS = D / 16;       // items of a head (two pieces of 8)
    constexpr int PITCH = D * B::BYTES + 16;             // LDS row, 16-byte aligned
    constexpr int kTile = kAppendTile;
    __shared__ __attribute__((aligned(16))) char smem[2 * kTile * PITCH];
    __shared__ int32_t slot_of[kTile];
    const int tid = threadIdx.x;
    const int h = blockIdx.x % a.heads;
    const int64_t t0 = (int64_t)(blockIdx.x / a.heads) * a.tile;
    const int n = (int)min((int64_t)a.tile, a.tokens - t0);
    if (tid < kTile) {
        int32_t s = -1;
        if (tid < n) s = a.slots[t0 + tid];
        slot_of[tid] = (uint64_t)(int64_t)s < (uint64_t)a.total_slots ? s : -1;
    }
    __syncthreads();
    const int q_heads = a.heads * a.group, per_token = (a.group + 2) * ITEMS;
    // items of a head are neighbouring lanes: 256 and ITEMS are powers of two
    for (int i = tid; i < n * per_token; i += 256) {
        const int p = i % ITEMS, row = i / ITEMS, t = row / (a.group + 2), which = row - t * (a.group + 2);
        const bool is_k = which == a.group, is_v = which == a.group + 1;
        const int head = is_v ? q_heads + a.heads + h : is_k ? q_heads + h : h * a.group + which;
        const bool turned = !is_v && p < a.rot / 16;
        int xa, xb;
        piece_dims<N>(p, is_v ? 0 : a.rot, a.interleaved, xa, xb);
        const __bf16* src = a.qkv + (t0 + t) * a.stride + (int64_t)head * D;
        const u32x4 ra = ld16(src + xa), rb = ld16(src + xb);
        Pieces<__bf16> v;
        widen<__bf16>(ra, v.a);
        widen<__bf16>(rb, v.b);
        if (turned) {
            const int64_t pos = a.positions[t0 + t];
            turn<__bf16>(v, p, (uint64_t)pos < (uint64_t)a.rows ? a.table + pos * a.rot : nullptr, a.interleaved, 1.f);
        }
        if (which < a.group) {
            __bf16* dst = a.q_out + ((t0 + t) * q_heads + head) * (int64_t)D;
            *reinterpret_cast<u32x4*>(dst + xa) = narrow<__bf16>(v.a);
            *reinterpret_cast<u32x4*>(dst + xb) = narrow<__bf16>(v.b);
            continue;
        }
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < N; ++j)
            top = max(top, max(__float_as_uint(v.a[j]) & 0x7fffffffu, __float_as_uint(v.b[j]) & 0x7fffffffu));
#pragma unroll
        for (int o = 1; o < ITEMS; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        float inv;
        const float scale = row_scale<FMT>(top, inv);
        typename Codes<FMT>::type ca = Codes<FMT>::of(v.a, inv), cb = Codes<FMT>::of(v.b, inv);
        char* lds = smem + (is_v ? kTile * PITCH : 0) + t * PITCH;
        *reinterpret_cast<typename Codes<FMT>::type*>(lds + xa * B::BYTES) = ca;
        *reinterpret_cast<typename Codes<FMT>::type*>(lds + xb * B::BYTES) = cb;
        const int32_t slot = slot_of[t];
        if (p == 0 && slot >= 0) {
            char* block = a.pool + ((int64_t)(slot / kKvPage) * a.heads + h) * B::SIZE;
            reinterpret_cast<float*>(block + (is_v ? B::VS : B::KS))[slot % kKvPage] = scale;
        }
    }
    __syncthreads();
    // K: a token's 16-byte pieces, tokens fastest
    for (int i = tid; i < a.tile * (D / E); i += 256) {
        const int t = i % a.tile, piece = i / a.tile;
        const int32_t slot = t < n ? slot_of[t] : -1;
        if (slot < 0) continue;
        char* block = a.pool + ((int64_t)(slot / kKvPage) * a.heads + h) * B::SIZE;
        *reinterpret_cast<u32x4*>(block + B::k_at(slot % kKvPage, piece * E)) =
            *reinterpret_cast<const u32x4*>(smem + t * PITCH + piece * 16);
    }
    // V: E tokens of a dimension, from the first token of the call that starts such a run on
    const int shift = slot_of[0] < 0 ? 0 : slot_of[0] % E;
    const int runs = (n + shift + E - 1) / E;
    const char* vs = smem + kTile * PITCH;
    for (int i = tid; i < runs * D; i += 256) {
        const int x = i % D, t = i / D * E - shift;
        bool whole = t >= 0 && t + E <= n;
        const int32_t first = whole ? slot_of[t] : -1;
        whole = whole && first >= 0 && first % E == 0;
        if (whole)
            for (int r = 1; r < E; ++r) whole = whole && slot_of[t + r] == first + r;
        if (whole) {
            union {
                u32x4 v;
                uint8_t b[16];
                uint16_t s[8];
            } c;
#pragma unroll
            for (int r = 0; r < E; ++r) {
                if constexpr (FMT == kKvBf16)
                    c.s[r] = *reinterpret_cast<const uint16_t*>(vs + (t + r) * PITCH + x * 2);
                else
                    c.b[r] = *reinterpret_cast<const uint8_t*>(vs + (t + r) * PITCH + x);
            }
            char* block = a.pool + ((int64_t)(first / kKvPage) * a.heads + h) * B::SIZE + B::PART;
            *reinterpret_cast<u32x4*>(block + B::v_at(first % kKvPage, x)) = c.v;
        } else {
            for (int r = 0; r < E; ++r) {
                if (t + r < 0 || t + r >= n) continue;
                const int32_t slot = slot_of[t + r];
                if (slot < 0) continue;
                char* at = a.pool + ((int64_t)(slot / kKvPage) * a.heads + h) * B::SIZE + B::PART +
                           B::v_at(slot % kKvPage, x);
                if constexpr (FMT == kKvBf16)
                    *reinterpret_cast<uint16_t*>(at) = *reinterpret_cast<const uint16_t*>(vs + (t + r) * PITCH + x * 2);
                else
                    *at = vs[(t + r) * PITCH + x];
            }
        }
    }
}

struct ReadArgs {
    const char* pool;
    const int32_t* slots;
    int64_t tokens, total_slots, k_blocks;
    int heads;
    __bf16* K;
    __bf16* V;
};

// 8 codes as fp32
template <int FMT>
__device__ __forceinline__ void decode8(const u32x4& v, float scale, float* f) {
    if constexpr (FMT == kKvBf16) {
        widen<__bf16>(v, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] *= scale;
    } else {
        const uint32_t u[2] = {v.x, v.y};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(u[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(u[j], true);
            f[4 * j] = lo[0] * scale;
            f[4 * j + 1] = lo[1] * scale;
            f[4 * j + 2] = hi[0] * scale;
            f[4 * j + 3] = hi[1] * scale;
        }
    }
}

// 4 words of bytes (rows) -> 4 words of bytes (columns); 2 x 2 halves of two words
__device__ __forceinline__ void transpose_bytes(uint32_t (&w)[4]) {
    const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);
    const uint32_t c = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
    w[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
    w[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    w[2] = __builtin_amdgcn_perm(d, c, 0x05040100u);
    w[3] = __builtin_amdgcn_perm(d, c, 0x07060302u);
}

// From blocks to rows, one item to a thread.  The first `k_blocks` workgroups read K, 16 bytes of a token
// to a lane, tokens fastest (neighbours lie in neighbouring rows of a chunk).  The others read V: a
// lane takes four dimensions of E tokens that lie together (64 bytes in a row), turns them in
// registers and writes four dimensions of each token; tokens that do not lie together go one by one.
// Runs of E tokens are counted from the first slot of the workgroup's tokens.  Measured, 8192 tokens of 8 heads
// of 128, fp8 (51 MB): 15.5 us, 3.3 TB/s.
template <int FMT, int D>
__global__ __launch_bounds__(256) void read_kernel(const ReadArgs a) {
    using B = KvBlock<FMT, D>;
    constexpr int E = B::E, LANES = D / 4, RUNS = 256 / LANES, PIECES = D / E;
    const int tid = threadIdx.x;
    auto block_of = [&](int32_t slot, int h) { return a.pool + ((int64_t)(slot / kKvPage) * a.heads + h) * B::SIZE; };
    auto inside = [&](int32_t slot) { return (uint64_t)(int64_t)slot < (uint64_t)a.total_slots; };
    if ((int64_t)blockIdx.x < a.k_blocks) {
        constexpr int TOKENS = 256 / PIECES;
        const int h = blockIdx.x % a.heads;
        const int64_t t = (int64_t)(blockIdx.x / a.heads) * TOKENS + tid % TOKENS;
        const int piece = tid / TOKENS;
        if (t >= a.tokens) return;
        const int32_t slot = a.slots[t];
        __bf16* out = a.K + (t * a.heads + h) * (int64_t)D + piece * E;
        u32x4 v = {0, 0, 0, 0};
        float scale = 0.f;
        if (inside(slot)) {
            const char* block = block_of(slot, h);
            v = ld16(block + B::k_at(slot % kKvPage, piece * E));
            scale = reinterpret_cast<const float*>(block + B::KS)[slot % kKvPage];
        }
#pragma unroll
        for (int j = 0; j < E / 8; ++j) {
            float f[8];
            decode8<FMT>(j ? u32x4{v.z, v.w, 0, 0} : v, scale, f);
            *reinterpret_cast<u32x4*>(out + 8 * j) = narrow<__bf16>(f);
        }
        return;
    }
    const int id = blockIdx.x - (int)a.k_blocks, h = id % a.heads;
    constexpr int TOKENS = (RUNS - 1) * E;  // with a first run cut short these are RUNS runs
    const int64_t t0 = (int64_t)(id / a.heads) * TOKENS;
    const int n = (int)min((int64_t)TOKENS, a.tokens - t0);
    const int32_t start = a.slots[t0];
    const int x = tid % LANES * 4, lane_r = tid % LANES, t = tid / LANES * E - (inside(start) ? start % E : 0);
    // each lane of a run looks at one of its slots
    int32_t mine = -1;
    if (lane_r < E && t + lane_r >= 0 && t + lane_r < n) mine = a.slots[t0 + t + lane_r];
    const int32_t first = __shfl(mine, 0, LANES);
    const bool fits = lane_r >= E || (first >= 0 && first % E == 0 && mine == first + lane_r && inside(mine));
    const uint64_t all = __ballot(fits) >> ((tid & 63) / LANES * LANES);
    constexpr uint64_t RUN = LANES == 32 ? 0xffffffffull : 0xffffull;
    if (t >= n) return;
    const int64_t step = (int64_t)a.heads * D;
    __bf16* out = a.V + ((t0 + t) * a.heads + h) * (int64_t)D + x;
    if ((all & RUN) == RUN) {
        const char* block = block_of(first, h);
        const int o = first % kKvPage;
        u32x4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = ld16(block + B::PART + B::v_at(o, x) + 16 * k);
#pragma unroll
        for (int q = 0; q < E / 4; ++q) {  // four tokens
            const f32x4 scale = *reinterpret_cast<const f32x4*>(block + B::VS + 4 * (o + 4 * q));
            if constexpr (FMT == kKvFp8) {
                uint32_t w[4] = {v[0][q], v[1][q], v[2][q], v[3][q]};
                transpose_bytes(w);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[r], false);
                    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[r], true);
                    *reinterpret_cast<uint2*>(out + (4 * q + r) * step) =
                        uint2{pack_bf16(lo[0] * scale[r], lo[1] * scale[r]), pack_bf16(hi[0] * scale[r], hi[1] * scale[r])};
                }
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int w = 2 * q + r / 2;  // the word of each dimension that holds the token
                    float f[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) f[k] = (r & 1 ? bf_hi(v[k][w]) : bf_lo(v[k][w])) * scale[r];
                    *reinterpret_cast<uint2*>(out + (4 * q + r) * step) = uint2{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])};
                }
            }
        }
        return;
    }
    for (int r = 0; r < E; ++r) {
        if (t + r < 0 || t + r >= n) continue;
        const int32_t slot = a.slots[t0 + t + r];
        float f[4] = {0.f, 0.f, 0.f, 0.f};
        if (inside(slot)) {
            const char* block = block_of(slot, h);
            const char* at = block + B::PART + B::v_at(slot % kKvPage, x);
            const float scale = reinterpret_cast<const float*>(block + B::VS)[slot % kKvPage];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (FMT == kKvBf16)
                    f[k] = bf_lo(*reinterpret_cast<const uint16_t*>(at + 16 * k)) * scale;
                else
                    f[k] = __builtin_amdgcn_cvt_pk_f32_fp8(*reinterpret_cast<const uint8_t*>(at + 16 * k), false)[0] * scale;
            }
        }
        *reinterpret_cast<uint2*>(out + r * step) = uint2{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])};
    }
}

}  // namespace kv

hipError_t launch_rotary_table(const double* inv_freq, int64_t rot, int64_t rows, double amplitude, float* table,
                               hipStream_t s) {
    const int64_t count = rows * (rot / 2);
    kv::rotary_table_kernel<<<dim3((unsigned)((count + 255) / 256)), 256, 0, s>>>(inv_freq, (int)(rot / 2), count,
                                                                                 amplitude, table);
    return hipGetLastError();
}

hipError_t launch_rotary(const void* x, int64_t x_stride, const int32_t* positions, const float* table, int64_t rows,
                         int64_t tokens, int64_t heads, int64_t d, int64_t rot, int interleaved, int inverse, int dtype,
                         void* out, int64_t out_stride, hipStream_t s) {
    const int64_t per_head = d / (dtype == 0 ? 8 : 16), per_token = heads * per_head;
    const dim3 grid((unsigned)((tokens * per_token + 255) / 256));
    const float sign = inverse ? -1.f : 1.f;
    if (dtype == 0)
        kv::rotary_kernel<float><<<grid, 256, 0, s>>>((const float*)x, x_stride, positions, table, rows, tokens,
                                                      (uint32_t)per_token, (uint32_t)per_head, (int)d, (int)rot,
                                                      interleaved, sign, (float*)out, out_stride);
    else
        kv::rotary_kernel<__bf16><<<grid, 256, 0, s>>>((const __bf16*)x, x_stride, positions, table, rows, tokens,
                                                       (uint32_t)per_token, (uint32_t)per_head, (int)d, (int)rot,
                                                       interleaved, sign, (__bf16*)out, out_stride);
    return hipGetLastError();
}

hipError_t launch_kv_append(const void* qkv, int64_t stride, const int32_t* slots, const int32_t* positions,
                            const float* table, int64_t rows, int64_t rot, int interleaved, int64_t tokens,
                            int64_t q_heads, const KvPool& c, void* q_out, hipStream_t s) {
    kv::AppendArgs a{(const __bf16*)qkv, stride, slots, positions, table, rows, tokens, c.pages * kKvPage, (int)c.heads,
                     (int)(q_heads / c.heads), (int)rot, interleaved, append_tile(tokens, c.heads, q_heads / c.heads, c.d), (char*)c.data,
                     (__bf16*)q_out};
    const dim3 grid((unsigned)((tokens + a.tile - 1) / a.tile * c.heads));
    if (c.format == kKvBf16) {
        if (c.d == 64)
            kv::append_kernel<kKvBf16, 64><<<grid, 256, 0, s>>>(a);
        else
            kv::append_kernel<kKvBf16, 128><<<grid, 256, 0, s>>>(a);
    } else {
        if (c.d == 64)
            kv::append_kernel<kKvFp8, 64><<<grid, 256, 0, s>>>(a);
        else
            kv::append_kernel<kKvFp8, 128><<<grid, 256, 0, s>>>(a);
    }
    return hipGetLastError();
}

template <int FMT, int D>
static hipError_t launch_read(kv::ReadArgs a, hipStream_t s) {
    using B = KvBlock<FMT, D>;
    const int64_t k_tokens = 256 / (D / B::E), v_tokens = (256 / (D / 4) - 1) * B::E;
    a.k_blocks = (a.tokens + k_tokens - 1) / k_tokens * a.heads;
    const int64_t v_blocks = (a.tokens + v_tokens - 1) / v_tokens * a.heads;
    kv::read_kernel<FMT, D><<<dim3((unsigned)(a.k_blocks + v_blocks)), 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvPool& c, const int32_t* slots, int64_t tokens, void* K, void* V, hipStream_t s) {
    const kv::ReadArgs a{(const char*)c.data, slots, tokens, c.pages * kKvPage, 0, (int)c.heads, (__bf16*)K, (__bf16*)V};
    if (c.format == kKvBf16) return c.d == 64 ? launch_read<kKvBf16, 64>(a, s) : launch_read<kKvBf16, 128>(a, s);
    return c.d == 64 ? launch_read<kKvFp8, 64>(a, s) : launch_read<kKvFp8, 128>(a, s);
}

}  // namespace dn
