// linear_fp8.hip -- products of e4m3 codes with the scales, a bias, an activation or gate, and a
// residual in their epilogue; the preparation of their weights.
//
// With x = sx_m X and W = sw_n C (X, C codes):  z = sx_m sw_n (X . C) + b_n,
//     out = act(z) + residual      or, gated,      out = act(z_gate) z_up + residual.
// The scales are constant along the reduction, so they wait for the epilogue -- and with them the
// RMSNorm that made X, whose 1 / rms is part of sx_m.
//
// v_mfma_f32_16x16x128_f8f6f4 takes 16 rows x 128 codes of either operand, 32 bytes to a lane.  Which
// 32 of the 128 k a lane holds is free as long as both operands agree: lane l takes bytes
// 16 (l >> 4) .. of the first and of the second 64-byte half, which is what two packed chunks
// (and two 16-byte pieces of a 128-byte stretch of an x row) give it.
#include <type_traits>
#include <utility>

#include "dn_device.hpp"
#include "dn_launch.hpp"
#include "fp8_rules.hpp"

namespace dn {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct Fp8Args {
    const char* x;         // codes [M][K]
    const float* xs;       // [M]
    const char* w;         // packed chunks
    const float* ws;       // scales, bias: [16 blocks], packed column order
    const float* bias;
    const void* residual;  // [M][N], or null
    void* out;             // [M][N]
    float* part;           // partial sums [splits][M][16 blocks]
    int64_t M, K, N, kchunks, blocks;
    int act, gated, out_f32, splits;
};

// Sums.  The 8-bit matrix instructions (this one and its half-rate relatives alike) add products in groups
// of 16 along k aligned to the group's largest, with 13 bits below it, and the groups in fp32 (probed with
// products that cancel): 1.5e-5 of a result of normal data in the 2-norm, for any K; sums of products of one sign
// come out 2.6e-6 of themselves low.  A bf16 output's rounding is 100 times that.  An fp32 output's is not: there the codes are widened to bf16, which
// holds them exactly, and the bf16 instructions keep their products and sums to 2^-24, at half the rate.
__device__ __forceinline__ bf16x8_t widen8(uint32_t lo, uint32_t hi) {
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const auto c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

template <bool F32>
__device__ __forceinline__ f32x4 mfma_codes(const u32x4& a0, const u32x4& a1, const u32x4& b0, const u32x4& b1, f32x4 acc) {
    if constexpr (!F32) {
        const i32x8 a = {(int)a0.x, (int)a0.y, (int)a0.z, (int)a0.w, (int)a1.x, (int)a1.y, (int)a1.z, (int)a1.w};
        const i32x8 b = {(int)b0.x, (int)b0.y, (int)b0.z, (int)b0.w, (int)b1.x, (int)b1.y, (int)b1.z, (int)b1.w};
        // scales 0: the instruction without block scales
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 0, 0, 0, 0, 0, 0);
    } else {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(a0.x, a0.y), widen8(b0.x, b0.y), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(a0.z, a0.w), widen8(b0.z, b0.w), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(a1.x, a1.y), widen8(b1.x, b1.y), acc, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(a1.z, a1.w), widen8(b1.z, b1.w), acc, 0, 0, 0);
    }
}

// ------------------------------------------------------------------------------- epilogue
// z / (1 + e^-t)
__device__ __forceinline__ float gate(float z, float t) { return z / (1.f + __builtin_amdgcn_exp2f(-t * kLog2eF)); }

// z Phi(z) = max(z, 0) - |z| q with the tail q = erfc(|z| / sqrt 2) / 2: nothing cancels at negative z, so the result is as
// good there as q is relative to itself.  q = t P(t) e^(-z^2 / 2), t = 1 / (1 + p |z|); P is fitted here, by exchange of the largest
// relative errors (Remez), for |z| to 13.5, where q leaves fp32: degree 7 to 1.3e-7 where the output is fp32 (WIDE), degree 4
// to 3.5e-5, a hundredth of the rounding, where it is bf16.  The power adds up to 1.5 z^2 2^-24 of itself.  (|z| stands still at
// 30, where q is 0, so that an infinity is not multiplied by 0.)  Less than half of erff's instructions: the GELU of
// 8192 x 28672 outputs cost 216 us of 1740 with it.
template <bool WIDE>
__device__ __forceinline__ float gelu(float z) {
    const float a = __builtin_fabsf(z), t = __builtin_amdgcn_rcpf(__builtin_fmaf(WIDE ? 0.30f : 0.38f, a, 1.f));
    float q;
    if constexpr (WIDE) {
        q = __builtin_fmaf(0.0359317251f, t, -0.158275962f);
        q = __builtin_fmaf(q, t, 0.208206534f);
        q = __builtin_fmaf(q, t, -0.0553937852f);
        q = __builtin_fmaf(q, t, 0.129469171f);
        q = __builtin_fmaf(q, t, 0.0996375009f);
        q = __builtin_fmaf(q, t, 0.120798357f);
        q = __builtin_fmaf(q, t, 0.119626388f);
    } else {
        q = __builtin_fmaf(-0.0899283141f, t, 0.188876390f);
        q = __builtin_fmaf(q, t, 0.0919798091f);
        q = __builtin_fmaf(q, t, 0.157829449f);
        q = __builtin_fmaf(q, t, 0.151225135f);
    }
    q *= t * __builtin_amdgcn_exp2f(-0.5f * kLog2eF * z * z);
    return __builtin_fmaf(-__builtin_fminf(a, 30.f), q, __builtin_fmaxf(z, 0.f));
}

template <bool WIDE>
__device__ __forceinline__ void activate8(float* v, int act) {
    switch (act) {  // uniform: outside the loops over values
        case 0: break;
        case 1:
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = v[e] < 0.f ? 0.f : v[e];
            break;
        case 2:
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = gate(v[e], v[e]);
            break;
        case 3:
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = gelu<WIDE>(v[e]);
            break;
        default:  // (1 + tanh a) / 2 = 1 / (1 + e^-2a), 2a = sqrt(8 / pi) (z + 0.044715 z^3)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = gate(v[e], v[e] * __builtin_fmaf(0.0713548162726f * v[e], v[e], 1.5957691216057308f));
    }
}

// Scales and biases of 8 columns.
struct Cols8 {
    f32x4 s[2], b[2];
    __device__ __forceinline__ void load(const float* ws, const float* bias) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s[i] = *reinterpret_cast<const f32x4*>(ws + 4 * i);
            b[i] = *reinterpret_cast<const f32x4*>(bias + 4 * i);
        }
    }
    __device__ __forceinline__ float z(float sum, float sx, int e) const {
        return __builtin_fmaf(sum * sx, s[e >> 2][e & 3], b[e >> 2][e & 3]);
    }
};

// 8 values of the residual
struct Residual8 {
    u32x4 w[2];
    __device__ __forceinline__ void load(const Fp8Args& p, int64_t at) {
        if (p.out_f32) {
            w[0] = ld16(reinterpret_cast<const float*>(p.residual) + at);
            w[1] = ld16(reinterpret_cast<const float*>(p.residual) + at + 4);
        } else {
            w[0] = ld16(reinterpret_cast<const __bf16*>(p.residual) + at);
        }
    }
    __device__ __forceinline__ void add(const Fp8Args& p, float* v) const {
        const uint32_t a[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
        if (p.out_f32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += __uint_as_float(a[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[2 * e] += bf_lo(a[e]);
                v[2 * e + 1] += bf_hi(a[e]);
            }
        }
    }
};
// STREAM: with the non-temporal hint (fp8_streams_out).
template <bool STREAM = false>
__device__ __forceinline__ void store16(void* to, const u32x4& v) {
    if constexpr (STREAM)
        __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(to));
    else
        *reinterpret_cast<u32x4*>(to) = v;
}
template <bool STREAM = false>
__device__ __forceinline__ void store8(const Fp8Args& p, int64_t at, const float* v) {
    if (p.out_f32) {
        float* o = reinterpret_cast<float*>(p.out) + at;
        store16<STREAM>(o, u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
        store16<STREAM>(o + 4, u32x4{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])});
    } else {
        store16<STREAM>(reinterpret_cast<__bf16*>(p.out) + at, u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]),
                                                                     pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])});
    }
}

// 8 output columns n .. of one row from their sums g (packed columns c ..) and, gated, u (c + 16 ..).
__device__ __forceinline__ void finish8(const Fp8Args& p, const float* g, const float* u, int64_t row, int64_t c, int64_t n) {
    const int64_t at = row * p.N + n;
    const float sx = p.xs[row];
    Cols8 k;
    k.load(p.ws + c, p.bias + c);
    Residual8 r;
    if (p.residual) r.load(p, at);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = k.z(g[e], sx, e);
    p.out_f32 ? activate8<true>(v, p.act) : activate8<false>(v, p.act);
    if (p.gated) {
        k.load(p.ws + c + 16, p.bias + c + 16);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= k.z(u[e], sx, e);
    }
    if (p.residual) r.add(p, v);
    store8(p, at, v);
}

// Columns c .. c + 7 of `cols` packed columns from column c0 on: which output they are.  Gated: c walks the
// gate blocks alone.
struct Column {
    int64_t packed, out;
};
__device__ __forceinline__ Column column_of(int64_t c0, int c, int gated) {
    if (!gated) return Column{c0 + c, c0 + c};
    const int block = c >> 4, in = c & 15;
    return Column{c0 + 32 * block + in, c0 / 2 + c};
}

// LDS serves a wave's instructions in order: what its lanes wrote before is what they read after, as long
// as the compiler keeps the order.
__device__ __forceinline__ void lds_in_order() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

// Joins the splits' partial sums in order: one thread to 8 output columns of a row.
__global__ __launch_bounds__(256) void fp8_join_kernel(Fp8Args p) {
    const int64_t per_row = p.N / 8, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= p.M * per_row) return;
    const int64_t row = i / per_row, ld = p.blocks * 16;
    const Column k = column_of(0, (int)(i % per_row * 8), p.gated);
    float g[8] = {}, u[8] = {};
    for (int s = 0; s < p.splits; ++s) {
        const float* in = p.part + ((int64_t)s * p.M + row) * ld + k.packed;
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] += in[e];
        if (p.gated)
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] += in[16 + e];
    }
    finish8(p, g, u, row, k.packed, k.out);
}

// ------------------------------------------------------------------------------- few rows
// The KS waves' sums of ROWS x 16 NC packed columns, LDR floats to a row and one wave's behind the other's in LDS.
template <int ROWS, int NC, int KS, int LDR>
__device__ __forceinline__ void finish_waves(const Fp8Args& p, const float* sums, int64_t m0, int64_t nb0) {
    const int per_row = p.gated ? NC : NC * 2, rows = (int)min((int64_t)ROWS, p.M - m0);
    for (int i = threadIdx.x; i < rows * per_row; i += KS * kWave) {
        const int r = i / per_row;
        const Column k = column_of(nb0 * 16, i % per_row * 8, p.gated);
        if (k.out >= p.N) continue;
        const float* in = sums + r * LDR + (k.packed - nb0 * 16);
        float g[8] = {}, u[8] = {};
#pragma unroll
        for (int w = 0; w < KS; ++w) {
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] += in[w * ROWS * LDR + e];
            if (p.gated)
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] += in[w * ROWS * LDR + 16 + e];
        }
        finish8(p, g, u, m0 + r, k.packed, k.out);
    }
}

// 16 rows x 16 NC packed columns to a workgroup, whose KS waves take every KS-th step of 128 codes of K: W comes straight
// from HBM into operand registers, 1 KiB to an instruction and read once; x, which every workgroup reads,
// from L2.  No barrier until the waves' sums meet in LDS.  U steps' loads are issued together.  Bound by W: one row
// 4096 -> 12288 9.5 us (5.3 TB/s with the launch), 8192 -> 28672 37 us (6.3 TB/s).
template <int NC, int KS, int U, bool F32>
__global__ __launch_bounds__(KS* kWave) void fp8_stream_kernel(Fp8Args p) {
    constexpr int LDR = NC * 16 + 4;
    __shared__ __attribute__((aligned(16))) float sums[KS * 16 * LDR];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles_m = (int)((p.M + 15) / 16), t = xcd_contiguous(blockIdx.x, gridDim.x);
    const int64_t m0 = (int64_t)(t % tiles_m) * 16, nb0 = (int64_t)(t / tiles_m) * NC;
    const int nst = (int)(p.kchunks / 2), at = (lane >> 4) * 16;
    const char* xr = p.x + min(m0 + (lane & 15), p.M - 1) * p.K;
    const char* wc[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) wc[c] = p.w + packed_chunk(min(nb0 + c, p.blocks - 1), 0, p.kchunks, lane);

    f32x4 acc[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s = wave; s < nst; s += KS * U) {
        u32x4 a[U][2], b[U][NC][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u == 0 || s + u * KS < nst) {
                const int64_t st = s + u * KS;
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int h = 0; h < 2; ++h) b[u][c][h] = ld16_stream(wc[c] + (st * 2 + h) * kChunkBytes);
#pragma unroll
                for (int h = 0; h < 2; ++h)  // pieces past K: the row's last one, against weights that are zero there
                    a[u][h] = ld16(xr + min(st * 128 + h * 64 + at, p.K - 16));
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u == 0 || s + u * KS < nst) {
#pragma unroll
                for (int c = 0; c < NC; ++c) acc[c] = mfma_codes<F32>(a[u][0], a[u][1], b[u][c][0], b[u][c][1], acc[c]);
            }
    }
    float* mine = sums + wave * 16 * LDR;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) mine[(4 * (lane >> 4) + i) * LDR + c * 16 + (lane & 15)] = acc[c][i];
    __syncthreads();
    finish_waves<16, NC, KS, LDR>(p, sums, m0, nb0);
}

// The same for 32 rows, whose x loads would be half lines: each wave copies its steps of x, as whole 128-byte lines, and
// of W into a ring of D slots of its own in LDS and waits for nobody.  Bound by the copies of x (from L2) and W together, about 55
// bytes a ns and CU: 32 rows 14336 -> 4096 (180 MB of L2 reads by the counters) 15.3 us (loads into registers 18.2), 4096 -> 4096 6.4 (7.3).
template <int NC, int KS, int D, bool F32>
__global__ __launch_bounds__(KS* kWave) void fp8_ring_kernel(Fp8Args p) {
    constexpr int ROWS = 32, P = 4 + 2 * NC, SLOT = P * kChunkBytes, LDR = NC * 16 + 4;
    static_assert(D * SLOT >= ROWS * LDR * 4, "a wave's sums fit its ring");
    static_assert((D - 1) * P < 64, "copies in flight");
    __shared__ __attribute__((aligned(1024))) char smem[KS * D * SLOT];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles_m = (int)((p.M + ROWS - 1) / ROWS), t = xcd_contiguous(blockIdx.x, gridDim.x);
    const int64_t m0 = (int64_t)(t % tiles_m) * ROWS, nb0 = (int64_t)(t / tiles_m) * NC;
    const int nst = (int)(p.kchunks / 2), n = (nst - wave + KS - 1) / KS;  // this wave's steps
    const uint64_t a_base = uniform_u64(p.x + m0 * p.K), b_base = uniform_u64(p.w + nb0 * p.kchunks * kChunkBytes);
    const uint32_t ring = lds_addr32(smem) + wave * D * SLOT, last = (uint32_t)(p.K - 16);
    char* mine = smem + wave * D * SLOT;
    uint32_t a_off[4], a_piece[4], b_off[NC];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int r = j * 8 + (lane >> 3);
        a_off[j] = (uint32_t)((min(m0 + r, p.M - 1) - m0) * p.K);
        a_piece[j] = (uint32_t)(((lane & 7) ^ a_swz(r)) * 16);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) b_off[c] = (uint32_t)packed_chunk(min(nb0 + c, p.blocks - 1) - nb0, 0, p.kchunks, lane);
    auto issue = [&](int i) {
        const int s = wave + i * KS;
        const uint32_t base = ring + (uint32_t)(i % D * SLOT);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                g2lds16_stream_sb(b_base + (uint64_t)(2 * s + h) * kChunkBytes, b_off[c], base + (4 + c * 2 + h) * kChunkBytes);
#pragma unroll
        for (int j = 0; j < 4; ++j)  // pieces past K: the row's last one, against weights that are zero there
            g2lds16_async_sb(a_base, a_off[j] + min((uint32_t)s * 128 + a_piece[j], last), base + j * kChunkBytes);
    };
    f32x4 acc[2][NC];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < D && i < n; ++i) issue(i);
    for (int i = 0; i < n; ++i) {
        if (i + D - 1 < n)
            wait_vmcnt<(D - 1) * P>();  // step i's copies; those of the next D - 1 may be on their way
        else
            wait_vmcnt<0>();
        lds_in_order();
        char* at = mine + i % D * SLOT;
        u32x4 a[2][2], b[NC][2];
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = r * 16 + (lane & 15);
                a[r][h] = lds_ld16(lds_ptr(at + row * 128 + (((h * 4 + (lane >> 4)) ^ a_swz(row)) << 4)));
            }
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) b[c][h] = lds_ld16(lds_ptr(at + (4 + c * 2 + h) * kChunkBytes + lane * 16));
        lds_in_order();
        if (i + D < n) {
            wait_lgkm0();  // step i is in registers: its slot is free
            issue(i + D);
        }
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int c = 0; c < NC; ++c) acc[r][c] = mfma_codes<F32>(a[r][0], a[r][1], b[c][0], b[c][1], acc[r][c]);
    }
    __syncthreads();
    float* sums = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                sums[(wave * ROWS + r * 16 + 4 * (lane >> 4) + i) * LDR + c * 16 + (lane & 15)] = acc[r][c][i];
    __syncthreads();
    finish_waves<ROWS, NC, KS, LDR>(p, sums, m0, nb0);
}

// f(0) .. f(N - 1) with constants: loops whose bodies the compiler would not unroll
template <class F, int... I>
__device__ __forceinline__ void unrolled_(F&& f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void unrolled(F&& f) {
    unrolled_(f, std::make_integer_sequence<int, N>{});
}

// ------------------------------------------------------------------------------- large tiles
// BM x BN tiles (packed columns), WM x WN waves, v_mfma_f32_32x32x64: a stage is 128 codes of K in two halves of 64.
// NST stages in LDS; the products of one half run while the fragments of the next are read, and the copies of
// stage s + NST are issued after the barrier in the middle of stage s, when every wave has read all of it.
// Lane l holds row (or column) l & 31 and, of a half's 64 codes, pieces 2 (l >> 5) and the next; its
// 16 sums are rows 8 (i / 4) + 4 (l >> 5) + i % 4 of column l & 31.
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct Piece2 {
    u32x4 a, b;
};
// Of n things done by the first by/8 of m steps: how many are done before step i.
constexpr int cut(int n, int by, int m, int i) { return n * i * 8 / (by * m) < n ? n * i * 8 / (by * m) : n; }
// Reads are done by the middle of a half's products, copies by three quarters (measured, 8192 x 8192 -> 28672: 1352 us;
// reads to the end 1387, both by the middle 1405).
constexpr int kReadsBy = 4, kCopiesBy = 6;

template <bool F32>
__device__ __forceinline__ f32x16 mfma_32(const Piece2& x, const Piece2& w, f32x16 acc) {
    if constexpr (!F32) {
        const i32x8 a = {(int)x.a.x, (int)x.a.y, (int)x.a.z, (int)x.a.w, (int)x.b.x, (int)x.b.y, (int)x.b.z, (int)x.b.w};
        const i32x8 b = {(int)w.a.x, (int)w.a.y, (int)w.a.z, (int)w.a.w, (int)w.b.x, (int)w.b.y, (int)w.b.z, (int)w.b.w};
        return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc, 0, 0, 0, 0, 0, 0);
    } else {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(x.a.x, x.a.y), widen8(w.a.x, w.a.y), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(x.a.z, x.a.w), widen8(w.a.z, w.a.w), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(x.b.x, x.b.y), widen8(w.b.x, w.b.y), acc, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(x.b.z, x.b.w), widen8(w.b.z, w.b.w), acc, 0, 0, 0);
    }
}

template <int BM, int BN, int WM, int WN, int NST, bool GATED, bool F32, bool STREAM = false>
__global__ __launch_bounds__(WM* WN* kWave) void fp8_tile_kernel(Fp8Args p) {
    constexpr int NW = WM * WN, WTM = BM / WM, WTN = BN / WN, FM = WTM / 32, FN = WTN / 32;
    constexpr int A_BYTES = BM * 128, STAGE = (BM + BN) * 128;
    constexpr int A_INS = BM / 8 / NW, B_INS = BN / 8 / NW, PER = A_INS + B_INS;
    constexpr int NMF = FM * FN, NRD = 2 * (FM + FN), LDR = 68;
    static_assert(FN % 2 == 0, "the epilogue takes 32 x 64 sums at a time");
    static_assert(NST * STAGE >= NW * 32 * LDR * 4, "the epilogue's sums fit the stages");
    __shared__ __attribute__((aligned(1024))) char smem[NST * STAGE];
    __shared__ float row_s[BM], col_s[BN], col_b[BN];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    // tiles: XCD-contiguous, then blocks of GM row blocks x all column tiles
    const int tiles_m = (int)((p.M + BM - 1) / BM), tiles_n = (int)((p.blocks * 16 + BN - 1) / BN);
    const int tiles = tiles_m * tiles_n, tt = xcd_contiguous(blockIdx.x, gridDim.x), t = tt % tiles, split = tt / tiles;
    constexpr int GM = 4;
    const int span = GM * tiles_n, first = t / span * GM, gsz = min(tiles_m - first, GM);
    const int pm = first + t % span % gsz, pn = t % span / gsz;
    const int64_t m0 = (int64_t)pm * BM, c0 = (int64_t)pn * BN, nb0 = c0 / 16;
    const int all = (int)(p.kchunks / 2), s0 = (int)((int64_t)all * split / p.splits),
              nst = (int)((int64_t)all * (split + 1) / p.splits) - s0;  // stages of this split
    for (int i = tid; i < BM; i += NW * kWave) row_s[i] = p.xs[min(m0 + i, p.M - 1)];
    for (int i = tid; i < BN; i += NW * kWave) {
        const int64_t c = min(c0 + i, p.blocks * 16 - 1);
        col_s[i] = p.ws[c];
        col_b[i] = p.bias[c];
    }

    uint32_t a_off[A_INS], b_off[B_INS];
    uint32_t a_piece[A_INS];
#pragma unroll
    for (int j = 0; j < A_INS; ++j) {
        const int r = (wave + j * NW) * 8 + (lane >> 3);
        a_off[j] = (uint32_t)((min(m0 + r, p.M - 1) - m0) * p.K);
        a_piece[j] = (uint32_t)(((lane & 7) ^ a_swz(r)) * 16);
    }
#pragma unroll
    for (int j = 0; j < B_INS; ++j) {
        const int c = wave + j * NW;
        b_off[j] = (uint32_t)packed_chunk(min(nb0 + (c >> 1), p.blocks - 1) - nb0, c & 1, p.kchunks, lane);
    }
    const uint64_t a_base = uniform_u64(p.x + m0 * p.K);
    const uint64_t b_base = uniform_u64(p.w + nb0 * p.kchunks * kChunkBytes);
    const uint32_t smem_addr = lds_addr32(smem), last = (uint32_t)(p.K - 16);
    // copy k of stage s's PER (this wave's), into slot s % NST
    auto issue = [&](int s, auto kc) {
        constexpr int k = decltype(kc)::value;
        const uint32_t base = smem_addr + (uint32_t)(s % NST * STAGE);
        if constexpr (k < A_INS)  // pieces past K: the row's last one, against weights that are zero there
            g2lds16_async_sb(a_base, a_off[k] + min((uint32_t)(s0 + s) * 128 + a_piece[k], last),
                             base + (uint32_t)((wave + k * NW) * kChunkBytes));
        else
            g2lds16_async_sb(b_base + (uint64_t)(s0 + s) * (2 * kChunkBytes), b_off[k - A_INS],
                             base + (uint32_t)(A_BYTES + (wave + (k - A_INS) * NW) * kChunkBytes));
    };
    const int g = lane >> 5;
    // reads k of a half's NRD: the pieces of row fragments, then of column fragments
    uint32_t a_at[FM][2];
#pragma unroll
    for (int fm = 0; fm < FM; ++fm) {
        const int r = wm * WTM + fm * 32 + (lane & 31);
        a_at[fm][0] = (uint32_t)(r * 128 + (((2 * g) ^ a_swz(r)) << 4));
        a_at[fm][1] = (uint32_t)(r * 128 + (((2 * g + 1) ^ a_swz(r)) << 4));
    }
    const uint32_t b_at = (uint32_t)(A_BYTES + (wn * WTN / 16 + ((lane >> 4) & 1)) * 2 * kChunkBytes + (lane & 15) * 16 + g * 512);
    auto read = [&](int s, int h, auto kc, Piece2(&fa)[FM], Piece2(&fb)[FN]) {
        constexpr int k = decltype(kc)::value;
        char* base = smem + s % NST * STAGE;
        u32x4 v;
        if constexpr (k < 2 * FM) {
            v = lds_ld16(lds_ptr(base + (a_at[k / 2][k & 1] ^ (h * 64))));
            (k & 1 ? fa[k / 2].b : fa[k / 2].a) = v;
        } else {
            constexpr int f = (k - 2 * FM) / 2;
            v = lds_ld16(lds_ptr(base + b_at + f * 4 * kChunkBytes + h * kChunkBytes + (k & 1) * 256));
            (k & 1 ? fb[f].b : fb[f].a) = v;
        }
    };
    f32x16 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    // The products of one half (fa, fb), and between them the reads of the next half (na, nb) from stage rs
    // and, with COPY, the copies of stage cs.
    auto compute = [&](Piece2(&fa)[FM], Piece2(&fb)[FN], int rs, int rh, Piece2(&na)[FM], Piece2(&nb)[FN], auto copies, int cs) {
        constexpr bool COPY = decltype(copies)::value;
        const bool copy = COPY && cs < nst;
        unrolled<NMF>([&](auto ic) {
            constexpr int i = decltype(ic)::value, fm = i / FN, fn = i % FN;
            constexpr int r0 = cut(NRD, kReadsBy, NMF, i), r1 = cut(NRD, kReadsBy, NMF, i + 1), k0 = cut(PER, kCopiesBy, NMF, i), k1 = cut(PER, kCopiesBy, NMF, i + 1);
            unrolled<r1 - r0>([&](auto k) { read(rs, rh, std::integral_constant<int, r0 + decltype(k)::value>{}, na, nb); });
            if constexpr (COPY && k1 > k0) {
                if (copy) unrolled<k1 - k0>([&](auto k) { issue(cs, std::integral_constant<int, k0 + decltype(k)::value>{}); });
            }
            acc[fm][fn] = mfma_32<F32>(fa[fm], fb[fn], acc[fm][fn]);
            __builtin_amdgcn_sched_barrier(0);
        });
    };

    for (int s = 0; s < NST && s < nst; ++s) unrolled<PER>([&](auto k) { issue(s, k); });
    if (nst >= NST)
        wait_vmcnt<(NST - 1) * PER>();  // stage 0
    else
        wait_vmcnt<0>();
    block_barrier();
    Piece2 fa0[FM], fb0[FN], fa1[FM], fb1[FN];
    unrolled<NRD>([&](auto k) { read(0, 0, k, fa0, fb0); });
    for (int s = 0; s < nst; ++s) {
        compute(fa0, fb0, s, 1, fa1, fb1, std::false_type{}, 0);
        // this wave's copies of stage s + 1 have landed (those of s + 2 .. s + NST - 1 may be on their way)
        if (NST > 2 && s + NST - 1 < nst)
            wait_vmcnt<(NST - 2) * PER>();
        else
            wait_vmcnt<0>();
        wait_lgkm0();  // this wave's reads of stage s are complete
        block_barrier();
        // past the end this reads stale data that is never used
        compute(fa1, fb1, s + 1, 0, fa0, fb0, std::true_type{}, s + NST);
    }
    if (p.part) {
        const int64_t ld = p.blocks * 16;
        unrolled<FM * FN>([&](auto ic) {
            constexpr int fm = decltype(ic)::value / FN, fn = decltype(ic)::value % FN;
            const int64_t c = c0 + wn * WTN + fn * 32 + (lane & 31);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int64_t row = m0 + wm * WTM + fm * 32 + 8 * (i / 4) + 4 * g + i % 4;
                if (row < p.M && c < ld) p.part[((int64_t)split * p.M + row) * ld + c] = acc[fm][fn][i];
            }
        });
        wait_lgkm0();
        return;
    }
    wait_lgkm0();
    __syncthreads();
    // 32 x 64 sums of a wave at a time through LDS: eight columns to a lane, whole 128-byte lines to a store.  Rows'
    // and columns' scales come from LDS, so that no step waits for memory.
    float* sums = reinterpret_cast<float*>(smem) + wave * 32 * LDR;
    constexpr int IT = GATED ? 2 : 4, PER_ROW = 64 / 8 / (GATED ? 2 : 1);
    const int col = GATED ? (lane % PER_ROW / 2) * 32 + (lane & 1) * 8 : lane % PER_ROW * 8;  // of the gate, packed
    unrolled<FN / 2>([&](auto fpc) {
        constexpr int fp = decltype(fpc)::value;
        const int pc = wn * WTN + fp * 64;  // the region's first packed column in the tile
        const int64_t n = GATED ? (c0 + pc) / 2 + lane % PER_ROW * 8 : c0 + pc + col;
        Cols8 k, ku;
        k.load(col_s + pc + col, col_b + pc + col);
        if (GATED) ku.load(col_s + pc + col + 16, col_b + pc + col + 16);
        unrolled<FM>([&](auto fmc) {
            constexpr int fm = decltype(fmc)::value;
            const int r0 = wm * WTM + fm * 32 + lane / PER_ROW;
            Residual8 res[IT];
            if (p.residual) {
#pragma unroll
                for (int it = 0; it < IT; ++it) {
                    const int64_t row = m0 + r0 + it * (64 / PER_ROW);
                    if (row < p.M && n < p.N) res[it].load(p, row * p.N + n);
                }
            }
#pragma unroll
            for (int f = 0; f < 2; ++f)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    sums[(8 * (i / 4) + 4 * g + i % 4) * LDR + f * 32 + (lane & 31)] = acc[fm][fp * 2 + f][i];
            lds_in_order();
#pragma unroll
            for (int it = 0; it < IT; ++it) {
                const int r = it * (64 / PER_ROW);
                const int64_t row = m0 + r0 + r;
                const float* at = sums + (lane / PER_ROW + r) * LDR + col;
                const f32x4 a0 = *reinterpret_cast<const f32x4*>(at), a1 = *reinterpret_cast<const f32x4*>(at + 4);
                const float sx = row_s[r0 + r];
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = k.z(e < 4 ? a0[e & 3] : a1[e & 3], sx, e);
                activate8<F32>(v, p.act);
                if (GATED) {
                    const f32x4 u0 = *reinterpret_cast<const f32x4*>(at + 16), u1 = *reinterpret_cast<const f32x4*>(at + 20);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] *= ku.z(e < 4 ? u0[e & 3] : u1[e & 3], sx, e);
                }
                if (p.residual) res[it].add(p, v);
                if (row < p.M && n < p.N) store8<STREAM>(p, row * p.N + n, v);
            }
            lds_in_order();
        });
    });
}

// ------------------------------------------------------------------------------- weights
struct Fp8Prep {
    const void* W;
    const float *scales, *bias;
    const void* gamma;
    int64_t K, N, kchunks;
    char* chunks;
    float *out_scales, *out_bias;
    int block0, step;  // packed block of the first 16 columns, and from 16 columns to the next
};

template <class T>
__device__ __forceinline__ float weight_at(const Fp8Prep& p, int64_t k, int64_t n) {
    const float w = to_f32<T>(reinterpret_cast<const T*>(p.W)[k * p.N + n]);
    return p.gamma ? w * to_f32<T>(reinterpret_cast<const T*>(p.gamma)[k]) : w;
}

// Scales (given, or from each column's largest value) and bias, in packed order; 64 columns to a workgroup.
template <class T>
__global__ __launch_bounds__(1024) void fp8_scales_kernel(Fp8Prep p) {
    const int col = threadIdx.x & 63, part = threadIdx.x >> 6;
    const int64_t n = (int64_t)blockIdx.x * 64 + col;
    uint32_t top = 0;
    if constexpr (!std::is_same<T, uint8_t>::value) {
        __shared__ uint32_t tops[16][64];
        if (n < p.N)
            for (int64_t k = part; k < p.K; k += 16) {
                const uint32_t u = __float_as_uint(weight_at<T>(p, k, n)) & 0x7fffffffu;
                top = u > top ? u : top;
            }
        tops[part][col] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i) top = tops[i][col] > top ? tops[i][col] : top;
    }
    if (part || n >= (p.N + 15) / 16 * 16) return;
    float s = 0.f, b = 0.f;
    if (n < p.N) {
        if constexpr (std::is_same<T, uint8_t>::value)
            s = p.scales[n];
        else
            s = top >= 0x7f800000u ? __builtin_nanf("") : __builtin_fmaxf(__uint_as_float(top) / 448.f, 7.52316385e-37f);
        if (p.bias) b = p.bias[n];
    }
    const int64_t c = (p.block0 + n / 16 * p.step) * 16 + n % 16;
    p.out_scales[c] = s;
    p.out_bias[c] = b;
}

// Chunks: one 16-byte piece (a column's 16 k) to a thread, 64 columns x 4 pieces to a workgroup.
template <class T>
__global__ __launch_bounds__(256) void fp8_pack_kernel(Fp8Prep p) {
    const int64_t n = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    if (n >= (p.N + 15) / 16 * 16) return;
    const int64_t nb = p.block0 + n / 16 * p.step;
    const int piece = threadIdx.x >> 6;
    for (int64_t kc = blockIdx.y; kc < p.kchunks; kc += gridDim.y) {
        const int64_t k0 = kc * 64 + piece * 16;
        u32x4 w = {0u, 0u, 0u, 0u};
        if (n < p.N && k0 < p.K) {  // K is a multiple of 16: whole pieces
            if constexpr (std::is_same<T, uint8_t>::value) {
                const uint8_t* in = reinterpret_cast<const uint8_t*>(p.W) + k0 * p.N + n;
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e >> 2] |= (uint32_t)in[e * p.N] << (8 * (e & 3));
            } else {
                const float s = p.out_scales[nb * 16 + n % 16];
                if (s == s) {  // a column with a NaN scale has codes 0
                    float f[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) f[e] = weight_at<T>(p, k0 + e, n) / s;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * e], f[4 * e + 1], 0, false);
                        w[e] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * e + 2], f[4 * e + 3], lo, true);
                    }
                }
            }
        }
        *reinterpret_cast<u32x4*>(p.chunks + packed_chunk(nb, kc, p.kchunks, (int)(n % 16) + 16 * piece)) = w;
    }
}

template <class T>
static hipError_t prepare_columns(const Fp8Prep& p, hipStream_t s) {
    const unsigned groups = (unsigned)((p.N + 63) / 64);
    fp8_scales_kernel<T><<<dim3(groups), 1024, 0, s>>>(p);
    fp8_pack_kernel<T><<<dim3(groups, (unsigned)(p.kchunks < 64 ? p.kchunks : 64)), 256, 0, s>>>(p);
    return hipGetLastError();
}

hipError_t launch_linear_fp8_prepare(const void* W, const float* scales, const void* gamma, const float* bias,
                                     const void* W_up, const float* up_scales, const float* up_bias, int64_t K, int64_t N,
                                     int dtype, void* packed, hipStream_t s) {
    const Fp8Layout l = fp8_layout(K, N, W_up != nullptr);
    char* base = reinterpret_cast<char*>(packed);
    for (int up = 0; up < (W_up ? 2 : 1); ++up) {
        const Fp8Prep p{up ? W_up : W, up ? up_scales : scales, up ? up_bias : bias, gamma, K, N, l.kchunks, base,
                        reinterpret_cast<float*>(base + l.scales), reinterpret_cast<float*>(base + l.bias), up, W_up ? 2 : 1};
        const hipError_t e = dtype == 0   ? prepare_columns<float>(p, s)
                             : dtype == 1 ? prepare_columns<__bf16>(p, s)
                                          : prepare_columns<uint8_t>(p, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <bool GATED, bool F32>
static void launch_tile(const Fp8Args& p, int tile, bool stream, dim3 grid, dim3 threads, hipStream_t s) {
    switch (tile) {
        case 0: fp8_tile_kernel<64, 64, 2, 1, 4, GATED, F32><<<grid, threads, 0, s>>>(p); break;
        case 1: fp8_tile_kernel<64, 128, 2, 2, 4, GATED, F32><<<grid, threads, 0, s>>>(p); break;
        case 2: fp8_tile_kernel<128, 128, 2, 2, 4, GATED, F32><<<grid, threads, 0, s>>>(p); break;
        case 3:
            stream ? fp8_tile_kernel<256, 128, 4, 2, 3, GATED, F32, true><<<grid, threads, 0, s>>>(p)
                   : fp8_tile_kernel<256, 128, 4, 2, 3, GATED, F32><<<grid, threads, 0, s>>>(p);
            break;
        default:
            if constexpr (!F32)
                stream ? fp8_tile_kernel<256, 256, 4, 2, 2, GATED, F32, true><<<grid, threads, 0, s>>>(p)
                       : fp8_tile_kernel<256, 256, 4, 2, 2, GATED, F32><<<grid, threads, 0, s>>>(p);
    }
}

template <bool F32>
static void launch_few_rows(const Fp8Args& p, int rf, int nc, dim3 grid, dim3 threads, hipStream_t s) {
    if (rf == 1) {
        switch (nc) {  // 2 steps' loads at a time while W's bytes in flight are few
            case 1: fp8_stream_kernel<1, 8, 2, F32><<<grid, threads, 0, s>>>(p); break;
            case 2: fp8_stream_kernel<2, 8, 2, F32><<<grid, threads, 0, s>>>(p); break;
            case 3: fp8_stream_kernel<3, 8, 1, F32><<<grid, threads, 0, s>>>(p); break;
            case 4: fp8_stream_kernel<4, 8, 1, F32><<<grid, threads, 0, s>>>(p); break;
            case 6: fp8_stream_kernel<6, 8, 1, F32><<<grid, threads, 0, s>>>(p); break;
            case 7:
                if constexpr (!F32) fp8_stream_kernel<7, 8, 1, F32><<<grid, threads, 0, s>>>(p);
                break;
            default: fp8_stream_kernel<8, 8, 1, F32><<<grid, threads, 0, s>>>(p);
        }
    } else {
        switch (nc) {
            case 1: fp8_ring_kernel<1, 8, 3, F32><<<grid, threads, 0, s>>>(p); break;
            case 2: fp8_ring_kernel<2, 8, 2, F32><<<grid, threads, 0, s>>>(p); break;
            case 3: fp8_ring_kernel<3, 4, 3, F32><<<grid, threads, 0, s>>>(p); break;
            case 4: fp8_ring_kernel<4, 4, 3, F32><<<grid, threads, 0, s>>>(p); break;
            case 6: fp8_ring_kernel<6, 4, 2, F32><<<grid, threads, 0, s>>>(p); break;
            default: fp8_ring_kernel<7, 4, 2, F32><<<grid, threads, 0, s>>>(p);
        }
    }
}

hipError_t launch_linear_fp8(const void* x, const float* xs, const void* packed, int64_t M, int64_t K, int64_t N, int gated,
                             int act, const void* residual, int out_dtype, const Fp8Plan& plan, void* workspace, void* out,
                             hipStream_t s) {
    const Fp8Layout l = fp8_layout(K, N, gated);
    const char* base = reinterpret_cast<const char*>(packed);
    const bool f32 = out_dtype == 0, stream = fp8_streams_out(plan, N, f32, reinterpret_cast<uintptr_t>(out));
    const Fp8Args p{reinterpret_cast<const char*>(x), xs, base, reinterpret_cast<const float*>(base + l.scales),
                    reinterpret_cast<const float*>(base + l.bias), residual, out,
                    plan.splits > 1 ? reinterpret_cast<float*>(workspace) : nullptr, M, K, N, l.kchunks, l.blocks, act, gated,
                    f32, (int)plan.splits};
    const dim3 grid((unsigned)fp8_workgroups(plan, M, l.blocks)), threads((unsigned)fp8_threads(plan));
    if (plan.tile < 0)
        f32 ? launch_few_rows<true>(p, plan.rf, plan.nc, grid, threads, s) : launch_few_rows<false>(p, plan.rf, plan.nc, grid, threads, s);
    else if (gated)
        f32 ? launch_tile<true, true>(p, plan.tile, stream, grid, threads, s)
            : launch_tile<true, false>(p, plan.tile, stream, grid, threads, s);
    else
        f32 ? launch_tile<false, true>(p, plan.tile, stream, grid, threads, s)
            : launch_tile<false, false>(p, plan.tile, stream, grid, threads, s);
    if (plan.splits > 1) fp8_join_kernel<<<dim3((unsigned)((M * (N / 8) + 255) / 256)), 256, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace dn
