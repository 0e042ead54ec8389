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
// products that cancel): 1.5e-5 of a result of normal data in the 2-norm, without bias, for any K.
// A bf16 output's rounding is 100 times that.  An fp32 output's is not: there the codes are widened to bf16, which
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

__device__ __forceinline__ float activation(float z, int act) {
    switch (act) {
        case 1: return z < 0.f ? 0.f : z;
        case 2: return gate(z, z);
        case 3: return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
        // (1 + tanh a) / 2 = 1 / (1 + e^-2a), 2a = sqrt(8 / pi) (z + 0.044715 z^3)
        case 4: return gate(z, z * __builtin_fmaf(0.0713548162726f * z, z, 1.5957691216057308f));
        default: return z;
    }
}

// 8 output columns n .. of one row from their sums g (packed columns c ..) and, gated, u (c + 16 ..).
__device__ __forceinline__ void finish8(const Fp8Args& p, const float* g, const float* u, int64_t row, int64_t c, int64_t n) {
    float v[8];
    const float sx = p.xs[row];
    const f32x4 s0 = *reinterpret_cast<const f32x4*>(p.ws + c), s1 = *reinterpret_cast<const f32x4*>(p.ws + c + 4);
    const f32x4 b0 = *reinterpret_cast<const f32x4*>(p.bias + c), b1 = *reinterpret_cast<const f32x4*>(p.bias + c + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(g[e] * sx, e < 4 ? s0[e & 3] : s1[e & 3], e < 4 ? b0[e & 3] : b1[e & 3]);
    if (p.act)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = activation(v[e], p.act);
    if (p.gated) {
        const f32x4 t0 = *reinterpret_cast<const f32x4*>(p.ws + c + 16), t1 = *reinterpret_cast<const f32x4*>(p.ws + c + 20);
        const f32x4 d0 = *reinterpret_cast<const f32x4*>(p.bias + c + 16), d1 = *reinterpret_cast<const f32x4*>(p.bias + c + 20);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] *= __builtin_fmaf(u[e] * sx, e < 4 ? t0[e & 3] : t1[e & 3], e < 4 ? d0[e & 3] : d1[e & 3]);
    }
    const int64_t at = row * p.N + n;
    if (p.out_f32) {
        float* o = reinterpret_cast<float*>(p.out) + at;
        if (p.residual) {
            const float* r = reinterpret_cast<const float*>(p.residual) + at;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += r[e];
        }
        *reinterpret_cast<f32x4*>(o) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4*>(o + 4) = f32x4{v[4], v[5], v[6], v[7]};
    } else {
        __bf16* o = reinterpret_cast<__bf16*>(p.out) + at;
        if (p.residual) {
            const u32x4 r = ld16(reinterpret_cast<const __bf16*>(p.residual) + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[2 * e] += bf_lo(r[e]);
                v[2 * e + 1] += bf_hi(r[e]);
            }
        }
        *reinterpret_cast<u32x4*>(o) =
            u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    }
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

// A wave's ROWS x COLS sums lie in LDS, LDR floats to a row: eight columns to a lane at a time.
template <int ROWS, int COLS, int LDR>
__device__ __forceinline__ void finish_region(const Fp8Args& p, const float* sums, int64_t row0, int64_t c0, int lane, int split) {
    const int per_row = p.part ? COLS / 8 : p.gated ? COLS / 16 : COLS / 8;
    for (int i = lane; i < ROWS * per_row; i += kWave) {
        const int r = i / per_row, c = i % per_row * 8;
        const int64_t row = row0 + r;
        if (row >= p.M) continue;
        if (p.part) {
            if (c0 + c >= p.blocks * 16) continue;
            float* o = p.part + ((int64_t)split * p.M + row) * (p.blocks * 16) + c0 + c;
            const f32x4* in = reinterpret_cast<const f32x4*>(sums + r * LDR + c);
            *reinterpret_cast<f32x4*>(o) = in[0];
            *reinterpret_cast<f32x4*>(o + 4) = in[1];
            continue;
        }
        const Column k = column_of(c0, c, p.gated);
        if (k.out >= p.N) continue;
        const float* g = sums + r * LDR + (k.packed - c0);
        float gv[8], uv[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) gv[e] = g[e];
#pragma unroll
        for (int e = 0; e < 8; ++e) uv[e] = p.gated ? g[16 + e] : 0.f;
        finish8(p, gv, uv, row, k.packed, k.out);
    }
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

// ------------------------------------------------------------------------------- ring kernel
// BM x BN tiles (packed columns) of WM x WN waves.  A stage is 128 codes of K: x rows as whole
// 128-byte lines, 8 rows to a copy, 16-byte pieces swizzled as in LayerNorm's large tiles; W as 1 KiB
// chunks.  NST stages in LDS, copies NST - 1 ahead, one barrier to a stage.
template <int BM, int BN, int WM, int WN, int NST, bool F32>
__global__ __launch_bounds__(WM* WN* kWave) void fp8_ring_kernel(Fp8Args p) {
    constexpr int NW = WM * WN, WTM = BM / WM, WTN = BN / WN, FM = WTM / 16, FN = WTN / 16;
    constexpr int A_BYTES = BM * 128, STAGE = (BM + BN) * 128;
    constexpr int PER = (BM + BN) / 8 / NW;
    constexpr int LDR = WTN + 4;
    static_assert((BM + BN) / 8 % NW == 0, "every wave issues the same number of copies");
    static_assert(NST * STAGE >= NW * WTM * LDR * 4, "the epilogue's sums fit the ring");
    __shared__ __attribute__((aligned(1024))) char smem[NST * STAGE];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int tiles_m = (int)((p.M + BM - 1) / BM), tiles_n = (int)((p.blocks * 16 + BN - 1) / BN);
    const int t = xcd_contiguous(blockIdx.x, gridDim.x);
    const int pm = t % tiles_m, pn = t / tiles_m % tiles_n, split = t / (tiles_m * tiles_n);
    const int64_t m0 = (int64_t)pm * BM, c0 = (int64_t)pn * BN, nb0 = c0 / 16;
    const int all = (int)(p.kchunks / 2), s0 = (int)((int64_t)all * split / p.splits),
              s1 = (int)((int64_t)all * (split + 1) / p.splits);

    const uint64_t a_base = uniform_u64(p.x + m0 * p.K);
    const uint64_t b_base = uniform_u64(p.w + nb0 * p.kchunks * kChunkBytes);
    const uint32_t smem_addr = lds_addr32(smem), last = (uint32_t)(p.K - 16);
    uint32_t off[PER], piece16[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int c = wave + j * NW;
        if (c < BM / 8) {
            const int r = c * 8 + (lane >> 3);
            off[j] = (uint32_t)((min(m0 + r, p.M - 1) - m0) * p.K);
            piece16[j] = (uint32_t)(((lane & 7) ^ a_swz(r)) * 16);
        } else {
            const int b = c - BM / 8;
            off[j] = (uint32_t)(packed_chunk(min(nb0 + (b >> 1), p.blocks - 1) - nb0, b & 1, p.kchunks, lane));
            piece16[j] = 0;
        }
    }
    auto issue = [&](int s) {
        const uint32_t base = smem_addr + (uint32_t)((s - s0) % NST * STAGE);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int c = wave + j * NW;
            if (c < BM / 8)  // pieces past K: the row's last one, against weights that are zero there
                g2lds16_async_sb(a_base, off[j] + min((uint32_t)s * 128 + piece16[j], last), base + c * kChunkBytes);
            else
                g2lds16_async_sb(b_base + (uint64_t)s * (2 * kChunkBytes), off[j], base + c * kChunkBytes);
        }
    };

    f32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < NST - 1 && s0 + j < s1; ++j) issue(s0 + j);
    for (int s = s0; s < s1; ++s) {
        if (s + NST - 2 < s1)
            wait_vmcnt<(NST - 2) * PER>();  // this wave's copies of stage s
        else
            wait_vmcnt<0>();
        block_barrier();  // every wave's, and every wave is done with the slot that is filled next
        if (s + NST - 1 < s1) issue(s + NST - 1);
        const char* base = smem + (s - s0) % NST * STAGE;
        u32x4 fa[FM][2], fb[FN][2];
#pragma unroll
        for (int fm = 0; fm < FM; ++fm)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = wm * WTM + fm * 16 + (lane & 15);
                fa[fm][h] = lds_ld16(lds_ptr((char*)base + r * 128 + (((h * 4 + (lane >> 4)) ^ a_swz(r)) << 4)));
            }
#pragma unroll
        for (int fn = 0; fn < FN; ++fn)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                fb[fn][h] = lds_ld16(lds_ptr((char*)base + A_BYTES + ((wn * FN + fn) * 2 + h) * kChunkBytes + lane * 16));
#pragma unroll
        for (int fm = 0; fm < FM; ++fm)
#pragma unroll
            for (int fn = 0; fn < FN; ++fn) acc[fm][fn] = mfma_codes<F32>(fa[fm][0], fa[fm][1], fb[fn][0], fb[fn][1], acc[fm][fn]);
    }
    __syncthreads();
    float* sums = reinterpret_cast<float*>(smem) + wave * WTM * LDR;
#pragma unroll
    for (int fm = 0; fm < FM; ++fm)
#pragma unroll
        for (int fn = 0; fn < FN; ++fn)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[(fm * 16 + 4 * (lane >> 4) + i) * LDR + fn * 16 + (lane & 15)] = acc[fm][fn][i];
    lds_in_order();
    finish_region<WTM, WTN, LDR>(p, sums, m0 + wm * WTM, c0 + wn * WTN, lane, split);
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

hipError_t launch_linear_fp8(const void* x, const float* xs, const void* packed, int64_t M, int64_t K, int64_t N, int gated,
                             int act, const void* residual, int out_dtype, void* workspace, int64_t splits_that_fit,
                             void* out, hipStream_t s) {
    const Fp8Layout l = fp8_layout(K, N, gated);
    const char* base = reinterpret_cast<const char*>(packed);
    const Fp8Plan plan = plan_fp8(M, K, l.blocks, splits_that_fit);
    Fp8Args p{reinterpret_cast<const char*>(x), xs, base, reinterpret_cast<const float*>(base + l.scales),
              reinterpret_cast<const float*>(base + l.bias), residual, out,
              plan.splits > 1 ? reinterpret_cast<float*>(workspace) : nullptr, M, K, N, l.kchunks, l.blocks, act, gated,
              out_dtype == 0, (int)plan.splits};
    const int64_t tiles = (M + plan.bm - 1) / plan.bm * ((l.blocks * 16 + plan.bn - 1) / plan.bn);
    const dim3 grid((unsigned)(tiles * plan.splits));
    if (p.out_f32)
        fp8_ring_kernel<64, 64, 2, 2, 4, true><<<grid, 256, 0, s>>>(p);
    else
        fp8_ring_kernel<64, 64, 2, 2, 4, false><<<grid, 256, 0, s>>>(p);
    if (plan.splits > 1) fp8_join_kernel<<<dim3((unsigned)((M * (N / 8) + 255) / 256)), 256, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace dn
