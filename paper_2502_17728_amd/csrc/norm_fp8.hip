// norm_fp8.hip -- rows on their way into an 8-bit product: the residual stream's addition, its
// RMSNorm, and e4m3 codes with one scale per row.
//
// With h = x + residual, RMSNorm gives y = r (h gamma), r = 1/sqrt(sum h^2 / K + eps) > 0.  A
// code is y / scale with scale = max |y| / 448: r stands in both and cancels, so the codes are
// those of a = h gamma and the scale is r max |a| / 448.  The normalization of Eq. (6) thereby
// moves past the product, into the scale that the product's epilogue applies.
//
// Bound by HBM: each value is read once, kept in registers over the reduction and written once.
#include "dn_device.hpp"
#include "dn_launch.hpp"
#include "fp8_rules.hpp"

namespace dn {

constexpr float kF8Max = 448.f;
constexpr float kLeastScale = 7.52316385e-37f;  // 2^-120

// What a row becomes.
enum class RowOut { kNorm, kNormFp8, kFp8 };

struct RowArgs {
    const void* x;
    const void* residual;  // null: none
    const void* gamma;     // null: ones
    void* sum;             // x + residual, rounded; null without a residual
    void* y;               // rows of T, or codes
    float* scales;
    int64_t M, K;
    float eps;
};

// a / s as a code's rounding sees it, s >= kExactFrom: inv = 1 / s to the nearest, and the remainder of a inv is exact and puts it
// right.  Next to a tie t of two codes (5 bits) a inv is one of the fp32 neighbours of a / s, so the remainder is s / 2
// steps of them at most, the error of its product with inv below 2^-25 steps, and no quotient of two 24-bit numbers is as near as that
// to the middle of two neighbours.  8192 x 8192 bf16 84.1 us, with the division 85.6; rows alone 4096 x 14336 26.2 and 31.5.
constexpr float kExactFrom = 2.01948392e-28f;  // 2^-92: the remainder's last bit is 2^-149 at least
__device__ __forceinline__ float quotient(float a, float s, float inv) {
    const float q = a * inv;
    return __builtin_fmaf(__builtin_fmaf(-q, s, a), inv, q);
}

// 8 consecutive values of a row as they lie in memory
template <class T>
struct Raw8;
template <>
struct Raw8<__bf16> {
    u32x4 w;
    __device__ __forceinline__ void load(const __bf16* p) { w = ld16(p); }
    __device__ __forceinline__ void get(float* f) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[2 * e] = bf_lo(w[e]);
            f[2 * e + 1] = bf_hi(w[e]);
        }
    }
    static __device__ __forceinline__ void put(__bf16* p, const float* f) {
        *reinterpret_cast<u32x4*>(p) =
            u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
    }
};
template <>
struct Raw8<float> {
    f32x4 a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const f32x4*>(p);
        b = *reinterpret_cast<const f32x4*>(p + 4);
    }
    __device__ __forceinline__ void get(float* f) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[e] = a[e];
            f[4 + e] = b[e];
        }
    }
    static __device__ __forceinline__ void put(float* p, const float* f) {
        *reinterpret_cast<f32x4*>(p) = f32x4{f[0], f[1], f[2], f[3]};
        *reinterpret_cast<f32x4*>(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
    }
};

__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// TPR threads to a row, NV pieces of 8 values to a thread; a workgroup takes 256 / TPR rows, or one.
template <class T, int TPR, int NV, RowOut OUT>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rows_kernel(RowArgs p) {
    constexpr int NT = TPR < 256 ? 256 : TPR, NW = TPR / kWave;
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * (NT / TPR) + threadIdx.x / TPR;
    if (row >= p.M) return;  // whole waves, and no barrier below where a workgroup has several rows
    const int pieces = (int)(p.K / 8);
    const T* x = reinterpret_cast<const T*>(p.x) + row * p.K;
    const T* res = reinterpret_cast<const T*>(p.residual) + row * p.K;
    const T* gamma = reinterpret_cast<const T*>(p.gamma);
    T* sum = reinterpret_cast<T*>(p.sum) + row * p.K;

    // every load first: sum may lie over x or residual, so no load may pass a store
    Raw8<T> rx[NV], rr[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (t + j * TPR < pieces) rx[j].load(x + (t + j * TPR) * 8);
    if (p.residual) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (t + j * TPR < pieces) rr[j].load(res + (t + j * TPR) * 8);
    }
    float a[NV][8], ss = 0.f;
    uint32_t top = 0;  // largest |a| by its bits: an infinity or NaN is above every number
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int at = (t + j * TPR) * 8;
        if (t + j * TPR >= pieces) continue;
        rx[j].get(a[j]);
        if (p.residual) {
            float r[8];
            rr[j].get(r);
#pragma unroll
            for (int e = 0; e < 8; ++e) a[j][e] += r[e];
            Raw8<T>::put(sum + at, a[j]);
        }
        if constexpr (OUT != RowOut::kFp8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(a[j][e], a[j][e], ss);
            if (gamma) {
                Raw8<T> rg;
                float g[8];
                rg.load(gamma + at);
                rg.get(g);
#pragma unroll
                for (int e = 0; e < 8; ++e) a[j][e] *= g[e];
            }
        }
        if constexpr (OUT != RowOut::kNorm) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t u = __float_as_uint(a[j][e]) & 0x7fffffffu;
                top = u > top ? u : top;
            }
        }
    }
    if constexpr (OUT != RowOut::kFp8) ss = wave_sum(ss);
    if constexpr (OUT != RowOut::kNorm) {
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) {
            const uint32_t u = __shfl_xor(top, o);
            top = u > top ? u : top;
        }
    }
    if constexpr (NW > 1) {
        __shared__ float part_ss[NW];
        __shared__ uint32_t part_top[NW];
        if ((threadIdx.x & 63) == 0) {
            part_ss[threadIdx.x >> 6] = ss;
            part_top[threadIdx.x >> 6] = top;
        }
        __syncthreads();
        ss = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            ss += part_ss[w];
            top = part_top[w] > top ? part_top[w] : top;
        }
    }
    const float r = OUT == RowOut::kFp8 ? 1.f : rstd_from_moments(ss / (float)p.K, 0.f, p.eps);
    if constexpr (OUT == RowOut::kNorm) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (t + j * TPR >= pieces) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) a[j][e] *= r;
            Raw8<T>::put(reinterpret_cast<T*>(p.y) + row * p.K + (t + j * TPR) * 8, a[j]);
        }
    } else {
        const bool bad = top >= 0x7f800000u;
        const float s = __builtin_fmaxf(__uint_as_float(top) / kF8Max, kLeastScale);
        const float inv = 1.f / s;
        if (t == 0) p.scales[row] = bad ? __builtin_nanf("") : s * r;
        char* codes = reinterpret_cast<char*>(p.y) + row * p.K;
        auto put = [&](auto quotient_of) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (t + j * TPR >= pieces) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e) a[j][e] = quotient_of(a[j][e]);
                uint2 w = {pack_e4m3(a[j][0], a[j][1], a[j][2], a[j][3]), pack_e4m3(a[j][4], a[j][5], a[j][6], a[j][7])};
                if (bad) w = uint2{0u, 0u};
                *reinterpret_cast<uint2*>(codes + (t + j * TPR) * 8) = w;
            }
        };
        if (s >= kExactFrom)
            put([&](float v) { return quotient(v, s, inv); });
        else
            put([&](float v) { return v / s; });
    }
}

// Only the kernels that plan_rows can choose: up to 2 pieces to each of 64 threads, 4 to each of 256 and, as long as rows
// can be, 4 (fp32) or 8 to each of 1024.
template <class T, int TPR, RowOut OUT>
static hipError_t launch_pieces(const RowArgs& p, int nv, hipStream_t s) {
    constexpr int NT = TPR < 256 ? 256 : TPR, MOST = TPR == 64 ? 2 : TPR == 256 || sizeof(T) == 4 ? 4 : 8;
    const dim3 grid((unsigned)((p.M + NT / TPR - 1) / (NT / TPR)));
    if (nv == 1)
        rows_kernel<T, TPR, 1, OUT><<<grid, NT, 0, s>>>(p);
    else if (nv == 2)
        rows_kernel<T, TPR, 2, OUT><<<grid, NT, 0, s>>>(p);
    else if (MOST == 4 || nv == 4)
        rows_kernel<T, TPR, MOST < 4 ? MOST : 4, OUT><<<grid, NT, 0, s>>>(p);
    else
        rows_kernel<T, TPR, MOST, OUT><<<grid, NT, 0, s>>>(p);
    return hipGetLastError();
}

template <class T, RowOut OUT>
static hipError_t launch_rows(const RowArgs& p, hipStream_t s) {
    const RowPlan plan = plan_rows(p.M, p.K);
    switch (plan.threads) {
        case 64: return launch_pieces<T, 64, OUT>(p, plan.pieces, s);
        case 256: return launch_pieces<T, 256, OUT>(p, plan.pieces, s);
        default: return launch_pieces<T, 1024, OUT>(p, plan.pieces, s);
    }
}

hipError_t launch_residual_rmsnorm(const void* x, const void* residual, const void* gamma, int64_t M, int64_t K, float eps,
                                   int dtype, void* sum, void* y, float* scales, hipStream_t s) {
    const RowArgs p{x, residual, gamma, sum, y, scales, M, K, eps};
    if (dtype == 0) return scales ? launch_rows<float, RowOut::kNormFp8>(p, s) : launch_rows<float, RowOut::kNorm>(p, s);
    return scales ? launch_rows<__bf16, RowOut::kNormFp8>(p, s) : launch_rows<__bf16, RowOut::kNorm>(p, s);
}

hipError_t launch_rows_fp8(const void* x, int64_t M, int64_t K, int dtype, void* codes, float* scales, hipStream_t s) {
    const RowArgs p{x, nullptr, nullptr, nullptr, codes, scales, M, K, 0.f};
    return dtype == 0 ? launch_rows<float, RowOut::kFp8>(p, s) : launch_rows<__bf16, RowOut::kFp8>(p, s);
}

}  // namespace dn
