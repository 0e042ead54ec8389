// abi.cpp -- the C ABI of libdn (declared in include/dn.h): argument
// validation on the host, then dispatch to the kernel launchers.  No entry
// point touches the HIP runtime before its arguments have been validated.
#include <math.h>
#include <stdint.h>

#include "dn.h"
#include "dn_launch.hpp"
#include "kv_layout.hpp"
#include "launch_rules.hpp"

namespace {

constexpr int kVersion = (0 << 16) | 1;

bool valid_dtype(int dt) { return dt == DN_F32 || dt == DN_BF16; }
size_t esize(int dt) { return dt == DN_F32 ? 4 : 2; }
bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// bytes = a * b * c without overflow (all >= 1); false on overflow.
bool bytes_of(int64_t a, int64_t b, int64_t c, size_t* out) {
    int64_t ab, abc;
    if (__builtin_mul_overflow(a, b, &ab) || __builtin_mul_overflow(ab, c, &abc)) return false;
    *out = (size_t)abc;
    return true;
}

// [p, p+n) and [q, q+m) intersect (NULL ranges never do).
bool overlaps(const void* p, size_t n, const void* q, size_t m) {
    if (!p || !q || n == 0 || m == 0) return false;
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return a < b + m && b < a + n;
}

dn_status from_hip(hipError_t e) { return e == hipSuccess ? DN_OK : DN_ERR_HIP; }

constexpr int64_t kMaxGridX = 0x7fffffff;
constexpr int64_t kMaxBatch = 65535;

}  // namespace

extern "C" {

DN_API const char* dn_status_string(int status) {
    switch (status) {
        case DN_OK: return "DN_OK";
        case DN_ERR_INVALID_ARG: return "DN_ERR_INVALID_ARG";
        case DN_ERR_UNSUPPORTED: return "DN_ERR_UNSUPPORTED";
        case DN_ERR_MISALIGNED: return "DN_ERR_MISALIGNED";
        case DN_ERR_HIP: return "DN_ERR_HIP";
        default: return "DN_ERR_UNKNOWN";
    }
}

DN_API int dn_version(void) { return kVersion; }

DN_API size_t ln_linear_packed_bytes(int64_t K, int64_t N, int dtype) {
    size_t wt;
    if (K < 1 || N < 1 || !valid_dtype(dtype) || !bytes_of(K, N, (int64_t)esize(dtype), &wt)) return 0;
    return dn::packed_layout(K, N, dtype).total;
}

static dn_status prepare_ln(const void* W, const void* gamma, const void* beta, const void* bias, int64_t K,
                            int64_t N, int dtype, int center, void* packed, size_t packed_bytes,
                            ln_linear_weights* w_out, hipStream_t stream) {
    if (!W || !gamma || !packed || !w_out || K < 1 || N < 1 || !valid_dtype(dtype)) return DN_ERR_INVALID_ARG;
    const size_t need = ln_linear_packed_bytes(K, N, dtype);
    if (need == 0 || packed_bytes < need) return DN_ERR_INVALID_ARG;
    if (K % 8 || N % 8) return DN_ERR_UNSUPPORTED;
    if (!aligned(W, 16) || !aligned(gamma, 16) || !aligned(beta, 16) || !aligned(bias, 16) || !aligned(packed, 256))
        return DN_ERR_MISALIGNED;
    const size_t es = esize(dtype);
    if (overlaps(packed, need, W, (size_t)K * N * es) || overlaps(packed, need, gamma, K * es) ||
        overlaps(packed, need, beta, K * es) || overlaps(packed, need, bias, N * es))
        return DN_ERR_INVALID_ARG;
    if ((N + 63) / 64 > kMaxGridX || (K + 63) / 64 > kMaxBatch) return DN_ERR_UNSUPPORTED;
    const dn_status st = from_hip(dn::launch_ln_prepare(W, gamma, beta, bias, K, N, dtype, center, packed, stream));
    if (st == DN_OK) {
        w_out->K = K;
        w_out->N = N;
        w_out->dtype = dtype;
        w_out->layout_version = DN_LN_LAYOUT_VERSION;
        w_out->packed = packed;
    }
    return st;
}

DN_API dn_status ln_linear_prepare(const void* W, const void* gamma, const void* beta, const void* bias,
                                   int64_t K, int64_t N, int dtype, void* packed, size_t packed_bytes,
                                   ln_linear_weights* w_out, hipStream_t stream) {
    return prepare_ln(W, gamma, beta, bias, K, N, dtype, 0, packed, packed_bytes, w_out, stream);
}

DN_API dn_status ln_linear_prepare_centered(const void* W, const void* gamma, const void* beta, const void* bias,
                                            int64_t K, int64_t N, int dtype, void* packed, size_t packed_bytes,
                                            ln_linear_weights* w_out, hipStream_t stream) {
    return prepare_ln(W, gamma, beta, bias, K, N, dtype, 1, packed, packed_bytes, w_out, stream);
}

static dn_status deferred_linear(const void* x, const ln_linear_weights* w, int64_t M, float eps, int rms,
                                 float* stats, void* out, hipStream_t stream, bool on_load = false,
                                 float* stats_out = nullptr) {
    if (!x || !w || !out || !w->packed || M < 1) return DN_ERR_INVALID_ARG;
    if (w->layout_version != DN_LN_LAYOUT_VERSION || w->K < 1 || w->N < 1 || !valid_dtype(w->dtype))
        return DN_ERR_INVALID_ARG;
    if (!isfinite(eps) || eps < 0.f) return DN_ERR_INVALID_ARG;
    const int64_t K = w->K, N = w->N;
    const int dt = w->dtype;
    size_t xb, ob;
    if (!bytes_of(M, K, (int64_t)esize(dt), &xb) || !bytes_of(M, N, (int64_t)esize(dt), &ob))
        return DN_ERR_INVALID_ARG;
    if (K % 8 || N % 8) return DN_ERR_UNSUPPORTED;
    if (!aligned(x, 16) || !aligned(out, 16) || !aligned(w->packed, 256)) return DN_ERR_MISALIGNED;
    const size_t pb = ln_linear_packed_bytes(K, N, dt);
    if (overlaps(out, ob, x, xb) || overlaps(out, ob, w->packed, pb)) return DN_ERR_INVALID_ARG;
    if (((M + 15) / 16) * ((N + 15) / 16) > kMaxGridX) return DN_ERR_UNSUPPORTED;
    if (on_load && !dn::ln_on_load_supported(M, K, N, dt)) return DN_ERR_UNSUPPORTED;
    if (stats) {
        if (!aligned(stats, 16)) return DN_ERR_MISALIGNED;
        const size_t sb = (size_t)M * 8;
        if (overlaps(stats, sb, x, xb) || overlaps(stats, sb, out, ob) || overlaps(stats, sb, w->packed, pb))
            return DN_ERR_INVALID_ARG;
        if (K > (dt == DN_F32 ? dn::kMaxRowElemsF32 : dn::kMaxRowElemsBf16) || (M + 3) / 4 > kMaxGridX)
            return DN_ERR_UNSUPPORTED;
        const dn_status st = from_hip(dn::launch_row_stats(x, M, K, eps, dt, stats, stream));
        if (st != DN_OK) return st;
    }
    if (on_load) return from_hip(dn::launch_ln_linear_on_load(x, w->packed, M, K, N, stats, out, stream));
    return from_hip(dn::launch_ln_linear_deferred(x, w->packed, M, K, N, dt, eps, rms, stats, out, stream,
                                                  stats_out));
}

DN_API dn_status ln_linear_deferred(const void* x, const ln_linear_weights* w, int64_t M, float eps, void* out,
                                    hipStream_t stream) {
    return deferred_linear(x, w, M, eps, 0, nullptr, out, stream);
}

DN_API dn_status ln_linear_serial(const void* x, const ln_linear_weights* w, int64_t M, float eps, float* stats,
                                  void* out, hipStream_t stream) {
    if (!stats) return DN_ERR_INVALID_ARG;
    return deferred_linear(x, w, M, eps, 0, stats, out, stream);
}

DN_API dn_status ln_linear_norm_on_load(const void* x, const ln_linear_weights* w, int64_t M, float eps,
                                        float* stats, void* out, hipStream_t stream) {
    if (!stats) return DN_ERR_INVALID_ARG;
    return deferred_linear(x, w, M, eps, 0, stats, out, stream, true);
}

// Post-LN placement: the deferred product plus the normalized rows themselves
// (the residual branch), from the statistics the product's kernel reduced.
static dn_status post_linear(const void* x, const ln_linear_weights* w, int64_t M, float eps, int rms,
                             const void* gamma, const void* beta, float* stats, void* y, void* out,
                             hipStream_t stream) {
    if (!x || !w || !gamma || !stats || !y || !out || M < 1) return DN_ERR_INVALID_ARG;
    if (w->layout_version != DN_LN_LAYOUT_VERSION || w->K < 1 || w->N < 1 || !valid_dtype(w->dtype))
        return DN_ERR_INVALID_ARG;
    const int64_t K = w->K;
    const size_t es = esize(w->dtype);
    size_t xb, sb, ob;
    if (!bytes_of(M, K, (int64_t)es, &xb) || !bytes_of(M, 2, 4, &sb) || !bytes_of(M, w->N, (int64_t)es, &ob))
        return DN_ERR_INVALID_ARG;
    if (K % 8) return DN_ERR_UNSUPPORTED;
    if (!aligned(gamma, 16) || !aligned(beta, 16) || !aligned(stats, 16) || !aligned(y, 16))
        return DN_ERR_MISALIGNED;
    const size_t pb = ln_linear_packed_bytes(K, w->N, w->dtype);
    if (overlaps(y, xb, x, xb) || overlaps(y, xb, out, ob) || overlaps(y, xb, stats, sb) ||
        overlaps(y, xb, w->packed, pb) || overlaps(y, xb, gamma, K * es) || overlaps(y, xb, beta, K * es) ||
        overlaps(stats, sb, x, xb) || overlaps(stats, sb, out, ob) || overlaps(stats, sb, w->packed, pb) ||
        overlaps(stats, sb, gamma, K * es) || overlaps(stats, sb, beta, K * es))
        return DN_ERR_INVALID_ARG;
    if ((M * K / (w->dtype == DN_F32 ? 4 : 8) + 255) / 256 > kMaxGridX) return DN_ERR_UNSUPPORTED;
    // the product with its concurrent statistics (validated as ln_linear_deferred), exporting them
    const dn_status st = deferred_linear(x, w, M, eps, rms, nullptr, out, stream, false, stats);
    if (st != DN_OK) return st;
    return from_hip(dn::launch_apply_norm(x, stats, gamma, rms ? nullptr : beta, M, K, w->dtype, y, stream));
}

DN_API dn_status ln_linear_deferred_post(const void* x, const ln_linear_weights* w, int64_t M, float eps,
                                         const void* gamma, const void* beta, float* stats, void* y, void* out,
                                         hipStream_t stream) {
    return post_linear(x, w, M, eps, 0, gamma, beta, stats, y, out, stream);
}

DN_API dn_status rms_linear_deferred_post(const void* x, const ln_linear_weights* w, int64_t M, float eps,
                                          const void* gamma, float* stats, void* y, void* out, hipStream_t stream) {
    return post_linear(x, w, M, eps, 1, gamma, nullptr, stats, y, out, stream);
}

DN_API dn_status rms_linear_deferred(const void* x, const ln_linear_weights* w, int64_t M, float eps, void* out,
                                     hipStream_t stream) {
    return deferred_linear(x, w, M, eps, 1, nullptr, out, stream);
}

DN_API size_t swiglu_packed_bytes(int64_t K, int64_t N, int dtype) {
    size_t wt;
    if (K < 1 || N < 1 || !valid_dtype(dtype) || !bytes_of(K, 2 * N + 32, (int64_t)esize(dtype), &wt)) return 0;
    return dn::swiglu_layout(K, N, dtype).total;
}

DN_API dn_status swiglu_prepare(const void* W_gate, const void* W_up, const void* gamma, int64_t K, int64_t N,
                                int dtype, void* packed, size_t packed_bytes, ln_linear_weights* w_out,
                                hipStream_t stream) {
    if (!W_gate || !W_up || !gamma || !packed || !w_out || K < 1 || N < 1 || !valid_dtype(dtype))
        return DN_ERR_INVALID_ARG;
    const size_t need = swiglu_packed_bytes(K, N, dtype);
    if (need == 0 || packed_bytes < need) return DN_ERR_INVALID_ARG;
    if (K % 8 || N % 8) return DN_ERR_UNSUPPORTED;
    if (!aligned(W_gate, 16) || !aligned(W_up, 16) || !aligned(gamma, 16) || !aligned(packed, 256))
        return DN_ERR_MISALIGNED;
    const size_t es = esize(dtype);
    if (overlaps(packed, need, W_gate, (size_t)K * N * es) || overlaps(packed, need, W_up, (size_t)K * N * es) ||
        overlaps(packed, need, gamma, K * es))
        return DN_ERR_INVALID_ARG;
    if ((2 * N + 255) / 256 > kMaxGridX || (K + 63) / 64 > kMaxBatch) return DN_ERR_UNSUPPORTED;
    const dn_status st = from_hip(dn::launch_swiglu_prepare(W_gate, W_up, gamma, K, N, dtype, packed, stream));
    if (st == DN_OK) {
        w_out->K = K;
        w_out->N = N;
        w_out->dtype = dtype;
        w_out->layout_version = DN_SWIGLU_LAYOUT_VERSION;
        w_out->packed = packed;
    }
    return st;
}

DN_API dn_status rms_swiglu_deferred(const void* x, const ln_linear_weights* w, int64_t M, float eps, void* h,
                                     hipStream_t stream) {
    if (!x || !w || !h || !w->packed || M < 1) return DN_ERR_INVALID_ARG;
    if (w->layout_version != DN_SWIGLU_LAYOUT_VERSION || w->K < 1 || w->N < 1 || !valid_dtype(w->dtype))
        return DN_ERR_INVALID_ARG;
    if (!isfinite(eps) || eps < 0.f) return DN_ERR_INVALID_ARG;
    const int64_t K = w->K, N = w->N;
    const int dt = w->dtype;
    size_t xb, ob;
    if (!bytes_of(M, K, (int64_t)esize(dt), &xb) || !bytes_of(M, N, (int64_t)esize(dt), &ob))
        return DN_ERR_INVALID_ARG;
    if (K % 8 || N % 8) return DN_ERR_UNSUPPORTED;
    if (!aligned(x, 16) || !aligned(h, 16) || !aligned(w->packed, 256)) return DN_ERR_MISALIGNED;
    const size_t pb = swiglu_packed_bytes(K, N, dt);
    if (overlaps(h, ob, x, xb) || overlaps(h, ob, w->packed, pb)) return DN_ERR_INVALID_ARG;
    if (((M + 15) / 16) * ((2 * N + 31) / 16) > kMaxGridX) return DN_ERR_UNSUPPORTED;
    return from_hip(dn::launch_swiglu_deferred(x, w->packed, M, K, N, dt, eps, 1, h, stream));
}

DN_API dn_status softmax_pv_deferred(const void* S, const void* V, int64_t BH, int64_t Lq, int64_t Lk, int64_t d,
                                     int causal, int dtype, void* out, hipStream_t stream) {
    if (!S || !V || !out || BH < 1 || Lq < 1 || Lk < 1 || d < 1 || !valid_dtype(dtype)) return DN_ERR_INVALID_ARG;
    if (causal != 0 && causal != 1) return DN_ERR_INVALID_ARG;
    if (causal && Lq != Lk) return DN_ERR_INVALID_ARG;
    size_t sb, vb, ob;
    int64_t bhlq;
    if (!bytes_of(BH, Lq, Lk * 2, &sb) || !bytes_of(BH, Lk, d * 2, &vb) || !bytes_of(BH, Lq, d * 2, &ob) ||
        __builtin_mul_overflow(BH, Lq, &bhlq))
        return DN_ERR_INVALID_ARG;
    if (dtype != DN_BF16 || (d != 64 && d != 128) || Lk % 8) return DN_ERR_UNSUPPORTED;
    if (Lq * Lk > (int64_t(1) << 31) || Lk * d * 2 >= (int64_t(1) << 32))
        return DN_ERR_UNSUPPORTED;  // one head's scores and values within 4 GiB
    if (!aligned(S, 16) || !aligned(V, 16) || !aligned(out, 16)) return DN_ERR_MISALIGNED;
    if (overlaps(out, ob, S, sb) || overlaps(out, ob, V, vb)) return DN_ERR_INVALID_ARG;
    if (BH * ((Lq + 255) / 256) > kMaxGridX) return DN_ERR_UNSUPPORTED;
    return from_hip(dn::launch_softmax_pv_deferred(S, V, BH, Lq, Lk, d, causal, out, stream));
}

// BH key/value heads, each read by `group` consecutive query heads (group = 1: one each).
static dn_status attention_grouped(const void* Q, const void* K, const void* V, int64_t BH, int64_t group,
                                   int64_t Lq, int64_t Lk, int64_t d, int causal, float scale, int dtype, void* out,
                                   hipStream_t stream) {
    if (!Q || !K || !V || !out || BH < 1 || group < 1 || Lq < 1 || Lk < 1 || d < 1 || !valid_dtype(dtype))
        return DN_ERR_INVALID_ARG;
    if (causal != 0 && causal != 1) return DN_ERR_INVALID_ARG;
    if (causal && Lq != Lk) return DN_ERR_INVALID_ARG;
    if (!isfinite(scale) || !(scale > 0.f)) return DN_ERR_INVALID_ARG;
    int64_t BHq;
    size_t qb, kb;
    if (__builtin_mul_overflow(BH, group, &BHq) || !bytes_of(BHq, Lq, d * 2, &qb) || !bytes_of(BH, Lk, d * 2, &kb))
        return DN_ERR_INVALID_ARG;
    const size_t ob = qb;
    if (dtype != DN_BF16 || (d != 64 && d != 128)) return DN_ERR_UNSUPPORTED;
    if (Lq * d * 2 >= (int64_t(1) << 31) || Lk * d * 2 >= (int64_t(1) << 31)) return DN_ERR_UNSUPPORTED;
    if (group > (int64_t(1) << 20)) return DN_ERR_UNSUPPORTED;
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(out, 16)) return DN_ERR_MISALIGNED;
    if (overlaps(out, ob, Q, qb) || overlaps(out, ob, K, kb) || overlaps(out, ob, V, kb)) return DN_ERR_INVALID_ARG;
    if (BHq * ((Lq + 255) / 256) > kMaxGridX) return DN_ERR_UNSUPPORTED;
    return from_hip(dn::launch_attention_deferred(Q, K, V, BHq, Lq, Lk, d, causal, scale, out, stream, (int)group));
}

DN_API dn_status attention_deferred(const void* Q, const void* K, const void* V, int64_t BH, int64_t Lq, int64_t Lk,
                                    int64_t d, int causal, float scale, int dtype, void* out, hipStream_t stream) {
    return attention_grouped(Q, K, V, BH, 1, Lq, Lk, d, causal, scale, dtype, out, stream);
}

DN_API dn_status attention_gqa_deferred(const void* Q, const void* K, const void* V, int64_t BH_kv, int64_t group,
                                        int64_t Lq, int64_t Lk, int64_t d, int causal, float scale, int dtype,
                                        void* out, hipStream_t stream) {
    return attention_grouped(Q, K, V, BH_kv, group, Lq, Lk, d, causal, scale, dtype, out, stream);
}

DN_API size_t attention_decode_workspace_bytes(int64_t BH, int64_t Lq, int64_t Lk, int64_t d) {
    size_t b;
    if (BH < 1 || Lq < 1 || Lq > 16 || Lk < 1 || (d != 64 && d != 128) || !bytes_of(BH, Lk, d * 2, &b))
        return 0;
    return dn::attention_decode_workspace_bytes(BH, Lq, Lk, d);
}

DN_API dn_status attention_decode_deferred(const void* Q, const void* K, const void* V, int64_t BH, int64_t Lq,
                                           int64_t Lk, int64_t d, float scale, int dtype, void* workspace,
                                           size_t workspace_bytes, void* out, hipStream_t stream) {
    if (!Q || !K || !V || !out || !workspace || BH < 1 || Lq < 1 || Lk < 1 || d < 1 || !valid_dtype(dtype))
        return DN_ERR_INVALID_ARG;
    if (!isfinite(scale) || !(scale > 0.f)) return DN_ERR_INVALID_ARG;
    size_t qb, kb;
    if (!bytes_of(BH, Lq, d * 2, &qb) || !bytes_of(BH, Lk, d * 2, &kb)) return DN_ERR_INVALID_ARG;
    if (dtype != DN_BF16 || (d != 64 && d != 128) || Lq > 16) return DN_ERR_UNSUPPORTED;
    if (Lk * d * 2 >= (int64_t(1) << 31)) return DN_ERR_UNSUPPORTED;
    // the least a call can work with, and what attention_decode_workspace_bytes asks for
    const size_t need = dn::attention_decode_least_bytes(BH, Lq, Lk, d);
    const size_t full = dn::attention_decode_workspace_bytes(BH, Lq, Lk, d);
    if (need == 0 || workspace_bytes < need) return DN_ERR_INVALID_ARG;
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(out, 16) || !aligned(workspace, 16))
        return DN_ERR_MISALIGNED;
    if (overlaps(out, qb, Q, qb) || overlaps(out, qb, K, kb) || overlaps(out, qb, V, kb) ||
        overlaps(workspace, need, Q, qb) || overlaps(workspace, need, K, kb) || overlaps(workspace, need, V, kb) ||
        overlaps(workspace, need, out, qb))
        return DN_ERR_INVALID_ARG;
    if (BH * 16 > kMaxGridX) return DN_ERR_UNSUPPORTED;  // grid: at most BH + 512 workgroups
    // no more than the least is used where the rest is missing or belongs to another argument
    const bool whole = workspace_bytes >= full && !overlaps(workspace, full, Q, qb) &&
                       !overlaps(workspace, full, K, kb) && !overlaps(workspace, full, V, kb) &&
                       !overlaps(workspace, full, out, qb);
    return from_hip(dn::launch_attention_decode(Q, K, V, BH, Lq, Lk, d, scale, workspace, whole ? full : need, out,
                                                stream));
}

DN_API dn_status attention_decode_deferred_noalloc(const void* Q, const void* K, const void* V, int64_t BH,
                                                   int64_t Lq, int64_t Lk, int64_t d, float scale, int dtype,
                                                   void* out, hipStream_t stream) {
    if (!Q || !K || !V || !out || BH < 1 || Lq < 1 || Lk < 1 || d < 1 || !valid_dtype(dtype))
        return DN_ERR_INVALID_ARG;
    if (!isfinite(scale) || !(scale > 0.f)) return DN_ERR_INVALID_ARG;
    size_t qb, kb;
    if (!bytes_of(BH, Lq, d * 2, &qb) || !bytes_of(BH, Lk, d * 2, &kb)) return DN_ERR_INVALID_ARG;
    if (dtype != DN_BF16 || (d != 64 && d != 128) || Lq > 16) return DN_ERR_UNSUPPORTED;
    if (Lk * d * 2 >= (int64_t(1) << 31)) return DN_ERR_UNSUPPORTED;
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(out, 16)) return DN_ERR_MISALIGNED;
    if (overlaps(out, qb, Q, qb) || overlaps(out, qb, K, kb) || overlaps(out, qb, V, kb)) return DN_ERR_INVALID_ARG;
    if (BH * 16 > kMaxGridX) return DN_ERR_UNSUPPORTED;
    if (dn::attention_decode_partials_bytes(BH, Lq, Lk, d) > dn::kDecodeScratchBytes) return DN_ERR_UNSUPPORTED;
    return from_hip(dn::launch_attention_decode_noalloc(Q, K, V, BH, Lq, Lk, d, scale, out, stream));
}

static dn_status row_norm(const void* x, const void* gamma, const void* beta, int64_t M, int64_t K, float eps,
                          int rms, int dtype, void* y, hipStream_t stream) {
    if (!x || !gamma || !y || M < 1 || K < 1 || !valid_dtype(dtype)) return DN_ERR_INVALID_ARG;
    if (!isfinite(eps) || eps < 0.f) return DN_ERR_INVALID_ARG;
    size_t xb;
    if (!bytes_of(M, K, (int64_t)esize(dtype), &xb)) return DN_ERR_INVALID_ARG;
    if (K % 8 || K > (dtype == DN_F32 ? dn::kMaxRowElemsF32 : dn::kMaxRowElemsBf16)) return DN_ERR_UNSUPPORTED;
    if (!aligned(x, 16) || !aligned(gamma, 16) || !aligned(beta, 16) || !aligned(y, 16)) return DN_ERR_MISALIGNED;
    const size_t es = esize(dtype);
    if (overlaps(y, xb, x, xb) || overlaps(y, xb, gamma, K * es) || overlaps(y, xb, beta, K * es))
        return DN_ERR_INVALID_ARG;
    if ((M + 3) / 4 > kMaxGridX) return DN_ERR_UNSUPPORTED;
    return from_hip(dn::launch_layernorm(x, gamma, beta, M, K, eps, rms, dtype, y, stream));
}

DN_API dn_status layernorm(const void* x, const void* gamma, const void* beta, int64_t M, int64_t K, float eps,
                           int dtype, void* y, hipStream_t stream) {
    return row_norm(x, gamma, beta, M, K, eps, 0, dtype, y, stream);
}

DN_API dn_status rmsnorm(const void* x, const void* gamma, int64_t M, int64_t K, float eps, int dtype, void* y,
                         hipStream_t stream) {
    return row_norm(x, gamma, nullptr, M, K, eps, 1, dtype, y, stream);
}

DN_API dn_status silu_mul(const void* g, const void* u, int64_t count, int dtype, void* h, hipStream_t stream) {
    if (!g || !u || !h || count < 1 || !valid_dtype(dtype)) return DN_ERR_INVALID_ARG;
    size_t b;
    if (!bytes_of(count, 1, (int64_t)esize(dtype), &b)) return DN_ERR_INVALID_ARG;
    if (count % 8) return DN_ERR_UNSUPPORTED;
    if (!aligned(g, 16) || !aligned(u, 16) || !aligned(h, 16)) return DN_ERR_MISALIGNED;
    if (overlaps(h, b, g, b) || overlaps(h, b, u, b)) return DN_ERR_INVALID_ARG;
    if ((count / 4 + 255) / 256 > kMaxGridX) return DN_ERR_UNSUPPORTED;
    return from_hip(dn::launch_silu_mul(g, u, count, dtype, h, stream));
}

DN_API dn_status softmax(const void* S, int64_t BH, int64_t Lq, int64_t Lk, int causal, int dtype, void* P,
                         hipStream_t stream) {
    if (!S || !P || BH < 1 || Lq < 1 || Lk < 1 || !valid_dtype(dtype)) return DN_ERR_INVALID_ARG;
    if (causal < 0 || causal > 2 || (causal && Lq != Lk)) return DN_ERR_INVALID_ARG;
    size_t sb;
    if (!bytes_of(BH, Lq, Lk * 2, &sb)) return DN_ERR_INVALID_ARG;
    if (dtype != DN_BF16 || Lk % 8 || Lk > dn::kMaxRowElemsBf16) return DN_ERR_UNSUPPORTED;
    if (!aligned(S, 16) || !aligned(P, 16)) return DN_ERR_MISALIGNED;
    if (overlaps(P, sb, S, sb)) return DN_ERR_INVALID_ARG;
    if ((BH * Lq + 3) / 4 > kMaxGridX) return DN_ERR_UNSUPPORTED;
    return from_hip(dn::launch_softmax(S, BH, Lq, Lk, causal, P, stream));
}

DN_API dn_status gemm(const void* A, const void* B, const void* bias, int64_t batch, int64_t M, int64_t K, int64_t N,
                      int b_layout, int a_causal, int dtype, void* C, hipStream_t stream) {
    if (!A || !B || !C || batch < 1 || M < 1 || K < 1 || N < 1 || !valid_dtype(dtype)) return DN_ERR_INVALID_ARG;
    if (b_layout < 0 || b_layout > 2 || (a_causal != 0 && a_causal != 1)) return DN_ERR_INVALID_ARG;
    if (a_causal && M != K) return DN_ERR_INVALID_ARG;
    if (b_layout == 2 && batch != 1) return DN_ERR_INVALID_ARG;
    const int64_t es = (int64_t)esize(dtype);
    size_t ab, bb, cb, t;
    if (!bytes_of(batch, M, K * es, &ab) || !bytes_of(batch, K, N * es, &bb) || !bytes_of(batch, M, N * es, &cb) ||
        !bytes_of(M, K, 1, &t) || !bytes_of(K, N, 1, &t))
        return DN_ERR_INVALID_ARG;
    if (b_layout == 2) bb = ln_linear_packed_bytes(K, N, dtype);
    if (K % 8 || N % 8) return DN_ERR_UNSUPPORTED;
    if (dtype == DN_F32 && (b_layout == 0 || a_causal)) return DN_ERR_UNSUPPORTED;
    if (a_causal && b_layout == 2) return DN_ERR_UNSUPPORTED;
    if (batch > kMaxBatch) return DN_ERR_UNSUPPORTED;
    if (!aligned(A, 16) || !aligned(B, b_layout == 2 ? 256 : 16) || !aligned(bias, 16) || !aligned(C, 16))
        return DN_ERR_MISALIGNED;
    if (overlaps(C, cb, A, ab) || overlaps(C, cb, B, bb) || overlaps(C, cb, bias, (size_t)(N * es)))
        return DN_ERR_INVALID_ARG;
    if (((M + 31) / 32) * ((N + 63) / 64) > kMaxGridX) return DN_ERR_UNSUPPORTED;
    return from_hip(dn::launch_gemm(A, B, bias, batch, M, K, N, b_layout, a_causal, dtype, C, stream));
}

// ------------------------------------------------------------------- rotary positions, paged cache
constexpr int64_t kMaxThreads = 0xffffffff;  // of a launch, as HIP counts them

// What a strided [T][width] array spans, from its first to past its last element.
static bool span_of(int64_t T, int64_t stride, int64_t width, int64_t es, size_t* out) {
    size_t all, last;
    if (!bytes_of(T - 1 > 0 ? T - 1 : 1, stride, es, &all) || !bytes_of(width, es, 1, &last)) return false;
    if (T == 1) all = 0;
    return !__builtin_add_overflow(all, last, out);
}

DN_API dn_status rotary_table(const double* inv_freq, int64_t rot, int64_t positions, double amplitude, float* table,
                              hipStream_t stream) {
    if (!inv_freq || !table || rot < 1 || positions < 1 || !isfinite(amplitude)) return DN_ERR_INVALID_ARG;
    size_t tb;
    if (!bytes_of(positions, rot, 4, &tb)) return DN_ERR_INVALID_ARG;
    if (rot % 16) return DN_ERR_UNSUPPORTED;
    if (!aligned(inv_freq, 8) || !aligned(table, 16)) return DN_ERR_MISALIGNED;
    if (overlaps(table, tb, inv_freq, (size_t)rot * 4)) return DN_ERR_INVALID_ARG;
    if (positions > INT32_MAX || positions * (rot / 2) > kMaxThreads - 255) return DN_ERR_UNSUPPORTED;
    return from_hip(dn::launch_rotary_table(inv_freq, rot, positions, amplitude, table, stream));
}

DN_API dn_status rotary_apply(const void* x, int64_t x_stride, const int32_t* positions, const float* table,
                              int64_t table_rows, int64_t T, int64_t H, int64_t d, int64_t rot, int interleaved,
                              int inverse, int dtype, void* out, int64_t out_stride, hipStream_t stream) {
    if (!x || !positions || !table || !out || table_rows < 1 || T < 1 || H < 1 || d < 1 || rot < 1 || rot > d ||
        !valid_dtype(dtype) || (interleaved != 0 && interleaved != 1) || (inverse != 0 && inverse != 1))
        return DN_ERR_INVALID_ARG;
    const int64_t es = (int64_t)esize(dtype);
    size_t hd, xb, ob, tb;
    if (!bytes_of(H, d, es, &hd) || x_stride < H * d || out_stride < H * d || !span_of(T, x_stride, H * d, es, &xb) ||
        !span_of(T, out_stride, H * d, es, &ob) || !bytes_of(table_rows, rot, 4, &tb))
        return DN_ERR_INVALID_ARG;
    if (d % 16 || rot % 16 || x_stride * es % 16 || out_stride * es % 16) return DN_ERR_UNSUPPORTED;
    if (!aligned(x, 16) || !aligned(out, 16) || !aligned(table, 16) || !aligned(positions, 4)) return DN_ERR_MISALIGNED;
    const bool in_place = out == x && out_stride == x_stride;
    if ((!in_place && overlaps(out, ob, x, xb)) || overlaps(out, ob, table, tb) ||
        overlaps(out, ob, positions, (size_t)T * 4))
        return DN_ERR_INVALID_ARG;
    const int64_t items = H * d / (dtype == DN_F32 ? 8 : 16);
    if (items > INT32_MAX || T > INT32_MAX || T > (kMaxThreads - 255) / items) return DN_ERR_UNSUPPORTED;
    return from_hip(dn::launch_rotary(x, x_stride, positions, table, table_rows, T, H, d, rot, interleaved, inverse,
                                      dtype, out, out_stride, stream));
}

static bool valid_kv(int64_t pages, int64_t heads, int64_t d, int format, size_t* bytes) {
    int64_t blocks, all;
    if (pages < 1 || heads < 1 || (d != 64 && d != 128) || (format != DN_KV_BF16 && format != DN_KV_FP8)) return false;
    if (pages > INT32_MAX / DN_KV_PAGE || heads > INT32_MAX || __builtin_mul_overflow(pages, heads, &blocks) ||
        __builtin_mul_overflow(blocks, (int64_t)dn::kv_block_bytes(d, format), &all))
        return false;
    *bytes = (size_t)all;
    return true;
}

DN_API size_t kv_cache_bytes(int64_t pages, int64_t heads, int64_t d, int format) {
    size_t b;
    return valid_kv(pages, heads, d, format, &b) ? b : 0;
}

DN_API dn_status kv_cache_describe(void* data, size_t bytes, int64_t pages, int64_t heads, int64_t d, int format,
                                   kv_cache* out) {
    if (!data || !out || pages < 1 || heads < 1 || d < 1 || (format != DN_KV_BF16 && format != DN_KV_FP8))
        return DN_ERR_INVALID_ARG;
    size_t need;
    if (!valid_kv(pages, heads, d, format, &need)) return DN_ERR_UNSUPPORTED;
    if (bytes < need) return DN_ERR_INVALID_ARG;
    if (!aligned(data, 256)) return DN_ERR_MISALIGNED;
    out->pages = pages;
    out->heads = heads;
    out->d = d;
    out->format = format;
    out->layout_version = DN_KV_LAYOUT_VERSION;
    out->data = data;
    return DN_OK;
}

// A described cache; its bytes.
static bool described(const kv_cache* c, size_t* bytes) {
    return c && c->data && c->layout_version == DN_KV_LAYOUT_VERSION &&
           valid_kv(c->pages, c->heads, c->d, c->format, bytes);
}
static dn::KvPool pool_of(const kv_cache* c) { return dn::KvPool{c->pages, c->heads, c->d, c->format, c->data}; }

DN_API dn_status kv_cache_append(const kv_cache* cache, const void* qkv, int64_t stride, const int32_t* slots,
                                 const int32_t* positions, const float* table, int64_t table_rows, int64_t rot,
                                 int interleaved, int64_t T, int64_t q_heads, int dtype, void* q_out,
                                 hipStream_t stream) {
    size_t cb, xb, qb = 0, tb = 0;
    if (!described(cache, &cb) || !qkv || !slots || T < 1 || q_heads < 0 || q_heads > INT32_MAX || !valid_dtype(dtype) ||
        (q_heads > 0) != (q_out != nullptr) || rot < 0 || rot > cache->d || (interleaved != 0 && interleaved != 1))
        return DN_ERR_INVALID_ARG;
    if (q_heads % cache->heads) return DN_ERR_INVALID_ARG;
    if (rot > 0 && (!positions || !table || table_rows < 1 || !bytes_of(table_rows, rot, 4, &tb)))
        return DN_ERR_INVALID_ARG;
    const int64_t width = (q_heads + 2 * cache->heads) * cache->d;
    if (stride < width || !span_of(T, stride, width, 2, &xb) || (q_heads && !bytes_of(T, q_heads, cache->d * 2, &qb)))
        return DN_ERR_INVALID_ARG;
    if (dtype != DN_BF16 || rot % 16 || stride % 8) return DN_ERR_UNSUPPORTED;
    if (!aligned(qkv, 16) || !aligned(q_out, 16) || !aligned(cache->data, 256) || !aligned(slots, 4) ||
        (rot > 0 && (!aligned(table, 16) || !aligned(positions, 4))))
        return DN_ERR_MISALIGNED;
    const size_t ib = (size_t)T * 4;
    const void* ins[4] = {qkv, slots, rot > 0 ? positions : nullptr, rot > 0 ? table : nullptr};
    const size_t in_bytes[4] = {xb, ib, ib, tb};
    for (int i = 0; i < 4; ++i)
        if (overlaps(cache->data, cb, ins[i], in_bytes[i]) || overlaps(q_out, qb, ins[i], in_bytes[i]))
            return DN_ERR_INVALID_ARG;
    if (overlaps(cache->data, cb, q_out, qb)) return DN_ERR_INVALID_ARG;
    // a workgroup's items fit 31 bits
    if (width > (int64_t(1) << 24) || T > INT32_MAX / 4) return DN_ERR_UNSUPPORTED;
    const int64_t tile = dn::append_tile(T, cache->heads, q_heads / cache->heads, cache->d);
    if ((T + tile - 1) / tile > kMaxThreads / 256 / cache->heads) return DN_ERR_UNSUPPORTED;
    return from_hip(dn::launch_kv_append(qkv, stride, slots, positions, table, table_rows, rot, interleaved, T, q_heads,
                                         pool_of(cache), q_out, stream));
}

DN_API dn_status kv_cache_read(const kv_cache* cache, const int32_t* slots, int64_t T, int dtype, void* K, void* V,
                               hipStream_t stream) {
    size_t cb, ob;
    if (!described(cache, &cb) || !slots || !K || !V || T < 1 || !valid_dtype(dtype) ||
        !bytes_of(T, cache->heads, cache->d * 2, &ob))
        return DN_ERR_INVALID_ARG;
    if (dtype != DN_BF16) return DN_ERR_UNSUPPORTED;
    if (!aligned(K, 16) || !aligned(V, 16) || !aligned(cache->data, 256) || !aligned(slots, 4)) return DN_ERR_MISALIGNED;
    const size_t ib = (size_t)T * 4;
    if (overlaps(K, ob, V, ob) || overlaps(K, ob, cache->data, cb) || overlaps(V, ob, cache->data, cb) ||
        overlaps(K, ob, slots, ib) || overlaps(V, ob, slots, ib))
        return DN_ERR_INVALID_ARG;
    // a workgroup takes 16 tokens of a head's K or 56 of its V at least
    if (T > INT32_MAX / 4 || (T + 15) / 16 + (T + 55) / 56 > kMaxThreads / 256 / cache->heads) return DN_ERR_UNSUPPORTED;
    return from_hip(dn::launch_kv_read(pool_of(cache), slots, T, K, V, stream));
}

// Sizes for which every count of the attention kernels fits its type, and every launch the device.
static bool attention_cache_sizes(int64_t T, int64_t B, int64_t q_heads, int64_t heads, int64_t d, int64_t width,
                                  int64_t prefix) {
    constexpr int64_t k31 = INT32_MAX;
    const bool counts =
        T <= k31 / 128 && B <= (int64_t(1) << 20) && q_heads <= (int64_t(1) << 16) && T * q_heads <= k31 / 2 &&
        width <= k31 / DN_KV_PAGE && prefix <= k31 - DN_KV_PAGE && (T + B) * heads <= k31 / 4 &&
        B * width < (int64_t(1) << 40) && (d == 64 || d == 128) &&
        // the weight of all work dealt in runs
        (T * q_heads / 256 + B * heads) * (q_heads / heads) <= (int64_t(1) << 61) / (width * DN_KV_PAGE + 256);
    if (!counts) return false;
    const dn::CacheWorkspace w =
        dn::cache_workspace(T, B, heads, q_heads / heads, d, width, (prefix + DN_KV_PAGE - 1) / DN_KV_PAGE);
    const int64_t own = w.own.grid * (w.own.rows == 256 ? 512 : 256), prefixes = w.prefix.grid * (w.prefix.rows == 256 ? 512 : 256);
    // tiles of 16 rows share a launch with the prefix's; the merge takes d / 16 threads a row, d / 8 behind a prefix
    return own + (w.own.rows == 16 ? prefixes : 0) <= kMaxThreads && prefixes <= kMaxThreads &&
           (w.own.slots == 0 || T * q_heads <= (kMaxThreads - 255) / (d / (prefix ? 8 : 16)));
}

DN_API size_t attention_cache_workspace_bytes(int64_t T, int64_t B, int64_t q_heads, int64_t heads, int64_t d,
                                              int64_t table_width, int64_t prefix_len) {
    if (T < 1 || B < 1 || heads < 1 || q_heads < 1 || q_heads % heads || table_width < 1 || prefix_len < 0 ||
        !attention_cache_sizes(T, B, q_heads, heads, d, table_width, prefix_len))
        return 0;
    return dn::cache_workspace(T, B, heads, q_heads / heads, d, table_width, (prefix_len + DN_KV_PAGE - 1) / DN_KV_PAGE)
        .total;
}

static dn_status attention_cache(const void* Q, int64_t q_stride, int64_t T, int64_t q_heads, const kv_cache* cache,
                                 const int32_t* prefix_table, int64_t prefix, const int32_t* table, int64_t width,
                                 const int32_t* q_start, const int32_t* kv_len, int64_t B, float scale, int dtype,
                                 void* workspace, size_t workspace_bytes, void* out, hipStream_t stream) {
    size_t cb, qb, ob, tb;
    if (!described(cache, &cb) || !Q || !table || !q_start || !kv_len || !workspace || !out || T < 1 || B < 1 ||
        q_heads < 1 || q_heads % cache->heads || width < 1 || !valid_dtype(dtype) || !isfinite(scale) || !(scale > 0.f))
        return DN_ERR_INVALID_ARG;
    if (!bytes_of(B, width, 4, &tb)) return DN_ERR_INVALID_ARG;
    if (!attention_cache_sizes(T, B, q_heads, cache->heads, cache->d, width, prefix)) return DN_ERR_UNSUPPORTED;
    const int64_t row = q_heads * cache->d;
    if (q_stride < row || !span_of(T, q_stride, row, 2, &qb) || !bytes_of(T, row, 2, &ob)) return DN_ERR_INVALID_ARG;
    if (dtype != DN_BF16 || q_stride % 8) return DN_ERR_UNSUPPORTED;
    const size_t need = attention_cache_workspace_bytes(T, B, q_heads, cache->heads, cache->d, width, prefix);
    if (workspace_bytes < need) return DN_ERR_INVALID_ARG;
    if (!aligned(Q, 16) || !aligned(out, 16) || !aligned(cache->data, 256) || !aligned(workspace, 256) ||
        !aligned(table, 4) || !aligned(q_start, 4) || !aligned(kv_len, 4) || !aligned(prefix_table, 4))
        return DN_ERR_MISALIGNED;
    const void* ins[6] = {Q, cache->data, table, q_start, kv_len, prefix_table};
    const size_t in_bytes[6] = {qb, cb, tb, (size_t)(B + 1) * 4, (size_t)B * 4, (size_t)((prefix + 63) / 64) * 4};
    for (int i = 0; i < 6; ++i)
        if (overlaps(out, ob, ins[i], in_bytes[i]) || overlaps(workspace, need, ins[i], in_bytes[i]))
            return DN_ERR_INVALID_ARG;
    if (overlaps(workspace, need, out, ob)) return DN_ERR_INVALID_ARG;
    return from_hip(dn::launch_attention_cache(
        dn::AttentionCacheCall{Q, q_stride, T, q_heads, pool_of(cache), prefix_table, prefix, table, width, q_start, kv_len,
                               B, scale, workspace, out},
        stream));
}

DN_API dn_status attention_cache_deferred(const void* Q, int64_t q_stride, int64_t T, int64_t q_heads,
                                          const kv_cache* cache, const int32_t* block_table, int64_t table_width,
                                          const int32_t* q_start, const int32_t* kv_len, int64_t B, float scale,
                                          int dtype, void* workspace, size_t workspace_bytes, void* out,
                                          hipStream_t stream) {
    return attention_cache(Q, q_stride, T, q_heads, cache, nullptr, 0, block_table, table_width, q_start, kv_len, B, scale,
                           dtype, workspace, workspace_bytes, out, stream);
}

DN_API dn_status attention_shared_prefix_deferred(const void* Q, int64_t q_stride, int64_t T, int64_t q_heads,
                                                  const kv_cache* cache, const int32_t* prefix_table,
                                                  int64_t prefix_len, const int32_t* block_table, int64_t table_width,
                                                  const int32_t* q_start, const int32_t* kv_len, int64_t B, float scale,
                                                  int dtype, void* workspace, size_t workspace_bytes, void* out,
                                                  hipStream_t stream) {
    if (!prefix_table || prefix_len < 1) return DN_ERR_INVALID_ARG;
    return attention_cache(Q, q_stride, T, q_heads, cache, prefix_table, prefix_len, block_table, table_width, q_start,
                           kv_len, B, scale, dtype, workspace, workspace_bytes, out, stream);
}

}  // extern "C"
