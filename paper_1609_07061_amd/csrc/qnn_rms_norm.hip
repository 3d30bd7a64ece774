// Root-mean-square norm of the residual stream, with the residual's addition before it and int8 codes with one scale a row behind it (what
// qnn_int8_gemm takes), and its gradient (straight through the quantizer, as Sec. 2.3 does for the sign).
//
// Forward: h = x + residual, r = 1 / sqrt(mean h^2 + eps), y = h r gamma, codes and scale of y (qnn_rows.h).  r is one positive number a row, so
// max |y| = r max |h gamma|: the sum and the maximum come from ONE pass over the row, which stays in registers, and the codes need no r at all.
// The norm and the codes take h in fp32; the sum that is written is rounded once.
// Bound by memory: 2 reads and a write of a 16-bit float and a write of a byte for each value (10000 x 4096 bf16 with a residual, 287 MB: 48.8 us, 5.9 TB/s;
// one row: 4.2 us, a launch).
#include <type_traits>

#include "qnn_rows.h"

namespace qnn {
namespace {

using namespace rows;

template <typename T, bool kOnce>
struct NormSource {
    struct Kept {
        float h[kVec];
    };
    const T *x, *residual;
    T *sum;
    const void *gamma;
    int64_t ldx, ldr, lds;
    bool gamma_f32;
    float eps;
    template <bool kShort>
    __device__ __forceinline__ void load(int64_t row, const Window &w, int64_t K, float (&v)[kVec], Kept &kept) const {
        const Raw<T> a = load_raw<kOnce, kShort>(x + row * ldx, w, K);
        float g[kVec];
        load_either<kShort, T>(gamma, gamma_f32, w, K, g);
        if (residual) {
            const Raw<T> b = load_raw<kOnce, kShort>(residual + row * ldr, w, K);
#pragma unroll
            for (int i = 0; i < kVec; ++i) kept.h[i] = (float)a.e[i] + (float)b.e[i];
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) kept.h[i] = (float)a.e[i];
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = kept.h[i] * g[i];
    }
    __device__ __forceinline__ float add(const Kept &kept, int i, float sum) const { return __fmaf_rn(kept.h[i], kept.h[i], sum); }
    __device__ __forceinline__ float factor(float total, int64_t K) const { return norm_factor(total, K, eps); }
    template <bool kShort>
    __device__ __forceinline__ void keep(int64_t row, const Window &w, int64_t K, const Kept &kept) const {
        if (sum) store_values<kOnce, kShort>(sum + row * lds, w, K, kept.h);
    }
};

// Gradient.  With g the gradient at y and z one that reaches h by another way (the residual path):
//   gh = r (gamma g - h r^2 mean(gamma g h)) + z,   ggamma = sum over the rows of g h r.
// A workgroup takes kGroups rows at a time, every gridDim-th such group, keeps its lanes' part of ggamma in registers over all of them and writes it once;
// the second kernel adds these partial sums in a fixed order.  Up to kParts of them, so that they are a small part of what is moved.  (10000 x 4096 bf16
// with a residual's gradient, 328 MB: 58.6 us, 5.6 TB/s, and 4.1 for the parts; one row at a time took 70.9 where two took 61.0, and with the next row's loads
// sent ahead 68.3 and 71.5: more registers, fewer waves.)
constexpr int kParts = 512;

template <typename T>
struct NormGradArgs {
    const T *grad, *h, *grad_sum;
    T *out;
    const void *gamma;
    int64_t ldg, ldh, ldz, ldo;
    bool gamma_f32;
    float eps;
    int64_t n_rows, K;
    float *parts;
};

// rows that a workgroup takes at a time, and its threads
constexpr int groups_of(int threads) { return threads == 64 ? 4 : (threads == 256 ? 2 : 1); }

template <typename T, int kThreads, int kPer, bool kOnce, bool kShort>
__global__ __launch_bounds__(kThreads *groups_of(kThreads)) void rms_norm_backward_kernel(const NormGradArgs<T> a) {
    constexpr int kGroups = groups_of(kThreads);
    __shared__ TwoSums shared[kGroups][2][kThreads / 64];
    __shared__ float joined[kGroups > 1 ? kThreads * kPer * kVec : 1];
    const int lane = threadIdx.x % kThreads, group = threadIdx.x / kThreads;
    float gamma[kPer][kVec], acc[kPer][kVec];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) acc[i][e] = 0.0f;
        load_either<kShort, T>(a.gamma, a.gamma_f32, Window((int64_t)(i * kThreads + lane) * kVec, a.K), a.K, gamma[i]);
    }
    struct Row {
        Raw<T> h[kPer], g[kPer], z[kPer];
    };
    const int64_t step = (int64_t)gridDim.x * kGroups;
    auto load = [&](int64_t row, Row &v) __attribute__((always_inline)) {
        if (row >= a.n_rows) return;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const Window w((int64_t)(i * kThreads + lane) * kVec, a.K);
            v.h[i] = load_raw<kOnce, kShort>(a.h + row * a.ldh, w, a.K);
            v.g[i] = load_raw<kOnce, kShort>(a.grad + row * a.ldg, w, a.K);
            if (a.grad_sum) v.z[i] = load_raw<kOnce, kShort>(a.grad_sum + row * a.ldz, w, a.K);
        }
    };
    int turn = 0;
    auto finish = [&](int64_t row, const Row &v) __attribute__((always_inline)) {
        TwoSums s = {0.0f, 0.0f};
        if (row < a.n_rows) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const Window w((int64_t)(i * kThreads + lane) * kVec, a.K);
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    const float hv = e >= w.skip && (!kShort || w.from + e < a.K) ? (float)v.h[i].e[e] : 0.0f;
                    s.a = __fmaf_rn(hv, hv, s.a);
                    s.b = __fmaf_rn(gamma[i][e] * (float)v.g[i].e[e], hv, s.b);
                }
            }
        }
        s = across<kThreads>(s, TwoSums::join, shared[group], turn);
        turn ^= 1;
        if (row >= a.n_rows) return;
        const float r = norm_factor(s.a, a.K, a.eps), c = r * r * (s.b / (float)a.K);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int64_t k = (int64_t)(i * kThreads + lane) * kVec;
            if (k < a.K) {
                float o[kVec];
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    const float hv = (float)v.h[i].e[e], gv = (float)v.g[i].e[e];
                    o[e] = r * __fmaf_rn(-hv, c, gamma[i][e] * gv);
                    if (a.grad_sum) o[e] += (float)v.z[i].e[e];
                    acc[i][e] = __fmaf_rn(gv, hv * r, acc[i][e]);
                }
                store_values<kOnce, kShort>(a.out + row * a.ldo, Window(k, a.K), a.K, o);
            }
        }
    };
    // (every group of a workgroup makes the same number of turns, with a row or without)
    const int64_t first = (int64_t)blockIdx.x * kGroups;
    Row v;
    for (int64_t row = first; row < a.n_rows; row += step) {
        load(row + group, v);
        finish(row + group, v);
    }
    float *part = a.parts + (int64_t)blockIdx.x * a.K;
    if constexpr (kGroups == 1) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int64_t k = (int64_t)(i * kThreads + lane) * kVec;
            if (k < a.K) store_values<false, kShort>(part, Window(k, a.K), a.K, acc[i]);
        }
    } else {  // the groups' sums, one after the other
        for (int w = 0; w < kGroups; ++w) {
            if (group == w) {
#pragma unroll
                for (int i = 0; i < kPer; ++i)
#pragma unroll
                    for (int e = 0; e < kVec; ++e) {
                        float &to = joined[(i * kVec + e) * kThreads + lane];  // (neighbouring lanes, neighbouring banks)
                        to = w == 0 ? acc[i][e] : to + acc[i][e];
                    }
            }
            __syncthreads();
        }
        for (int k = threadIdx.x; k < a.K; k += blockDim.x) {
            const int v = k / kVec, e = k - (int)Window((int64_t)v * kVec, a.K).from;  // value k: lane, and place in its window
            part[k] = joined[((v / kThreads) * kVec + e) * kThreads + v % kThreads];
        }
    }
}

constexpr int64_t kWidest = 2048 * kVec;  // of the gradient, whose rows stay in registers
int64_t parts_of(int64_t rows) { return rows < kParts ? rows : kParts; }

template <typename T, int kThreads, int kPer, bool kShort = false>
int launch_backward(const NormGradArgs<T> &a, float *grad_gamma, hipStream_t s) {
    const int64_t blocks = ceil_div(a.n_rows, groups_of(kThreads)), parts = blocks < kParts ? blocks : kParts;
    const bool once = beyond_caches((a.grad_sum ? 4.0 : 3.0) * sizeof(T) * (double)a.n_rows * (double)a.K);
    auto kernel = once ? rms_norm_backward_kernel<T, kThreads, kPer, !kShort, kShort> : rms_norm_backward_kernel<T, kThreads, kPer, false, kShort>;
    if (int rc = QNN_LAUNCH("rms_norm_backward", kernel, dim3((unsigned)parts), dim3(kThreads * groups_of(kThreads)), 0, s, a)) return rc;
    const AddParts all = {a.parts, (int32_t)parts, grad_gamma};
    return QNN_LAUNCH("rms_norm_backward", add_parts_kernel, dim3((unsigned)ceil_div(a.K, 32)), dim3(1024), 0, s, all, all, a.K);
}

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" int qnn_rms_norm_quant(const void *x, int64_t ldx, const void *residual, int64_t ld_residual, int type, const void *gamma, int gamma_type,
                                  float eps, int64_t rows, int64_t K, void *sum, int64_t ld_sum, int8_t *codes, int64_t ld_codes, float *scale,
                                  void *stream) {
    if (rows < 0 || K < 1) return fail(QNN_ERR_SHAPE, "rms_norm_quant: rows = %lld, K = %lld", (long long)rows, (long long)K);
    if (!rows::known_type(type) || (gamma_type != QNN_F32 && gamma_type != type))
        return fail(QNN_ERR_SHAPE, "rms_norm_quant: types %d, %d (gamma: float32, or as x)", type, gamma_type);
    if (!(eps >= 0.0f) || eps > 3.0e38f) return fail(QNN_ERR_SHAPE, "rms_norm_quant: eps = %g", (double)eps);
    if (ldx < K || (residual && ld_residual < K) || (sum && ld_sum < K) || ld_codes < K)
        return fail(QNN_ERR_SHAPE, "rms_norm_quant: leading dimension too small");
    if (rows == 0) return QNN_OK;
    if (!x || !gamma || !codes || !scale) return fail(QNN_ERR_NULL, "rms_norm_quant: NULL pointer");
    const int w = rows::value_bytes(type);
    if (!rows::aligned_to(x, w) || !rows::aligned_to(residual, w) || !rows::aligned_to(sum, w) || !rows::aligned_to(gamma, rows::value_bytes(gamma_type)) ||
        !rows::aligned_to(scale, 4))
        return fail(QNN_ERR_ALIGN, "rms_norm_quant: pointer not aligned to its type");
    return rows::with_type(type, [&](auto tag) {
        typedef decltype(tag) T;
        auto launch = [&](auto once) {
            const NormSource<T, decltype(once)::value> src = {static_cast<const T *>(x), static_cast<const T *>(residual), static_cast<T *>(sum), gamma, ldx,
                                                              ld_residual, ld_sum, gamma_type == QNN_F32, eps};
            return rows::launch_quant_rows("rms_norm_quant", src, rows, K, codes, ld_codes, scale, static_cast<hipStream_t>(stream));
        };
        const double bytes = (w * (1.0 + (residual ? 1.0 : 0.0) + (sum ? 1.0 : 0.0)) + 1.0) * (double)rows * (double)K;
        return rows::beyond_caches(bytes) ? launch(std::true_type{}) : launch(std::false_type{});
    });
}

extern "C" size_t qnn_rms_norm_backward_workspace_bytes(int64_t rows, int64_t K) {
    return rows < 1 || K < 1 || K > kWidest ? 0 : (size_t)parts_of(rows) * (size_t)K * 4;
}

extern "C" int qnn_rms_norm_backward(const void *grad, int64_t ld_grad, const void *h, int64_t ld_h, const void *grad_sum, int64_t ld_grad_sum, int type,
                                     const void *gamma, int gamma_type, float eps, int64_t rows, int64_t K, void *grad_h, int64_t ld_grad_h,
                                     float *grad_gamma, void *workspace, size_t workspace_bytes, void *stream) {
    if (rows < 1 || K < 1) return fail(QNN_ERR_SHAPE, "rms_norm_backward: rows = %lld, K = %lld", (long long)rows, (long long)K);
    if (!rows::known_type(type) || (gamma_type != QNN_F32 && gamma_type != type))
        return fail(QNN_ERR_SHAPE, "rms_norm_backward: types %d, %d (gamma: float32, or as h)", type, gamma_type);
    if (!(eps >= 0.0f) || eps > 3.0e38f) return fail(QNN_ERR_SHAPE, "rms_norm_backward: eps = %g", (double)eps);
    if (ld_grad < K || ld_h < K || (grad_sum && ld_grad_sum < K) || ld_grad_h < K)
        return fail(QNN_ERR_SHAPE, "rms_norm_backward: leading dimension too small");
    if (K > kWidest) return fail(QNN_ERR_UNSUPPORTED, "rms_norm_backward: K = %lld, at most %lld", (long long)K, (long long)kWidest);
    if (!grad || !h || !gamma || !grad_h || !grad_gamma) return fail(QNN_ERR_NULL, "rms_norm_backward: NULL pointer");
    const int w = rows::value_bytes(type);
    if (!rows::aligned_to(grad, w) || !rows::aligned_to(h, w) || !rows::aligned_to(grad_sum, w) || !rows::aligned_to(grad_h, w) ||
        !rows::aligned_to(gamma, rows::value_bytes(gamma_type)) || !rows::aligned_to(grad_gamma, 4))
        return fail(QNN_ERR_ALIGN, "rms_norm_backward: pointer not aligned to its type");
    const size_t need = qnn_rms_norm_backward_workspace_bytes(rows, K);
    if (!workspace || !rows::aligned_to(workspace, 256) || workspace_bytes < need)
        return fail(QNN_ERR_WORKSPACE, "rms_norm_backward: workspace NULL, misaligned or smaller than %zu bytes", need);
    return rows::with_type(type, [&](auto tag) {
        typedef decltype(tag) T;
        const NormGradArgs<T> a = {static_cast<const T *>(grad), static_cast<const T *>(h), static_cast<const T *>(grad_sum), static_cast<T *>(grad_h),
                                   gamma, ld_grad, ld_h, ld_grad_sum, ld_grad_h, gamma_type == QNN_F32, eps, rows, K, static_cast<float *>(workspace)};
        hipStream_t s = static_cast<hipStream_t>(stream);
        if (K < kVec) return launch_backward<T, 64, 1, true>(a, grad_gamma, s);
        if (K <= 64 * kVec) return launch_backward<T, 64, 1>(a, grad_gamma, s);
        if (K <= 128 * kVec) return launch_backward<T, 64, 2>(a, grad_gamma, s);
        if (K <= 256 * kVec) return launch_backward<T, 256, 1>(a, grad_gamma, s);
        if (K <= 512 * kVec) return launch_backward<T, 256, 2>(a, grad_gamma, s);
        if (K <= 1024 * kVec) return launch_backward<T, 512, 2>(a, grad_gamma, s);
        return launch_backward<T, 512, 4>(a, grad_gamma, s);
    });
}
