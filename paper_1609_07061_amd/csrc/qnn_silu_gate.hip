// Gated activation between the two products of a feed-forward block, y = up * gate / (1 + exp(-gate)), with int8 codes and one scale a row behind it
// (what qnn_int8_gemm takes), and its gradient (straight through the quantizer, as Sec. 2.3 does for the sign).
// Bound by memory: 2 reads of a 16-bit float and a write of a byte for each value (10000 x 4096 bf16, 205 MB: 35.6 us, 5.7 TB/s); gradient: 3 reads and 2
// writes (2240 x 2501 fp16, 56 MB: 10.8 us, 5.2 TB/s).
#include <type_traits>

#include "qnn_rows.h"

namespace qnn {
namespace {

using namespace rows;

template <typename T, bool kOnce>
struct GateSource {
    struct Kept {};
    const T *gate, *up;
    int64_t ld_gate, ld_up;
    template <bool kShort>
    __device__ __forceinline__ void load(int64_t row, const Window &w, int64_t K, float (&v)[kVec], Kept &) const {
        const Raw<T> a = load_raw<kOnce, kShort>(gate + row * ld_gate, w, K), b = load_raw<kOnce, kShort>(up + row * ld_up, w, K);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = silu((float)a.e[i]) * (float)b.e[i];
    }
    __device__ __forceinline__ float add(const Kept &, int, float sum) const { return sum; }
    __device__ __forceinline__ float factor(float, int64_t) const { return 1.0f; }
    template <bool kShort>
    __device__ __forceinline__ void keep(int64_t, const Window &, int64_t, const Kept &) const {}
};

// With s = 1 / (1 + exp(-gate)): ggate = g up s (1 + gate (1 - s)), gup = g gate s
template <typename T, bool kOnce, bool kShort>
__global__ __launch_bounds__(256) void silu_gate_backward_kernel(const T *grad, int64_t ldg, const T *gate, int64_t ld_gate, const T *up, int64_t ld_up,
                                                                 int64_t n_rows, int64_t F, int64_t groups, T *grad_gate, int64_t ld_ggate, T *grad_up,
                                                                 int64_t ld_gup) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n_rows * groups; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / groups;
        const Window w((i - row * groups) * kVec, F);
        const Raw<T> a = load_raw<kOnce, kShort>(gate + row * ld_gate, w, F), b = load_raw<kOnce, kShort>(up + row * ld_up, w, F),
                     c = load_raw<kOnce, kShort>(grad + row * ldg, w, F);
        float p[kVec], q[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            const float x = (float)a.e[e], s = sigmoid(x), g = (float)c.e[e];
            p[e] = g * (float)b.e[e] * s * __fmaf_rn(x, 1.0f - s, 1.0f);
            q[e] = g * x * s;
        }
        store_values<kOnce, kShort>(grad_gate + row * ld_ggate, w, F, p);
        store_values<kOnce, kShort>(grad_up + row * ld_gup, w, F, q);
    }
}

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" int qnn_silu_gate_quant(const void *gate, int64_t ld_gate, const void *up, int64_t ld_up, int type, int64_t rows, int64_t F, int8_t *codes,
                                   int64_t ld_codes, float *scale, void *stream) {
    if (rows < 0 || F < 1) return fail(QNN_ERR_SHAPE, "silu_gate_quant: rows = %lld, F = %lld", (long long)rows, (long long)F);
    if (!rows::known_type(type)) return fail(QNN_ERR_SHAPE, "silu_gate_quant: type %d", type);
    if (ld_gate < F || ld_up < F || ld_codes < F) return fail(QNN_ERR_SHAPE, "silu_gate_quant: leading dimension too small");
    if (rows == 0) return QNN_OK;
    if (!gate || !up || !codes || !scale) return fail(QNN_ERR_NULL, "silu_gate_quant: NULL pointer");
    const int w = rows::value_bytes(type);
    if (!rows::aligned_to(gate, w) || !rows::aligned_to(up, w) || !rows::aligned_to(scale, 4))
        return fail(QNN_ERR_ALIGN, "silu_gate_quant: pointer not aligned to its type");
    return rows::with_type(type, [&](auto tag) {
        typedef decltype(tag) T;
        auto launch = [&](auto once) {
            const GateSource<T, decltype(once)::value> src = {static_cast<const T *>(gate), static_cast<const T *>(up), ld_gate, ld_up};
            return rows::launch_quant_rows("silu_gate_quant", src, rows, F, codes, ld_codes, scale, static_cast<hipStream_t>(stream));
        };
        return rows::beyond_caches((2.0 * w + 1.0) * (double)rows * (double)F) ? launch(std::true_type{}) : launch(std::false_type{});
    });
}

extern "C" int qnn_silu_gate_backward(const void *grad, int64_t ld_grad, const void *gate, int64_t ld_gate, const void *up, int64_t ld_up, int type,
                                      int64_t rows, int64_t F, void *grad_gate, int64_t ld_grad_gate, void *grad_up, int64_t ld_grad_up, void *stream) {
    if (rows < 0 || F < 1) return fail(QNN_ERR_SHAPE, "silu_gate_backward: rows = %lld, F = %lld", (long long)rows, (long long)F);
    if (!rows::known_type(type)) return fail(QNN_ERR_SHAPE, "silu_gate_backward: type %d", type);
    if (ld_grad < F || ld_gate < F || ld_up < F || ld_grad_gate < F || ld_grad_up < F)
        return fail(QNN_ERR_SHAPE, "silu_gate_backward: leading dimension too small");
    if (rows == 0) return QNN_OK;
    if (!grad || !gate || !up || !grad_gate || !grad_up) return fail(QNN_ERR_NULL, "silu_gate_backward: NULL pointer");
    const int w = rows::value_bytes(type);
    if (!rows::aligned_to(grad, w) || !rows::aligned_to(gate, w) || !rows::aligned_to(up, w) || !rows::aligned_to(grad_gate, w) ||
        !rows::aligned_to(grad_up, w))
        return fail(QNN_ERR_ALIGN, "silu_gate_backward: pointer not aligned to its type");
    const int64_t groups = ceil_div(F, rows::kVec), blocks = ceil_div(rows * groups, 256);
    return rows::with_type(type, [&](auto tag) {
        typedef decltype(tag) T;
        auto kernel = rows::beyond_caches(5.0 * w * (double)rows * (double)F) ? silu_gate_backward_kernel<T, true, false> : silu_gate_backward_kernel<T, false, false>;
        if (F < rows::kVec) kernel = silu_gate_backward_kernel<T, false, true>;
        return QNN_LAUNCH("silu_gate_backward", kernel, dim3((unsigned)(blocks > 16384 ? 16384 : blocks)), dim3(256), 0,
                          static_cast<hipStream_t>(stream), static_cast<const T *>(grad), ld_grad, static_cast<const T *>(gate), ld_gate,
                          static_cast<const T *>(up), ld_up, rows, F, groups, static_cast<T *>(grad_gate), ld_grad_gate, static_cast<T *>(grad_up),
                          ld_grad_up);
    });
}
