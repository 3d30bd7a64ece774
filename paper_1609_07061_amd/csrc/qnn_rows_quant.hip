// Rows of floats to int8 codes with one scale a row (qnn_rows.h), without a norm or an activation: the attention's result in front of the output product.
// Bound by memory: a read of every value and a write of a byte (8192 x 4096 bf16: 101 MB in 24 us; one row: 3.7, its launch).
#include <type_traits>

#include "qnn_rows.h"

namespace qnn {
namespace {

using namespace rows;

template <typename T, bool kOnce>
struct PlainSource {
    struct Kept {};
    static constexpr bool kExact = true;
    const T *x;
    int64_t ldx;
    template <bool kShort>
    __device__ __forceinline__ void load(int64_t row, const Window &w, int64_t K, float (&v)[kVec], Kept &) const {
        const Raw<T> a = load_raw<kOnce, kShort>(x + row * ldx, w, K);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = (float)a.e[i];
    }
    __device__ __forceinline__ float add(const Kept &, int, float sum) const { return sum; }
    __device__ __forceinline__ float factor(float, int64_t) const { return 1.0f; }
    template <bool kShort>
    __device__ __forceinline__ void keep(int64_t, const Window &, int64_t, const Kept &) const {}
};

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" int qnn_rows_quant(const void *x, int64_t ldx, int type, int64_t rows, int64_t K, int8_t *codes, int64_t ld_codes, float *scale, void *stream) {
    if (rows < 0 || K < 1) return fail(QNN_ERR_SHAPE, "rows_quant: rows = %lld, K = %lld", (long long)rows, (long long)K);
    if (!rows::known_type(type)) return fail(QNN_ERR_SHAPE, "rows_quant: type %d", type);
    if (ldx < K || ld_codes < K) return fail(QNN_ERR_SHAPE, "rows_quant: leading dimension too small");
    if (rows == 0) return QNN_OK;
    if (!x || !codes || !scale) return fail(QNN_ERR_NULL, "rows_quant: NULL pointer");
    const int w = rows::value_bytes(type);
    if (!rows::aligned_to(x, w) || !rows::aligned_to(scale, 4)) return fail(QNN_ERR_ALIGN, "rows_quant: pointer not aligned to its type");
    return rows::with_type(type, [&](auto tag) {
        typedef decltype(tag) T;
        auto launch = [&](auto once) {
            const PlainSource<T, decltype(once)::value> src = {static_cast<const T *>(x), ldx};
            return rows::launch_quant_rows("rows_quant", src, rows, K, codes, ld_codes, scale, static_cast<hipStream_t>(stream));
        };
        return rows::beyond_caches((w + 1.0) * (double)rows * (double)K) ? launch(std::true_type{}) : launch(std::false_type{});
    });
}
