// Rows of floats that become int8 codes with one scale a row: typed loads and stores, the quantizer, reductions, and the kernel that the norm and
// the gated activation share (they differ in where a row's values come from).
//
// The quantizer: for a row y with a = max_k |y_k|, scale = a / 127 and code_k = rint(y_k 127 / a), ties to even, so code * scale is within scale / 2 of
// y and nothing is clipped.  a = 0: scale and codes 0.  A value that is not finite: scale NaN and codes 0, so that whatever is formed from the row is
// NaN too.  (LinearQuant of Sec. 3 has one step for a whole tensor; activations of a language model differ in size from token to token.)
#pragma once
#include <type_traits>

#include "qnn_internal.h"

namespace qnn {
namespace rows {

typedef __bf16 bf16;
typedef _Float16 f16;

constexpr int kVec = 8;  // consecutive values of a row that a lane takes: one 16-byte load of 16-bit floats, one 8-byte store of codes

template <typename T>
struct Raw {
    T e[kVec];
};
// The kVec values of a row of K that belong to the lane at k: the window from `from` on, of which the values before `skip` are another lane's (or nobody's).
// A row's last window ends where the row does, so that every load is whole, wide and within the row; loads that a lane's place in the row decided upon
// would have to be waited for one by one.  kShort: rows of fewer values than a window, loaded and stored one by one.
struct Window {
    int64_t from;
    int skip;
    __device__ __forceinline__ Window(int64_t k, int64_t K) : from(K < kVec ? k : (k < K - kVec ? k : K - kVec)), skip((int)((k - from) < kVec ? k - from : kVec)) {}
};
// kOnce: past the caches, for matrices that they could not hold anyway (10000 x 4096 bf16 and its residual to sum and codes, 287 MB: 88.6 -> 52.0 us; but
// 60 MB of fp32 20 -> 22).
typedef uint32_t Words4 __attribute__((ext_vector_type(4), aligned(2)));
template <bool kOnce, bool kShort, typename T>
__device__ __forceinline__ Raw<T> load_raw(const T *row, const Window &w, int64_t K) {
    Raw<T> r;
    if constexpr (kShort) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) r.e[i] = w.from + i < K ? row[w.from + i] : (T)0.0f;
    } else if constexpr (kOnce) {
        Words4 v[sizeof r / 16];
#pragma unroll
        for (int i = 0; i < (int)(sizeof r / 16); ++i) v[i] = __builtin_nontemporal_load(reinterpret_cast<const Words4 *>(row + w.from) + i);
        __builtin_memcpy(&r, v, sizeof r);
    } else {
        __builtin_memcpy(&r, row + w.from, sizeof r);
    }
    return r;
}
template <bool kOnce, bool kShort, typename T>
__device__ __forceinline__ void store_values(T *row, const Window &w, int64_t K, const float (&v)[kVec]) {
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        float x = v[i];
        // From the value in fp32.  (A product that the compiler rounds to fp16 in one instruction now and then differs in the last place from one that it rounds
        // twice, and which it takes depends on the variant and on the place in a window.)
        if constexpr (std::is_same<T, f16>::value) asm("" : "+v"(x));
        r.e[i] = (T)x;  // to nearest, ties to even
    }
    if (!kShort && w.skip == 0) {
        if constexpr (kOnce) {
            Words4 u[sizeof r / 16];
            __builtin_memcpy(u, &r, sizeof r);
#pragma unroll
            for (int i = 0; i < (int)(sizeof r / 16); ++i) __builtin_nontemporal_store(u[i], reinterpret_cast<Words4 *>(row + w.from) + i);
        } else {
            __builtin_memcpy(row + w.from, &r, sizeof r);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i >= w.skip && w.from + i < K) row[w.from + i] = r.e[i];
    }
}
// Whether a call's matrices, this many bytes together, are for the caches or not (256 MB on the card)
inline bool beyond_caches(double bytes) { return bytes > 128e6; }
// kVec values of fp32 or T, as is_f32 (the same for all lanes) says
template <bool kShort, typename T>
__device__ __forceinline__ void load_either(const void *p, bool is_f32, const Window &w, int64_t K, float (&v)[kVec]) {
    if (is_f32) {
        const Raw<float> r = load_raw<false, kShort>(static_cast<const float *>(p), w, K);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = r.e[i];
    } else {
        const Raw<T> r = load_raw<false, kShort>(static_cast<const T *>(p), w, K);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = (float)r.e[i];
    }
}

// |v| as an integer that orders like it, with every NaN above infinity: a maximum of these loses none
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// How a row is quantized, from the largest magnitude of its values (before a common factor that its scale takes in)
struct Quantizer {
    float mul, pre, scale;  // code = rint((v * pre) * mul)
    bool zero;              // all codes are 0
    __device__ __forceinline__ Quantizer(uint32_t top_bits, float factor) {
        const float top = __uint_as_float(top_bits);
        scale = top * factor / 127.0f;
        const bool fine = top_bits < 0x7F800000u && magnitude(scale) < 0x7F800000u;
        zero = !fine || top_bits == 0u;
        pre = top < 0x1p-64f ? 0x1p64f : 1.0f;  // (127 / top stays finite)
        mul = zero ? 0.0f : 127.0f / (top * pre);
        if (top_bits == 0u && magnitude(factor) <= 0x7F800000u)
            scale = 0.0f;
        else if (!fine)
            scale = __uint_as_float(0x7FC00000u);
    }
    // adding 1.5 * 2^23 rounds to the nearest integer, ties to even, and leaves it in the low bits
    __device__ __forceinline__ uint32_t code(float v) const { return __float_as_uint(__fmaf_rn(v * pre, mul, 12582912.0f)) & 0xFFu; }
    __device__ __forceinline__ uint32_t four(float a, float b, float c, float d) const {
        return zero ? 0u : code(a) | code(b) << 8 | code(c) << 16 | code(d) << 24;
    }
};
template <bool kShort>
__device__ __forceinline__ void store_codes(int8_t *row, const Window &at, int64_t K, const Quantizer &q, const float (&v)[kVec]) {
    const uint32_t w[2] = {q.four(v[0], v[1], v[2], v[3]), q.four(v[4], v[5], v[6], v[7])};
    if (!kShort && at.skip == 0) {
        __builtin_memcpy(row + at.from, w, sizeof w);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i >= at.skip && at.from + i < K) row[at.from + i] = (int8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
}

// 1 / (1 + exp(-x)), within 3 units in the last place; below 2^-126 it is 0.  exp(-x) = 2^n 2^f with n + f = -x log2(e), f to twice the digits.  Infinities have
// the limits; a NaN is lost, and has to be in the factor beside.  (With expf
// and a correctly rounded quotient the vector ALU bounds the gated activation: 47 us at 10000 x 4096, 205 MB.)
__device__ __forceinline__ float sigmoid(float x) {
    constexpr float kLog2e = 0x1.715476p+0f, kRest = 0x1.4ae0cp-26f;  // together log2(e)
    const float y = __builtin_amdgcn_fmed3f(x, -1000.0f, 1000.0f), n = rintf(y * -kLog2e), f = __fmaf_rn(y, -kRest, __fmaf_rn(y, -kLog2e, -n));
    const float e = __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(f), (int)n);
    return __builtin_amdgcn_rcpf(1.0f + e);
}
__device__ __forceinline__ float silu(float x) { return x * sigmoid(x); }

// Sums over the lanes that share a row, given to all of them: a wave, or a workgroup of kThreads, whose waves meet in `shared` (two buffers used in
// turn: a wave writes one only behind the barrier after which every wave has read the other)
template <int kThreads, typename V, typename Join>
__device__ __forceinline__ V across(V v, Join join, V (*shared)[kThreads / 64], int turn) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v = join(v, v.shuffled(d));
    if constexpr (kThreads > 64) {
        constexpr int kWaves = kThreads / 64;
        if ((threadIdx.x & 63) == 0) shared[turn][threadIdx.x % kThreads >> 6] = v;
        __syncthreads();
        v = shared[turn][0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v = join(v, shared[turn][w]);
    }
    return v;
}
struct SumTop {
    float sum;
    uint32_t top;
    __device__ __forceinline__ SumTop shuffled(int d) const { return {__shfl_xor(sum, d), (uint32_t)__shfl_xor((int)top, d)}; }
    static __device__ __forceinline__ SumTop join(const SumTop &a, const SumTop &b) { return {a.sum + b.sum, a.top > b.top ? a.top : b.top}; }
};
struct TwoSums {
    float a, b;
    __device__ __forceinline__ TwoSums shuffled(int d) const { return {__shfl_xor(a, d), __shfl_xor(b, d)}; }
    static __device__ __forceinline__ TwoSums join(const TwoSums &x, const TwoSums &y) { return {x.a + y.a, x.b + y.b}; }
};

// `blocks` workgroups of up to 1024 threads, and less than a line of them more, in lines of kLine: HIP launches fewer than 2^32 threads along a dimension
constexpr int64_t kLine = 1 << 21;
inline dim3 grid_of(int64_t blocks) { return blocks <= kLine ? dim3((unsigned)blocks) : dim3((unsigned)kLine, (unsigned)ceil_div(blocks, kLine)); }
__device__ __forceinline__ uint32_t block_number() { return blockIdx.y * (uint32_t)kLine + blockIdx.x; }

constexpr int rows_per_block(int threads) { return threads >= 256 ? 1 : 256 / threads; }

// One row per kThreads lanes.  Source: `load<kShort>(row, window, K, values, kept)` the values to be quantized, up to the factor `factor(sum)`;
// `add(kept, i, sum)` the sum with value i's part; `keep<kShort>(row, window, K, kept)` writes what else it does.
// kPer: windows that a lane keeps in registers; 0: as many as there are, loaded a second time for the codes.
template <typename Source, int kThreads, int kPer, bool kShort>
__global__ __launch_bounds__(kThreads >= 256 ? kThreads : 256) void quant_rows_kernel(const Source src, int64_t n_rows, int64_t K, int8_t *codes,
                                                                                     int64_t ld_codes, float *scale) {
    __shared__ SumTop shared[2][kThreads / 64];
    const int lane = threadIdx.x % kThreads;
    const int64_t row = (int64_t)block_number() * rows_per_block(kThreads) + threadIdx.x / kThreads;
    if (row >= n_rows) return;  // (the same for all lanes of a row, and a workgroup with a barrier has one)
    constexpr int kHeld = kPer > 0 ? kPer : 1;
    float v[kHeld][kVec];
    typename Source::Kept kept[kHeld];
    SumTop s = {0.0f, 0u};
    auto stats = [&](int i, const Window &w) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            const bool mine = e >= w.skip && (!kShort || w.from + e < K);
            s.sum = mine ? src.add(kept[i], e, s.sum) : s.sum;
            s.top = max(s.top, mine ? magnitude(v[i][e]) : 0u);
        }
    };
    auto give = [&](const Quantizer &q, int i, const Window &w) __attribute__((always_inline)) {
        src.template keep<kShort>(row, w, K, kept[i]);
        store_codes<kShort>(codes + row * ld_codes, w, K, q, v[i]);
    };
    if constexpr (kPer > 0) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) src.template load<kShort>(row, Window((int64_t)(i * kThreads + lane) * kVec, K), K, v[i], kept[i]);
#pragma unroll
        for (int i = 0; i < kPer; ++i) stats(i, Window((int64_t)(i * kThreads + lane) * kVec, K));
    } else {
        for (int64_t k = lane * kVec; k < K; k += kThreads * kVec) {
            src.template load<kShort>(row, Window(k, K), K, v[0], kept[0]);
            stats(0, Window(k, K));
        }
    }
    s = across<kThreads>(s, SumTop::join, shared, 0);
    const Quantizer q(s.top, src.factor(s.sum, K));
    if (lane == 0) scale[row] = q.scale;
    if constexpr (kPer > 0) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int64_t k = (int64_t)(i * kThreads + lane) * kVec;
            if (k < K) give(q, i, Window(k, K));
        }
    } else {
        for (int64_t k = lane * kVec; k < K; k += kThreads * kVec) {
            src.template load<kShort>(row, Window(k, K), K, v[0], kept[0]);
            give(q, 0, Window(k, K));
        }
    }
}

template <typename Source, int kThreads, int kPer, bool kShort = false>
int launch_shape(const char *what, const Source &src, int64_t n_rows, int64_t K, int8_t *codes, int64_t ld_codes, float *scale, hipStream_t s) {
    const int64_t blocks = ceil_div(n_rows, rows_per_block(kThreads));
    if (blocks > 0x7FFFFFFFLL) return fail(QNN_ERR_SHAPE, "%s: %lld rows", what, (long long)n_rows);
    return QNN_LAUNCH(what, (quant_rows_kernel<Source, kThreads, kPer, kShort>), grid_of(blocks), dim3(kThreads >= 256 ? kThreads : 256), 0, s, src, n_rows, K, codes,
                      ld_codes, scale);
}
// Lanes and groups by the length of a row
template <typename Source>
int launch_quant_rows(const char *what, const Source &src, int64_t n_rows, int64_t K, int8_t *codes, int64_t ld_codes, float *scale, hipStream_t s) {
    if (K < kVec) return launch_shape<Source, 64, 1, true>(what, src, n_rows, K, codes, ld_codes, scale, s);
    if (K <= 64 * kVec) return launch_shape<Source, 64, 1>(what, src, n_rows, K, codes, ld_codes, scale, s);
    if (K <= 128 * kVec) return launch_shape<Source, 64, 2>(what, src, n_rows, K, codes, ld_codes, scale, s);
    if (K <= 256 * kVec) return launch_shape<Source, 256, 1>(what, src, n_rows, K, codes, ld_codes, scale, s);
    if (K <= 512 * kVec) return launch_shape<Source, 256, 2>(what, src, n_rows, K, codes, ld_codes, scale, s);
    if (K <= 1024 * kVec) return launch_shape<Source, 256, 4>(what, src, n_rows, K, codes, ld_codes, scale, s);
    if (K <= 4096 * kVec) return launch_shape<Source, 1024, 4>(what, src, n_rows, K, codes, ld_codes, scale, s);
    return launch_shape<Source, 1024, 0>(what, src, n_rows, K, codes, ld_codes, scale, s);
}

// Arguments of the float matrices of these calls
inline int value_bytes(int type) { return type == QNN_F32 ? 4 : 2; }
inline bool known_type(int type) { return type == QNN_F32 || type == QNN_F16 || type == QNN_BF16; }
inline bool aligned_to(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }
// f(T{}) for the C++ type of `type`
template <typename F>
int with_type(int type, F f) {
    if (type == QNN_F32) return f(0.0f);
    if (type == QNN_F16) return f((f16)0.0f);
    return f((bf16)0.0f);
}

}  // namespace rows
}  // namespace qnn
