// Attention over a paged cache of int8 codes: what the kernels share.
//
// Of a query q (a row of D floats) and the keys it sees, code rows c_j with scales a_j and value codes v_j with scales b_j:
//   s_j = scale a_j (q . c_j), capped and biased as asked;   out = sum_j 2^(t_j - R) b_j v_j / sum_j 2^(t_j - R),   t_j = s_j log2(e).
// One pass over the keys.  Both products are matrix instructions on float16 operands with sums in fp32: a code is exact in float16; q is brought to 2^13 .. 2^14 by a
// power of two, so that values 2^-28 of its largest still have all of their digits; the weight w_j = 2^(t_j - R) b_j is what meets the value codes.  fp32 queries
// and their weights are held in two parts, 22 digits; of 16-bit ones the weight's rounding is 2^-12, an eighth of the bf16 result's.
// R follows the largest of t_j + log2(b_j) seen, so that w_j is at most 2^15 and the largest about 2^8: small weights keep their digits down to 2^-22 of it, however
// the scales b_j differ.  It moves only when a weight would pass 2^15: the sums are multiplied by a power then, and nothing else.  Sums that belong to different R
// (of waves, of parts of the keys) are joined in a fixed order.
#pragma once
#include <type_traits>

#include "qnn_paged.h"

namespace qnn {
namespace attention {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504f;
constexpr float kLowest = -100.0f;  // log2 of the least scale of values that R follows (zeros have none)

struct Args {
    const void *q;
    void *out;
    int64_t ld_q, step_q, ld_out, step_out;
    const int8_t *k, *v;
    const float *k_scale, *v_scale;
    paged::Pages pages;
    const int32_t *starts, *lengths;
    const float *slopes;
    const uint64_t *tree;
    float scale, cap;
    int64_t tokens, sequences;
    int32_t type, D, heads_q, group, splits, blocks;  // blocks: of rows, for each sequence and head of the cache
    uint32_t group_inverse, heads_inverse, splits_inverse, blocks_inverse;
    float *part;   // [splits][tokens][heads_q][D]: sums, where splits > 1
    float2 *state;  // [splits][tokens][heads_q]: R, sum of 2^(t - R)
};

// Four codes as float16: the byte u = code + 128 behind 0x64 is 1024 + u.  lo, hi: codes 0, 1 and 2, 3
__device__ __forceinline__ h2 halves(uint32_t biased_pair) {
    union {
        uint32_t u;
        h2 h;
    } x = {biased_pair};
    return x.h + h2{(_Float16)-1152.0f, (_Float16)-1152.0f};
}
constexpr uint32_t kBias = 0x80808080u, kExponents = 0x64646464u;
__device__ __forceinline__ h4 four_codes(uint32_t x) {
    x ^= kBias;
    const h2 lo = halves(__builtin_amdgcn_perm(kExponents, x, 0x04010400u)), hi = halves(__builtin_amdgcn_perm(kExponents, x, 0x04030402u));
    return h4{lo[0], lo[1], hi[0], hi[1]};
}
__device__ __forceinline__ h8 eight_codes(uint32_t x, uint32_t y) {
    const h4 a = four_codes(x), b = four_codes(y);
    return h8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// tanh within some 5 units in the last place: 1 - 2 / (e^2x + 1), and the beginning of its series where that would lose digits
__device__ __forceinline__ float tanh_of(float x) {
    const float size = __uint_as_float(rows::magnitude(x)), a = size > 20.0f ? 20.0f : size, s = a * a;
    const float far = 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(a * (2.0f * kLog2e)));
    float near = __fmaf_rn(s, -8.86323553e-3f, 2.18694885e-2f);  // -1382 / 155925, 62 / 2835
    near = __fmaf_rn(s, near, -5.39682540e-2f), near = __fmaf_rn(s, near, 0.133333333f), near = __fmaf_rn(s, near, -0.333333333f);
    near = __fmaf_rn(a * s, near, a);
    return copysignf(a < 0.35f ? near : far, x);
}

// A sequence as the kernels need it
struct Sequence {
    int64_t first;    // its first new token
    int32_t n, fresh, base;  // tokens, new ones that the call has, n - all new ones (below 0: the first of these have no place)
    int32_t in_table;        // tokens that the table has room for, at most n
};
constexpr int32_t kLongest = 0x7FFFF000;  // (steps beyond a sequence's end still have numbers)
__device__ __forceinline__ Sequence sequence_at(const Args &a, uint32_t b) {
    const int32_t first = a.starts[b], fresh = max(a.starts[b + 1] - first, 0), n = min(max(a.lengths[b], 0), kLongest);
    const int64_t room = a.pages.width * a.pages.page;
    const bool fine = first >= 0 && first < a.tokens;
    return {first, n, fine ? (int32_t)min((int64_t)fresh, a.tokens - first) : 0, n - fresh, (int32_t)min((int64_t)n, room)};
}

// A row of queries: token i of the sequence's new ones, head of the queries
struct Row {
    int32_t i;
    int64_t token, head;
};
__device__ __forceinline__ Row row_at(const Args &a, const Sequence &s, uint32_t row, uint32_t head) {
    uint32_t in_group;
    const uint32_t i = quotient(row, (uint32_t)a.group, a.group_inverse, in_group);
    return {(int32_t)i, s.first + i, (int64_t)head * a.group + in_group};
}

// 16 floats of a query at p (fp32, fp16 or bf16)
__device__ __forceinline__ void load_values(const void *p, int64_t at, int type, float (&x)[16]) {
    auto take = [&](auto tag) __attribute__((always_inline)) {
        typedef decltype(tag) T;
        T e[16];
        __builtin_memcpy(e, static_cast<const T *>(p) + at, sizeof e);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = (float)e[i];
    };
    if (type == QNN_F32)
        take(0.0f);
    else if (type == QNN_F16)
        take((rows::f16)0.0f);
    else
        take((rows::bf16)0.0f);
}
__device__ __forceinline__ void store_values(void *p, int64_t at, int type, const float (&x)[8]) {
    const rows::Window w(0, 8);
    if (type == QNN_F32)
        rows::store_values<false, false>(static_cast<float *>(p) + at, w, 8, x);
    else if (type == QNN_F16)
        rows::store_values<false, false>(static_cast<rows::f16 *>(p) + at, w, 8, x);
    else
        rows::store_values<false, false>(static_cast<rows::bf16 *>(p) + at, w, 8, x);
}

// A query's lanes: DP / 64 runs of 16 values, 64 c + 16 g + 0 .. 15 with g = lane / 16, as float16 operands for the products with 16 bytes of code each
template <int DP, int kParts>
struct Query {
    h8 part[kParts][DP / 64][2];
    float mult;  // scale of the sums: scale * 2^(what was taken out)
    __device__ __forceinline__ void load(const Args &a, const Row &row) {
        const int g = (threadIdx.x & 63) >> 4;
        float x[DP / 64][16];
        uint32_t top = 0u;
#pragma unroll
        for (int c = 0; c < DP / 64; ++c) {
            const int d = 64 * c + 16 * g;
            if (d < a.D) {
                load_values(a.q, row.token * a.ld_q + row.head * a.step_q + d, a.type, x[c]);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[c][i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) top = max(top, rows::magnitude(x[c][i]));
        }
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        const bool fine = top < 0x7F800000u;
        const int e = fine && top ? __builtin_amdgcn_frexp_expf(__uint_as_float(top)) : 0;
        mult = __builtin_amdgcn_ldexpf(a.scale, e - 14);
#pragma unroll
        for (int c = 0; c < DP / 64; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float y = fine ? __builtin_amdgcn_ldexpf(x[c][i], 14 - e) : __uint_as_float(0x7FC00000u);
                const _Float16 hi = (_Float16)y;
                part[0][c][i >> 3][i & 7] = hi;
                if constexpr (kParts == 2) part[1][c][i >> 3][i & 7] = (_Float16)(y - (float)hi);
            }
    }
};

// What a row sees beyond the keys that all rows of a block see
struct Sight {
    int32_t last;     // causal: the last key
    uint64_t mask;    // tree
    float slope;      // times log2(e)
    int32_t place;
    __device__ __forceinline__ void load(const Args &a, const Sequence &s, const Row &row) {
        last = s.base + row.i;
        mask = a.tree ? a.tree[row.token] : 0ull;
        place = a.tree ? s.base - 1 + __popcll(mask) : last;
        slope = a.slopes ? a.slopes[row.head] * kLog2e : 0.0f;
    }
    __device__ __forceinline__ bool sees(const Args &a, const Sequence &s, int32_t key) const {
        if (!a.tree) return key <= last;
        const int32_t drafted = key - s.base;
        return drafted < 0 || (drafted < 64 && (mask >> (drafted & 63) & 1ull));
    }
};

}  // namespace attention
}  // namespace qnn
