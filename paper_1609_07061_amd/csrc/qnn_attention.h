// Attention over a paged cache of int8 codes: what the kernels share.
//
// Of a query q (a row of D floats) and the keys it sees, code rows c_j with scales a_j and value codes v_j with scales b_j:
//   s_j = scale a_j (q . c_j), capped and biased as asked;   out = sum_j 2^(t_j - R) b_j v_j / sum_j 2^(t_j - R),   t_j = s_j log2(e).
// One pass over the keys.  Both products are matrix instructions on float16 operands with sums in fp32: a code is exact in float16; q is brought to 2^13 .. 2^14 by a
// power of two, so that values 2^-28 of its largest still have all of their digits; the weight w_j = 2^(t_j - R) b_j is what meets the value codes.  Of bf16 results
// an eighth of their own rounding is the weights' (half a step is 2^-11 of a weight, 2^-8 of a result); for fp16 and fp32 results weights are held in two parts, 22
// digits, and so are fp32 queries.
// R follows the largest of t_j + log2(b_j) seen, so that w_j is at most 2^15 and the largest about 2^8: small weights keep their digits down to 2^-22 of it, however
// the scales b_j differ.  It moves only when a weight would pass 2^15: the sums are multiplied by a power then, and nothing else.  Sums that belong to different R
// (of waves, of parts of the keys) are joined in a fixed order.
// The sum below the line has the factors 2^(t_j - R) without b_j, which are large where b_j is small, and where it is 0 nothing is seen of them in w_j: log2(b_j) counts as
// kLowest at least, so that they are at most 2^104 of the keys that R has followed, and R moves too when a lane's sum of a step passes 2^109.  (2^22 tokens of zeros in one
// part of the keys stay within fp32.)
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
constexpr float kLowest = -96.0f;   // log2 of the least scale of values that R follows: what zeros count as
constexpr float kOfSum = 0x1p-94f;  // weight that a sum of 2^(t - R) counts as, over the up to 16 keys that a lane has at a time: 2^109 moves R, and each is up to 2^104 then

// A lane's number that the compiler cannot see through: what follows from it is worked out where it is needed.  (Worked out once before the loops, addresses take
// some 100 registers, and the sums are spilled.)
__device__ __forceinline__ int opaque(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// log2 of a scale of values, rounded up, for R to follow
__device__ __forceinline__ float log_scale(float v) { return v != 0.0f ? fmaxf((float)__builtin_amdgcn_frexp_expf(v), kLowest) : kLowest; }

// The root of what sums that belong to one R are multiplied by for another one.  (Sums of 2^(t - R) are up to 2^128 and may count where the factor itself is below the normal
// numbers: they take the root twice.)
__device__ __forceinline__ float root_of(float level, float top) { return level == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(0.5f * (level - top)); }

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
    int32_t D, heads_q, group, splits, blocks;  // blocks: of rows, for each sequence and head of the cache
    int32_t short_rows;  // 0, or: sequences of at most this many rows are the kernel's for few, the others that for many
    uint32_t group_inverse, heads_inverse, heads_q_inverse, splits_inverse, blocks_inverse;
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

// Capped scores times log2(e): cap log2(e) tanh(x) with x = score / cap.  Two ways, by the call's cap:
//   1 - 2 / (e^2x + 1) from y = 2 log2(e) x (the query's factor has it all), off by up to 2^-21 of the cap.  Of a cap of 64 that is 2^-15, a sixteenth of half a step of float16, so
//   this is the way up to there, but for fp32 results;
//   close: from the score itself and, where |x| < 0.35, the beginning of tanh's series times it, so that small scores keep their digits whatever the cap is.  (With it for a cap
//   of 50: 40 drafted tokens of 8 sequences of up to 4099, fp16, 59 us for 53; the last 2048 of 8192, bf16, 578 for 420.)
constexpr float kCloseFrom = 64.0f;
struct Cap {
    float size, before, inverse;  // cap log2(e); what the query's factor takes; 1 / size
};
template <typename T>
constexpr bool kAlwaysClose = std::is_same<T, float>::value;
template <bool kClose>
__device__ __forceinline__ Cap cap_of(const Args &a) {
    const float size = fminf(a.cap * kLog2e, 3.4028234e38f);
    return {size, kClose ? kLog2e : 2.0f * kLog2e / a.cap, 1.0f / size};
}
template <bool kClose>
__device__ __forceinline__ float capped(const Cap &c, float y) {
    if constexpr (!kClose) return __fmaf_rn(-2.0f * c.size, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(y)), c.size);
    const float x = y * c.inverse, s = x * x;
    const float far = c.size * __fmaf_rn(-2.0f, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * (2.0f * kLog2e))), 1.0f);
    float near = __fmaf_rn(s, -8.86323553e-3f, 2.18694885e-2f);  // -1382 / 155925, 62 / 2835
    near = __fmaf_rn(s, near, -5.39682540e-2f), near = __fmaf_rn(s, near, 0.133333333f), near = __fmaf_rn(s, near, -0.333333333f);
    return fabsf(x) < 0.35f ? __fmaf_rn(y * s, near, y) : far;
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

template <typename T>
struct Parts {
    static constexpr int kQuery = std::is_same<T, float>::value ? 2 : 1, kWeight = std::is_same<T, rows::bf16>::value ? 1 : 2;
};

// A row of queries from the power of two that brings its largest value to 2^13 .. 2^14.  `top`: the largest magnitude, as rows::magnitude has it
struct Scaling {
    int exponent;
    bool fine;
    __device__ __forceinline__ explicit Scaling(uint32_t top)
        : exponent(top > 0u && top < 0x7F800000u ? __builtin_amdgcn_frexp_expf(__uint_as_float(top)) - 14 : -14), fine(top < 0x7F800000u) {}
    __device__ __forceinline__ float of(float x) const { return fine ? __builtin_amdgcn_ldexpf(x, -exponent) : __uint_as_float(0x7FC00000u); }
    __device__ __forceinline__ float mult(float scale) const { return __builtin_amdgcn_ldexpf(scale, exponent); }  // of the sums
};
template <int kParts>
__device__ __forceinline__ void split(float y, _Float16 (&part)[kParts]) {
    // (from the value in fp32: a product that the compiler rounds to fp16 in one instruction may differ from the one that it takes off for the second part)
    if constexpr (kParts == 2) asm("" : "+v"(y));
    part[0] = (_Float16)y;
    if constexpr (kParts == 2) part[1] = (_Float16)(y - (float)part[0]);
}

template <typename T>
__device__ __forceinline__ void store_eight(void *p, int64_t at, const float (&x)[8]) {
    rows::store_values<false, false>(static_cast<T *>(p) + at, rows::Window(0, 8), 8, x);
}

// What a row sees beyond the keys that all rows of a block see: those up to `last`, and of a tree's drafted ones those in `mask`
struct Sight {
    int32_t last;
    uint64_t mask;
    float slope;  // times log2(e)
    int32_t place;
    __device__ __forceinline__ void load(const Args &a, const Sequence &s, const Row &row) {
        mask = a.tree ? a.tree[row.token] : 0ull;
        last = a.tree ? s.base - 1 : s.base + row.i;
        place = a.tree ? s.base - 1 + __popcll(mask) : last;
        slope = a.slopes ? a.slopes[row.head] * kLog2e : 0.0f;
    }
    // kTree: whether there are masks.  (Without branches: sixteen keys' branches one after the other take longer than the products.)
    template <bool kTree>
    __device__ __forceinline__ bool sees(const Sequence &s, int32_t key) const {
        const bool before = key <= last;
        if constexpr (!kTree) return before;
        const uint32_t drafted = (uint32_t)(key - s.base);
        return before | ((drafted < 64u) & (bool)(mask >> (drafted & 63u) & 1ull));
    }
};

// How a call is split: rows of a workgroup, blocks of rows for each sequence and head of the cache, and parts of the keys
struct Plan {
    int rows;
    int64_t blocks, splits;
};
constexpr int kMostSplits = 128;

// qnn_cache_attention_many.hip: the kernel for many rows
constexpr int many_rows(int64_t D) { return D <= 128 ? 256 : 128; }  // of a workgroup
// (two parts of a query of 256 values and its sums are more than a lane's registers)
constexpr bool takes_many(int64_t D, int type) { return D <= 128 || type != QNN_F32; }
int launch_many(const Args &a, int type, dim3 grid, hipStream_t s);

}  // namespace attention
}  // namespace qnn
