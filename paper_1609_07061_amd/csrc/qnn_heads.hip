// Heads of queries and keys: root-mean-square norm, rotation by the tokens' positions, and, for a paged cache, int8 codes of keys and values; the gradient of norm
// and rotation.
//
// Forward: r = 1 / sqrt(mean h^2 + eps) of a head's D values, n = h r gamma, every pair (n_a, n_b) turned by its angle.  A head is D / 16 lanes of two windows of
// eight values each, so that a lane has both halves of eight pairs, whichever way pairs are formed; the sum of squares and, for codes, the largest magnitude are
// joined across the lanes without LDS.  Angles are formed once for a token, in 64 bits (position * frequency in quarter turns, its fraction to fp32), and stay as
// cosine and sine in LDS for all heads.
// Bound by memory: a read and a write of every value (8192 tokens of 40 heads of 128, bf16: 168 MB in 38 us; with a workgroup for every group of tokens, which asks for
// its weights anew, 49; the gradient, two reads: 252 MB in 52 us and 4.6 for the weights' sums; keys and values of 4096 tokens to the cache, 8 heads each beside 32 of
// queries: 50 MB read, 42 written in 27, of which the look-ups before each workgroup's only group are some 8).  Few tokens: the launch (20 tokens: 5.8 us; of the gradient 2000: 19, in groups as for many 32).
#include <type_traits>

#include "qnn_paged.h"

namespace qnn {
namespace {

using namespace rows;
using paged::kNoRow;

struct Matrix {  // heads of tokens
    const void *p;
    int64_t ld, step;
    template <typename T>
    __device__ __forceinline__ T *at(int64_t token, int64_t head) const {
        return static_cast<T *>(const_cast<void *>(p)) + token * ld + head * step;
    }
};

// cos and sin of position * quarters quarter turns, quarters = freq * 2 / pi: the fraction of the quarter turn, at most half in size, in fp32; Taylor's polynomials
// on +-pi/4, whose first terms left out are below 2^-29 and 2^-32
__device__ __forceinline__ float2 turn_of(int32_t position, double quarters) {
    const double x = (double)position * quarters, n = rint(x);
    const float a = (float)((x - n) * 1.5707963267948966), s = a * a;
    float sin = __fmaf_rn(s, 2.75573192e-6f, -1.98412698e-4f);
    sin = __fmaf_rn(s, sin, 8.33333333e-3f), sin = __fmaf_rn(s, sin, -0.166666667f), sin = __fmaf_rn(a * s, sin, a);
    float cos = __fmaf_rn(s, -2.75573192e-7f, 2.48015873e-5f);
    cos = __fmaf_rn(s, cos, -1.38888889e-3f), cos = __fmaf_rn(s, cos, 4.16666667e-2f), cos = __fmaf_rn(s, cos, -0.5f), cos = __fmaf_rn(s, cos, 1.0f);
    const int quarter = (int)(n - 4.0 * floor(n * 0.25));  // 0 .. 3
    const float c = (quarter & 1) ? sin : cos, d = (quarter & 1) ? cos : sin;
    return make_float2((quarter == 1 || quarter == 2) ? -c : c, (quarter & 2) ? -d : d);
}

// A reduction over the G lanes of a head, G = 4, 8 or 16 neighbours, given to all of them
template <int kControl>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kControl, 0xF, 0xF, true);
}
template <int G, typename Join>
__device__ __forceinline__ uint32_t over_head(uint32_t v, Join join) {
    v = join(v, moved<0xB1>(v));                          // lane xor 1
    v = join(v, moved<0x4E>(v));                          // lane xor 2
    if constexpr (G >= 8) v = join(v, moved<0x141>(v));   // 7 - lane: all of a four are alike by now
    if constexpr (G >= 16) v = join(v, moved<0x140>(v));  // 15 - lane
    return v;
}
template <int G>
__device__ __forceinline__ float sum_of_head(float v) {
    return __uint_as_float(over_head<G>(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
template <int G>
__device__ __forceinline__ uint32_t most_of_head(uint32_t v) {
    return over_head<G>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

constexpr int kThreads = 256, kMostPairs = paged::kMostD / 2;

struct Angles {
    const int32_t *positions, *axis;
    const double *freq;
    int64_t ld;
    int32_t axes, pairs, neighbours;
    uint32_t pairs_inverse;
};

// The turns of tokens t0 .. t0 + n - 1 into LDS, pair by pair
__device__ __forceinline__ void turns_of(const Angles &a, int64_t t0, int n, float2 (*turns)[kMostPairs]) {
    if (a.pairs == 0) return;
    for (uint32_t x = threadIdx.x; x < (uint32_t)(n * a.pairs); x += kThreads) {
        uint32_t pair;
        const uint32_t token = quotient(x, (uint32_t)a.pairs, a.pairs_inverse, pair);
        const int32_t axis = a.axis ? min(max(a.axis[pair], 0), a.axes - 1) : 0;
        turns[token][pair] = turn_of(a.positions[axis * a.ld + t0 + token], a.freq[pair] * 0.63661977236758134);
    }
}

// A lane's two windows of a head, 8 values each, and its pairs
struct Lane {
    int first, second, pair;
    bool on, turns, neighbours;
    __device__ __forceinline__ Lane(int unit, int D, const Angles &a) : on(unit < D / 16), turns(unit < a.pairs / 8), neighbours(a.neighbours != 0) {
        const bool halves = turns && !neighbours;
        pair = 8 * unit;
        first = on ? (halves ? 8 * unit : 16 * unit) : 0;
        second = on ? (halves ? a.pairs + 8 * unit : 16 * unit + 8) : 0;
    }
};
// The pairs of x (first window) and y (second), turned by kSign times their angles
template <int kSign>
__device__ __forceinline__ void turn(const Lane &l, const float2 *turns, float (&x)[kVec], float (&y)[kVec]) {
    if (!l.turns) return;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        const float2 t = turns[l.pair + i];
        const float c = t.x, s = kSign > 0 ? t.y : -t.y;
        if (l.neighbours) {
            float &a = i < 4 ? x[2 * i] : y[2 * i - 8], &b = i < 4 ? x[2 * i + 1] : y[2 * i - 7];
            const float u = __fmaf_rn(a, c, -(b * s)), v = __fmaf_rn(b, c, a * s);
            a = u, b = v;
        } else {
            const float u = __fmaf_rn(x[i], c, -(y[i] * s)), v = __fmaf_rn(y[i], c, x[i] * s);
            x[i] = u, y[i] = v;
        }
    }
}
// gamma of the lane's values
template <typename T>
__device__ __forceinline__ void load_gamma(const void *gamma, bool is_f32, const Lane &l, int D, float (&x)[kVec], float (&y)[kVec]) {
    load_either<false, T>(gamma, is_f32, Window(l.first, D), D, x);
    load_either<false, T>(gamma, is_f32, Window(l.second, D), D, y);
}

// norm_factor of a head, from the sum of its squares: the root's reciprocal within a unit in the last place, without a root and a quotient.  Infinite for a head of zeros
// without eps, as for one whose squares are below the normal numbers: heads_kernel tells them apart.
__device__ __forceinline__ float head_factor(float total, float inverse_D, float eps) {
    const float mean = __fmaf_rn(total, inverse_D, eps);
    if (mean < 0x1p-126f) return __uint_as_float(0x7F800000u);
    return magnitude(mean) < 0x7F800000u ? __builtin_amdgcn_rsqf(mean) : __uint_as_float(0x7FC00000u);
}

// Sequence of a token: the last that begins at or before it, found by a whole wave, 64 beginnings at a time.  -1: none
__device__ __forceinline__ int64_t sequence_of(const int32_t *starts, int64_t sequences, int64_t token) {
    int64_t lo = 0, n = sequences;
    const int lane = threadIdx.x & 63;
    while (true) {
        const int64_t step = (n + 63) / 64, at = lane * step;
        const int c = __popcll(__ballot(at < n && starts[lo + (at < n ? at : 0)] <= token));
        if (c == 0) return -1;
        lo += (c - 1) * step;
        if (step == 1) break;
        n = n - (c - 1) * step < step ? n - (c - 1) * step : step;
    }
    return token < starts[lo + 1] ? lo : -1;
}

struct HeadsArgs {
    Matrix q, k, v, q_out, k_out;
    const void *gamma_q, *gamma_k;
    bool gamma_f32;
    float eps, inverse_D;
    Angles angles;
    int64_t tokens;
    int32_t D, heads_q, heads_k, per_block;  // per_block: tokens of a workgroup
    uint32_t heads_inverse;                  // of all heads of a token
    // appending: k_out and v_out are codes
    paged::Pages pages;
    const int32_t *starts, *lengths;
    int64_t sequences;
    int8_t *codes_k, *codes_v;
    float *scale_k, *scale_v;
};

constexpr int kMostTokens = 4;

// kOnce: past the caches (beyond_caches)
template <typename T, int G, bool kAppend, bool kOnce>
__global__ __launch_bounds__(kThreads) void heads_kernel(const HeadsArgs a) {
    __shared__ float2 turns[kMostTokens][kMostPairs];
    __shared__ uint32_t places[kMostTokens];
    __shared__ bool known[kMostTokens];  // to a sequence
    const int unit = threadIdx.x % G;
    const Lane lane(unit, a.D, a.angles);
    const Window first(lane.first, a.D), second(lane.second, a.D);
    const uint32_t heads = (uint32_t)(a.heads_q + (kAppend ? 2 : 1) * a.heads_k);
    // (the weights stay in registers: asked for with an item, they would come behind the next one's values, which would be waited for)
    float gamma[2][2][kVec];
    if (a.gamma_q) {
        load_gamma<T>(a.gamma_q, a.gamma_f32, lane, a.D, gamma[0][0], gamma[0][1]);
        load_gamma<T>(a.heads_k > 0 ? a.gamma_k : a.gamma_q, a.gamma_f32, lane, a.D, gamma[1][0], gamma[1][1]);
    }
    for (int64_t t0 = (int64_t)blockIdx.x * a.per_block; t0 < a.tokens; t0 += (int64_t)gridDim.x * a.per_block) {
        const int n_tokens = (int)(a.tokens - t0 < a.per_block ? a.tokens - t0 : a.per_block);
        const uint32_t items = (uint32_t)n_tokens * heads;
        struct Item {
            uint32_t token, head;
            Raw<T> x, y;
        };
        auto load = [&](uint32_t n, Item &i) __attribute__((always_inline)) {
            if (n >= items) return;
            i.token = quotient(n, heads, a.heads_inverse, i.head);
            const bool q = i.head < (uint32_t)a.heads_q, k = i.head < (uint32_t)(a.heads_q + a.heads_k);
            const Matrix &m = q ? a.q : (k ? a.k : a.v);
            const T *const from = m.at<const T>(t0 + i.token, i.head - (q ? 0u : (k ? (uint32_t)a.heads_q : (uint32_t)(a.heads_q + a.heads_k))));
            i.x = load_raw<kOnce, false>(from, first, a.D);
            i.y = load_raw<kOnce, false>(from, second, a.D);
        };
        Item now, next;
        uint32_t n = threadIdx.x / G;
        load(n, now);
        __syncthreads();  // (the turns and places of the group before are read)
        if constexpr (kAppend) {
            const int token = threadIdx.x >> 6;
            if (token < n_tokens) {
                const int64_t t = t0 + token, b = sequence_of(a.starts, a.sequences, t);
                uint32_t row = kNoRow;
                if (b >= 0) {
                    const int64_t at = (int64_t)a.lengths[b] - (a.starts[b + 1] - t);
                    if (at >= 0) row = paged::row_of(a.pages, paged::place_of(a.pages, b, (uint32_t)at), 0u);
                }
                if ((threadIdx.x & 63) == 0) places[token] = row, known[token] = b >= 0;
            }
        }
        turns_of(a.angles, t0, n_tokens, turns);
        __syncthreads();
        for (; n < items; n += kThreads / G) {
            load(n + kThreads / G, next);
            const bool q = now.head < (uint32_t)a.heads_q, k = now.head < (uint32_t)(a.heads_q + a.heads_k);
            float x[kVec], y[kVec];
#pragma unroll
            for (int i = 0; i < kVec; ++i) x[i] = lane.on ? (float)now.x.e[i] : 0.0f, y[i] = lane.on ? (float)now.y.e[i] : 0.0f;
            if (!kAppend || q || k) {
                if (a.gamma_q) {
                    float sum = 0.0f;
#pragma unroll
                    for (int i = 0; i < kVec; ++i) sum = __fmaf_rn(x[i], x[i], sum), sum = __fmaf_rn(y[i], y[i], sum);
                    float r = head_factor(sum_of_head<G>(sum), a.inverse_D, a.eps);
                    if (magnitude(r) == 0x7F800000u) {  // (the same for all lanes of the head)
                        uint32_t top = 0u;
#pragma unroll
                        for (int i = 0; i < kVec; ++i) top = max(top, max(magnitude(x[i]), magnitude(y[i])));
                        if (most_of_head<G>(top) == 0u) r = 0.0f;
                    }
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        x[i] = x[i] * r * (q ? gamma[0][0][i] : gamma[1][0][i]);
                        y[i] = y[i] * r * (q ? gamma[0][1][i] : gamma[1][1][i]);
                    }
                }
                turn<1>(lane, turns[now.token], x, y);
            }
            if (!kAppend || q) {
                const Matrix &m = q ? a.q_out : a.k_out;
                T *const to = m.at<T>(t0 + now.token, now.head - (q ? 0u : (uint32_t)a.heads_q));
                if (lane.on && (!kAppend || known[now.token])) {
                    store_values<kOnce, false>(to, first, a.D, x);
                    store_values<kOnce, false>(to, second, a.D, y);
                }
            } else {
                uint32_t top = 0u;
#pragma unroll
                for (int i = 0; i < kVec; ++i) top = max(top, lane.on ? max(magnitude(x[i]), magnitude(y[i])) : 0u);
                const ExactQuantizer quantizer(most_of_head<G>(top), 1.0f);
                const uint32_t place = places[now.token], head = now.head - (uint32_t)(a.heads_q + (k ? 0 : a.heads_k));
                if (place != kNoRow && lane.on) {
                    const uint32_t row = place + head * a.pages.page;
                    int8_t *const to = (k ? a.codes_k : a.codes_v) + (int64_t)row * a.D;
                    store_codes<false>(to, first, a.D, quantizer, x);
                    store_codes<false>(to, second, a.D, quantizer, y);
                    if (unit == 0) (k ? a.scale_k : a.scale_v)[row] = quantizer.scale;
                }
            }
            now = next;
        }
    }
}

// Gradient (formulas in qnn.h).  The first blocks_q workgroups take the queries' heads, the others the keys'; each goes through every so many groups of tokens, keeps its lanes' part of
// the weight's gradient in registers over all of them and writes it once; a second kernel adds these parts in a fixed order.
struct HeadsGradArgs {
    Matrix grad[2], h[2], out[2];
    const void *gamma[2];
    bool gamma_f32;
    float eps, inverse_D;
    Angles angles;
    int64_t tokens;
    int32_t D, per_block, heads[2], blocks[2];
    uint32_t heads_inverse[2];
    float *parts;
};

template <typename T, int G, bool kOnce>
__global__ __launch_bounds__(kThreads) void heads_backward_kernel(const HeadsGradArgs a) {
    __shared__ float2 turns[kMostTokens][kMostPairs];
    __shared__ float joined[kThreads][17];
    const int side = blockIdx.x < (unsigned)a.blocks[0] ? 0 : 1, block = (int)blockIdx.x - (side ? a.blocks[0] : 0), blocks = a.blocks[side];
    const Matrix grad = a.grad[side], h = a.h[side], out = a.out[side];
    const void *const gamma = a.gamma[side];
    const uint32_t heads = (uint32_t)a.heads[side], heads_inverse = a.heads_inverse[side];
    const int unit = threadIdx.x % G;
    const Lane lane(unit, a.D, a.angles);
    const Window first(lane.first, a.D), second(lane.second, a.D);
    float gx[kVec], gy[kVec], sx[kVec], sy[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) gx[i] = gy[i] = 1.0f, sx[i] = sy[i] = 0.0f;
    if (gamma) load_gamma<T>(gamma, a.gamma_f32, lane, a.D, gx, gy);
    for (int64_t t0 = (int64_t)block * a.per_block; t0 < a.tokens; t0 += (int64_t)blocks * a.per_block) {
        const int n_tokens = (int)(a.tokens - t0 < a.per_block ? a.tokens - t0 : a.per_block);
        __syncthreads();  // (the turns of the group before are read)
        turns_of(a.angles, t0, n_tokens, turns);
        __syncthreads();
        const uint32_t items = (uint32_t)n_tokens * heads;
        for (uint32_t n = threadIdx.x / G; n < items; n += kThreads / G) {
            uint32_t head;
            const uint32_t token = quotient(n, heads, heads_inverse, head);
            const T *const from = grad.at<const T>(t0 + token, head);
            const Raw<T> g0 = load_raw<kOnce, false>(from, first, a.D), g1 = load_raw<kOnce, false>(from, second, a.D);
            Raw<T> h0, h1;
            if (gamma) {
                const T *const values = h.at<const T>(t0 + token, head);
                h0 = load_raw<kOnce, false>(values, first, a.D), h1 = load_raw<kOnce, false>(values, second, a.D);
            }
            float x[kVec], y[kVec];
#pragma unroll
            for (int i = 0; i < kVec; ++i) x[i] = lane.on ? (float)g0.e[i] : 0.0f, y[i] = lane.on ? (float)g1.e[i] : 0.0f;
            turn<-1>(lane, turns[token], x, y);
            if (gamma) {
                float u[kVec], v[kVec], sum = 0.0f, dot = 0.0f;
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    u[i] = lane.on ? (float)h0.e[i] : 0.0f, v[i] = lane.on ? (float)h1.e[i] : 0.0f;
                    sum = __fmaf_rn(u[i], u[i], sum), sum = __fmaf_rn(v[i], v[i], sum);
                    dot = __fmaf_rn(gx[i] * x[i], u[i], dot), dot = __fmaf_rn(gy[i] * y[i], v[i], dot);
                }
                const float r = head_factor(sum_of_head<G>(sum), a.inverse_D, a.eps), c = r * r * (sum_of_head<G>(dot) * a.inverse_D);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    sx[i] = __fmaf_rn(x[i], u[i] * r, sx[i]), sy[i] = __fmaf_rn(y[i], v[i] * r, sy[i]);
                    x[i] = r * __fmaf_rn(-u[i], c, gx[i] * x[i]), y[i] = r * __fmaf_rn(-v[i], c, gy[i] * y[i]);
                }
            }
            if (lane.on) {
                T *const to = out.at<T>(t0 + token, head);
                store_values<kOnce, false>(to, first, a.D, x);
                store_values<kOnce, false>(to, second, a.D, y);
            }
        }
    }
    if (!gamma) return;
#pragma unroll
    for (int i = 0; i < kVec; ++i) joined[threadIdx.x][i] = sx[i], joined[threadIdx.x][kVec + i] = sy[i];
    __syncthreads();
    // value i of unit u, over the heads that the workgroup has at a time
    for (int x = threadIdx.x; x < 2 * kVec * (a.D / 16); x += kThreads) {
        const int u = x / (2 * kVec), i = x % (2 * kVec);
        float s = 0.0f;
        for (int group = 0; group < kThreads / G; ++group) s += joined[group * G + u][i];
        const Lane at(u, a.D, a.angles);
        a.parts[(int64_t)blockIdx.x * a.D + (i < kVec ? at.first + i : at.second + i - kVec)] = s;
    }
}

constexpr int64_t kResident = 4, kMostBlocks = 1024;  // workgroups of heads_kernel on a compute unit; of the gradient, at most

// Workgroups of the two sides: in proportion to their heads, and so that all have the same number of groups or one less
struct Split {
    int64_t q, k;
};
Split limits_of(int64_t heads_q, int64_t heads_k) {
    auto of = [&](int64_t heads) -> int64_t {
        const int64_t most = kMostBlocks * heads / (heads_q + heads_k);
        return heads == 0 ? 0 : (most < 1 ? 1 : most);
    };
    return {of(heads_q), of(heads_k)};
}
Split split_of(int64_t tokens, int64_t heads_q, int64_t heads_k, int64_t per_block) {
    const int64_t groups = ceil_div(tokens, per_block);
    const Split limits = limits_of(heads_q, heads_k);
    auto of = [&](int64_t limit) -> int64_t { return limit == 0 ? 0 : ceil_div(groups, ceil_div(groups, limit)); };
    return {of(limits.q), of(limits.k)};
}
// Tokens that a workgroup takes at a time: one while there are few, so that they spread over the card
int tokens_per_block(int64_t tokens) { return tokens < 4 * 1024 ? 1 : kMostTokens; }
int tokens_per_group(int64_t tokens) { return tokens < 512 ? 1 : kMostTokens; }  // of the gradient

int check_heads(const char *what, const Matrix &m, int64_t heads, int64_t D, int64_t tokens, int type) {
    if (heads == 0) return QNN_OK;
    if (!paged::heads_fit(m.ld, m.step, heads, D, tokens)) return fail(QNN_ERR_SHAPE, "%s: heads of %lld values at strides %lld, %lld overlap", what, (long long)D, (long long)m.ld, (long long)m.step);
    if (!m.p) return fail(QNN_ERR_NULL, "%s: NULL pointer", what);
    if (!aligned_to(m.p, value_bytes(type))) return fail(QNN_ERR_ALIGN, "%s: pointer not aligned to its type", what);
    return QNN_OK;
}

int check_common(const char *what, int64_t tokens, int64_t D, int64_t heads_q, int64_t heads_k, int type, const void *gamma_q, const void *gamma_k, int gamma_type, float eps,
                 const qnn_rotation *r) {
    if (tokens < 0 || tokens > 0x7FFFFFFF || heads_q < 0 || heads_k < 0 || heads_q + heads_k < 1 || heads_q > 65535 || heads_k > 65535)
        return fail(QNN_ERR_SHAPE, "%s: %lld tokens, %lld and %lld heads", what, (long long)tokens, (long long)heads_q, (long long)heads_k);
    if (D < 16 || D > paged::kMostD || D % 16) return fail(QNN_ERR_UNSUPPORTED, "%s: heads of %lld values (a multiple of 16, at most 256)", what, (long long)D);
    if (!known_type(type) || ((gamma_q || gamma_k) && gamma_type != QNN_F32 && gamma_type != type))
        return fail(QNN_ERR_SHAPE, "%s: types %d, %d (gamma: float32, or as the heads)", what, type, gamma_type);
    if (!(eps >= 0.0f) || eps > 3.0e38f) return fail(QNN_ERR_SHAPE, "%s: eps = %g", what, (double)eps);
    if ((heads_q > 0 && heads_k > 0 && !gamma_q != !gamma_k) || (heads_q == 0 && gamma_q) || (heads_k == 0 && gamma_k))
        return fail(QNN_ERR_SHAPE, "%s: a gamma for queries and keys, or for neither", what);
    if ((gamma_q && !aligned_to(gamma_q, value_bytes(gamma_type))) || (gamma_k && !aligned_to(gamma_k, value_bytes(gamma_type))))
        return fail(QNN_ERR_ALIGN, "%s: gamma not aligned to its type", what);
    if (!r) return fail(QNN_ERR_NULL, "%s: NULL rotation", what);
    if (r->pairs < 0 || r->pairs % 8 || 2 * (int64_t)r->pairs > D || (r->pairs > 0 && (r->axes < 1 || r->ld_positions < 0 || (r->axes > 1 && r->ld_positions < tokens))))
        return fail(QNN_ERR_SHAPE, "%s: %d pairs (a multiple of 8, at most half of %lld), %d axes of %lld positions", what, r->pairs, (long long)D, r->axes, (long long)r->ld_positions);
    return QNN_OK;
}
int check_rotation_pointers(const char *what, const qnn_rotation &r) {
    if (r.pairs == 0) return QNN_OK;
    if (!r.positions || !r.freq) return fail(QNN_ERR_NULL, "%s: NULL pointer in the rotation", what);
    if (!aligned_to(r.positions, 4) || !aligned_to(r.freq, 8) || !aligned_to(r.axis, 4)) return fail(QNN_ERR_ALIGN, "%s: pointer in the rotation not aligned to its type", what);
    return QNN_OK;
}
Angles angles_of(const qnn_rotation &r) {
    return {r.positions, r.axis, r.freq, r.ld_positions, r.axes, r.pairs, r.neighbours, r.pairs > 0 ? inverse_of(r.pairs) : 0u};
}

// f(integral_constant of the lanes of a head)
template <typename F>
int with_lanes(int64_t D, F f) {
    if (D <= 64) return f(std::integral_constant<int, 4>{});
    if (D <= 128) return f(std::integral_constant<int, 8>{});
    return f(std::integral_constant<int, 16>{});
}

template <bool kAppend>
int launch_heads(const char *what, int type, HeadsArgs a, hipStream_t s) {
    a.per_block = tokens_per_block(a.tokens);
    a.heads_inverse = inverse_of(a.heads_q + (kAppend ? 2 : 1) * a.heads_k);
    // as many workgroups as are resident, each with the same number of groups of tokens or one less
    const int64_t groups = ceil_div(a.tokens, a.per_block);
    const dim3 grid((unsigned)ceil_div(groups, ceil_div(groups, kResident * (int64_t)compute_units())));
    return with_type(type, [&](auto tag) {
        typedef decltype(tag) T;
        return with_lanes(a.D, [&](auto lanes) {
            constexpr int G = decltype(lanes)::value;
            const double values = 2.0 * (double)a.tokens * a.D * (a.heads_q + a.heads_k);
            auto kernel = beyond_caches(sizeof(T) * values) ? heads_kernel<T, G, kAppend, true> : heads_kernel<T, G, kAppend, false>;
            return QNN_LAUNCH(what, kernel, grid, dim3(kThreads), 0, s, a);
        });
    });
}

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" int qnn_qk_norm_rotate(const void *q, int64_t ld_q, int64_t step_q, int64_t heads_q, const void *k, int64_t ld_k, int64_t step_k, int64_t heads_k, int type,
                                  const void *gamma_q, const void *gamma_k, int gamma_type, float eps, const qnn_rotation *rotation, int64_t tokens, int64_t D,
                                  void *q_out, int64_t ld_q_out, int64_t step_q_out, void *k_out, int64_t ld_k_out, int64_t step_k_out, void *stream) {
    const char *const what = "qk_norm_rotate";
    if (int rc = check_common(what, tokens, D, heads_q, heads_k, type, gamma_q, gamma_k, gamma_type, eps, rotation)) return rc;
    if (tokens == 0) return QNN_OK;
    HeadsArgs a = {};
    a.q = {q, ld_q, step_q}, a.k = {k, ld_k, step_k}, a.q_out = {q_out, ld_q_out, step_q_out}, a.k_out = {k_out, ld_k_out, step_k_out};
    for (const Matrix *m : {&a.q, &a.q_out})
        if (int rc = check_heads(what, *m, heads_q, D, tokens, type)) return rc;
    for (const Matrix *m : {&a.k, &a.k_out})
        if (int rc = check_heads(what, *m, heads_k, D, tokens, type)) return rc;
    if (int rc = check_rotation_pointers(what, *rotation)) return rc;
    a.gamma_q = gamma_q ? gamma_q : gamma_k, a.gamma_k = gamma_k, a.gamma_f32 = gamma_type == QNN_F32, a.eps = eps;
    a.angles = angles_of(*rotation), a.tokens = tokens, a.D = (int32_t)D, a.inverse_D = 1.0f / (float)D, a.heads_q = (int32_t)heads_q, a.heads_k = (int32_t)heads_k;
    return launch_heads<false>(what, type, a, static_cast<hipStream_t>(stream));
}

extern "C" size_t qnn_qk_norm_rotate_backward_workspace_bytes(int64_t tokens, int64_t heads_q, int64_t heads_k, int64_t D) {
    if (tokens < 1 || tokens > 0x7FFFFFFF || heads_q < 0 || heads_k < 0 || heads_q > 65535 || heads_k > 65535 || heads_q + heads_k < 1 || D < 16 || D > paged::kMostD) return 0;
    // (more tokens may have fewer workgroups, but never need less)
    const Split limits = limits_of(heads_q, heads_k);
    return (size_t)((tokens < limits.q ? tokens : limits.q) + (tokens < limits.k ? tokens : limits.k)) * (size_t)D * 4;
}

extern "C" int qnn_qk_norm_rotate_backward(const void *grad_q, int64_t ld_grad_q, int64_t step_grad_q, const void *grad_k, int64_t ld_grad_k, int64_t step_grad_k,
                                           const void *q, int64_t ld_q, int64_t step_q, int64_t heads_q, const void *k, int64_t ld_k, int64_t step_k, int64_t heads_k,
                                           int type, const void *gamma_q, const void *gamma_k, int gamma_type, float eps, const qnn_rotation *rotation,
                                           int64_t tokens, int64_t D, void *out_q, int64_t ld_out_q, int64_t step_out_q, void *out_k, int64_t ld_out_k,
                                           int64_t step_out_k, float *grad_gamma_q, float *grad_gamma_k, void *workspace, size_t workspace_bytes, void *stream) {
    const char *const what = "qk_norm_rotate_backward";
    if (int rc = check_common(what, tokens, D, heads_q, heads_k, type, gamma_q, gamma_k, gamma_type, eps, rotation)) return rc;
    const bool norm = gamma_q || gamma_k;
    if (tokens == 0 && norm) return fail(QNN_ERR_SHAPE, "%s: no tokens", what);
    if (tokens == 0) return QNN_OK;
    HeadsGradArgs a = {};
    a.grad[0] = {grad_q, ld_grad_q, step_grad_q}, a.grad[1] = {grad_k, ld_grad_k, step_grad_k};
    a.h[0] = {q, ld_q, step_q}, a.h[1] = {k, ld_k, step_k};
    a.out[0] = {out_q, ld_out_q, step_out_q}, a.out[1] = {out_k, ld_out_k, step_out_k};
    const int64_t heads[2] = {heads_q, heads_k};
    float *const grad_gamma[2] = {grad_gamma_q, grad_gamma_k};
    a.gamma[0] = gamma_q, a.gamma[1] = gamma_k;
    for (int i = 0; i < 2; ++i) {
        for (const Matrix *m : {&a.grad[i], &a.out[i]})
            if (int rc = check_heads(what, *m, heads[i], D, tokens, type)) return rc;
        if (norm)
            if (int rc = check_heads(what, a.h[i], heads[i], D, tokens, type)) return rc;
        if (norm && heads[i] > 0 && !grad_gamma[i]) return fail(QNN_ERR_NULL, "%s: NULL pointer", what);
        if (!aligned_to(grad_gamma[i], 4)) return fail(QNN_ERR_ALIGN, "%s: gradient of gamma not aligned to its type", what);
    }
    if (int rc = check_rotation_pointers(what, *rotation)) return rc;
    const size_t need = norm ? qnn_qk_norm_rotate_backward_workspace_bytes(tokens, heads_q, heads_k, D) : 0;
    if (need > 0 && (!workspace || !aligned_to(workspace, 256) || workspace_bytes < need))
        return fail(QNN_ERR_WORKSPACE, "%s: workspace NULL, misaligned or smaller than %zu bytes", what, need);
    a.gamma_f32 = gamma_type == QNN_F32, a.eps = eps, a.angles = angles_of(*rotation), a.tokens = tokens, a.D = (int32_t)D, a.inverse_D = 1.0f / (float)D;
    a.per_block = tokens_per_group(tokens), a.parts = static_cast<float *>(workspace);
    const Split split = split_of(tokens, heads_q, heads_k, a.per_block);
    a.blocks[0] = (int32_t)split.q, a.blocks[1] = (int32_t)split.k;
    for (int i = 0; i < 2; ++i) a.heads[i] = (int32_t)heads[i], a.heads_inverse[i] = inverse_of(heads[i] > 0 ? heads[i] : 1);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int rc = with_type(type, [&](auto tag) {
        typedef decltype(tag) T;
        return with_lanes(D, [&](auto lanes) {
            constexpr int G = decltype(lanes)::value;
            auto kernel = beyond_caches(sizeof(T) * (norm ? 3.0 : 2.0) * (double)tokens * (double)(heads_q + heads_k) * (double)D) ? heads_backward_kernel<T, G, true>
                                                                                                                                     : heads_backward_kernel<T, G, false>;
            return QNN_LAUNCH(what, kernel, dim3((unsigned)(split.q + split.k)), dim3(kThreads), 0, s, a);
        });
    });
    if (rc || !norm) return rc;
    const AddParts q_parts = {a.parts, (int32_t)split.q, grad_gamma_q}, k_parts = {a.parts + split.q * D, (int32_t)split.k, grad_gamma_k};
    const bool both = heads_q > 0 && heads_k > 0;
    return QNN_LAUNCH(what, add_parts_kernel, dim3((unsigned)ceil_div(D, 32), both ? 2 : 1), dim3(1024), 0, s, heads_q > 0 ? q_parts : k_parts, k_parts, D);
}

extern "C" int qnn_cache_append(const qnn_paged_cache *cache, const void *q, int64_t ld_q, int64_t step_q, int64_t heads_q, const void *k, int64_t ld_k, int64_t step_k,
                                const void *v, int64_t ld_v, int64_t step_v, int type, const void *gamma_q, const void *gamma_k, int gamma_type, float eps,
                                const qnn_rotation *rotation, int64_t tokens, void *q_out, int64_t ld_q_out, int64_t step_q_out, void *stream) {
    const char *const what = "cache_append";
    if (int rc = paged::check_cache(what, cache)) return rc;
    const int64_t D = cache->D;
    if (int rc = check_common(what, tokens, D, heads_q, cache->heads, type, gamma_q, gamma_k, gamma_type, eps, rotation)) return rc;
    if (tokens == 0 || cache->sequences == 0) return QNN_OK;
    HeadsArgs a = {};
    a.q = {q, ld_q, step_q}, a.k = {k, ld_k, step_k}, a.v = {v, ld_v, step_v}, a.q_out = {q_out, ld_q_out, step_q_out};
    for (const Matrix *m : {&a.q, &a.q_out})
        if (int rc = check_heads(what, *m, heads_q, D, tokens, type)) return rc;
    for (const Matrix *m : {&a.k, &a.v})
        if (int rc = check_heads(what, *m, cache->heads, D, tokens, type)) return rc;
    if (int rc = check_rotation_pointers(what, *rotation)) return rc;
    if (int rc = paged::check_cache_pointers(what, cache)) return rc;
    a.gamma_q = gamma_q ? gamma_q : gamma_k, a.gamma_k = gamma_k, a.gamma_f32 = gamma_type == QNN_F32, a.eps = eps;
    a.angles = angles_of(*rotation), a.tokens = tokens, a.D = (int32_t)D, a.inverse_D = 1.0f / (float)D, a.heads_q = (int32_t)heads_q, a.heads_k = (int32_t)cache->heads;
    a.pages = paged::pages_of(*cache), a.starts = cache->starts, a.lengths = cache->lengths, a.sequences = cache->sequences;
    a.codes_k = cache->k, a.codes_v = cache->v, a.scale_k = cache->k_scale, a.scale_v = cache->v_scale;
    return launch_heads<true>(what, type, a, static_cast<hipStream_t>(stream));
}
