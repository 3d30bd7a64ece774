// Mixture-of-experts layer on int8 codes for a few tokens, in two kernels.  What bounds it is reading the chosen experts' weights once.
//   moe_gate_up_kernel: a workgroup has 16 columns of one expert's inner width, that is 32 rows of W1, and all the tokens that chose the expert; which
//     tokens these are it finds itself from the logits.  The activation goes to the workspace in fp32, beside the largest magnitude of each token's 16
//     values; the expert's first workgroup also writes the tokens' weights.
//   moe_down_kernel: a workgroup has 16 columns of the output, that is 16 rows of every expert's W2.  It quantizes the activations as it reads them (a
//     row's scale is known once the first kernel has ended), multiplies expert by expert and adds the weighted results in the order of the choices.
// Both give 16 x 16 blocks of sums to the matrix cores, with the weights on the row side, and split k over their waves.
#include "qnn_int8.h"

namespace qnn {
namespace int8 {
namespace {

using rows::magnitude;
using rows::Quantizer;

static_assert(QNN_MOE_MAX_TOKENS == 64, "one lane a token");

struct Route {  // a choice of a token: `weight` is exp(logit - largest logit); NaN: the token's logits say nothing; 0: takes no part
    int32_t expert;
    float weight;
};

struct MoeArgs {
    const int8_t *x, *W1, *W2;
    const float *scale_x, *logits, *scale1, *scale2;
    int64_t ldx, ld_logits, ld_w1, ld_w2, H, F, ldo;
    int tokens, experts, top;
    // workspace: [tokens * top] routes, [tokens * top][F] activations, [tokens * top][ceil(F / 16)] largest magnitudes
    Route *route;
    float *act;
    uint32_t *tops;
    int64_t chunks;
};

// Lane t: where expert e stands among the choices of token t, 0 the first (top or more: not chosen), and its weight
__device__ __forceinline__ int rank_of(const MoeArgs &a, int e, int t, float &weight) {
    const float *const l = a.logits + (int64_t)(t < a.tokens ? t : 0) * a.ld_logits;
    const float mine = l[e];
    auto key = [](float v) __attribute__((always_inline)) {  // an unsigned integer in the order of the values; NaN somewhere, but a total order
        const uint32_t b = __float_as_uint(v + 0.0f);        // (-0 counts as +0)
        return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    };
    const uint32_t own = key(mine);
    int rank = 0;
    float top = -INFINITY;
    bool nan = false;
    for (int j = 0; j < a.experts; ++j) {
        const float v = l[j];
        const uint32_t k = key(v);
        rank += k > own || (k == own && j < e);
        top = fmaxf(top, v);
        nan |= v != v;
    }
    weight = nan || top == INFINITY ? __uint_as_float(0x7FC00000u) : (top == -INFINITY ? 0.0f : expf(mine - top));
    return rank;
}

template <int kTiles>
__global__ __launch_bounds__(256) void moe_gate_up_kernel(const MoeArgs a) {
    constexpr int kWaves = 4;
    __shared__ int32_t sums[kWaves][2][16 * kTiles][17];
    __shared__ int list[64], slot_of[64];
    const int e = blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    float weight;
    const int rank = rank_of(a, e, lane, weight);
    const bool mine = lane < a.tokens && rank < a.top;
    if (mine && blockIdx.x == 0 && wave == 0) a.route[lane * a.top + rank] = Route{e, weight};
    const bool chosen = mine && weight > 0.0f;
    const uint64_t who = __ballot(chosen);
    const int count = __popcll(who);
    if (count == 0) return;
    if (wave == 0 && chosen) {
        const int at = __popcll(who & ((1ull << lane) - 1ull));
        list[at] = lane;
        slot_of[at] = lane * a.top + rank;
    }
    __syncthreads();
    const int64_t f0 = (int64_t)blockIdx.x * 16;
    const int8_t *w_row[2], *x_row[kTiles];
    const int64_t f_row = min(f0 + r, a.F - 1);
#pragma unroll
    for (int c = 0; c < 2; ++c) w_row[c] = a.W1 + ((int64_t)e * 2 * a.F + c * a.F + f_row) * a.ld_w1;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) x_row[t] = a.x + (int64_t)list[min(16 * t + r, count - 1)] * a.ldx;
    v4i acc[2][kTiles] = {};
    multiply_rows<2, kTiles, (kTiles == 1 ? 4 : 2)>(w_row, x_row, a.H, 64 * wave, 64 * kWaves, acc);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) sums[wave][c][16 * t + r][4 * g + v] = acc[c][t][v];
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * count; i += 256) {  // (16 lanes of a wave share a token)
        const int m = i >> 4, c = i & 15;
        const int64_t f = f0 + c;
        float y = 0.0f;
        if (f < a.F) {
            int32_t s0 = 0, s1 = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) s0 += sums[w][0][m][c], s1 += sums[w][1][m][c];
            const float sx = a.scale_x[list[m]];
            const float *const s = a.scale1 + (int64_t)e * 2 * a.F + f;
            const float gate = (float)s0 * sx * s[0], up = (float)s1 * sx * s[a.F];
            y = rows::silu(gate) * up;
            a.act[(int64_t)slot_of[m] * a.F + f] = y;
        }
        uint32_t top = magnitude(y);
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
        if (c == 0) a.tops[(int64_t)slot_of[m] * a.chunks + blockIdx.x] = top;
    }
}

template <typename T, int kTiles>
__global__ __launch_bounds__(512) void moe_down_kernel(const MoeArgs a, T *out) {
    constexpr int kWaves = 8, kRows = 16 * kTiles, kSlots = kRows * QNN_MOE_MAX_TOP;
    constexpr int kChunk = kTiles == 1 ? 2048 : 1024, kPitch = kChunk + 16;  // codes of the inner width that are in LDS at a time
    __shared__ __attribute__((aligned(16))) uint8_t codes[kRows * kPitch];
    __shared__ int32_t sums[kWaves][kRows][17];
    __shared__ float result[kSlots][16];
    __shared__ Route route[kSlots];
    __shared__ float mul[kSlots], pre[kSlots], scale[kSlots];
    __shared__ int order[kSlots], start[QNN_MOE_MAX_EXPERTS + 1];
    const int t = threadIdx.x, wave = t >> 6, lane = t & 63, r = lane & 15, g = lane >> 4, slots = a.tokens * a.top;
    const int64_t n0 = (int64_t)blockIdx.x * 16, n_row = min(n0 + r, a.H - 1);
    for (int s = t; s < slots; s += 512) {
        const Route c = a.route[s];
        route[s] = Route{c.weight > 0.0f ? c.expert : -1, c.weight};
    }
    __syncthreads();
    // how each activation is quantized
    for (int s = wave; s < slots; s += kWaves) {
        if (route[s].expert < 0) continue;
        uint32_t top = 0u;
        for (int64_t c = lane; c < a.chunks; c += 64) top = max(top, a.tops[(int64_t)s * a.chunks + c]);
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
        const Quantizer q(top, 1.0f);
        if (lane == 0) mul[s] = q.zero ? 0.0f : q.mul, pre[s] = q.zero ? 0.0f : q.pre, scale[s] = q.scale;
    }
    // the choices in the order of their experts
    if (wave == 0) {
        int at = 0;
        for (int e = 0; e < a.experts; ++e) {
            if (lane == 0) start[e] = at;
            for (int s0 = 0; s0 < slots; s0 += 64) {
                const bool is = s0 + lane < slots && route[s0 + lane].expert == e;
                const uint64_t who = __ballot(is);
                if (is) order[at + __popcll(who & ((1ull << lane) - 1ull))] = s0 + lane;
                at += __popcll(who);
            }
        }
        if (lane == 0) start[a.experts] = at;
    }
    __syncthreads();
    for (int e = 0; e < a.experts; ++e) {
        const int first = start[e], count = start[e + 1] - first;
        if (count == 0) continue;
        const int8_t *const w_row = a.W2 + ((int64_t)e * a.H + n_row) * a.ld_w2;
        v4i acc[kTiles] = {};
        for (int64_t f0 = 0; f0 < a.F; f0 += kChunk) {
            const int here = (int)min((int64_t)kChunk, a.F - f0), groups = (here + 63) / 64 * 16;  // groups of four codes, zeros up to a whole step
            for (int i = t; i < count * groups; i += 512) {
                const int m = i / groups, f = 4 * (i - m * groups), s = order[first + m];
                const float *const p = a.act + (int64_t)s * a.F + f0 + f;
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = f + j < here ? p[j] : 0.0f;
                uint32_t w = 0u;
                if (pre[s] != 0.0f) {
                    Quantizer q(0u, 1.0f);
                    q.mul = mul[s], q.pre = pre[s], q.zero = false;
                    w = q.four(v[0], v[1], v[2], v[3]);
                }
                *reinterpret_cast<uint32_t *>(&codes[m * kPitch + f]) = w;
            }
            __syncthreads();
            for (int k = 64 * wave; k < here; k += 64 * kWaves) {
                const v4i w = load16(w_row, f0 + k + 16 * g, a.F);
#pragma unroll
                for (int j = 0; j < kTiles; ++j) {
                    const v4i x = *reinterpret_cast<const v4i *>(&codes[(16 * j + r) * kPitch + k + 16 * g]);
                    acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, acc[j], 0, 0, 0);
                }
            }
            __syncthreads();
        }
#pragma unroll
        for (int j = 0; j < kTiles; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) sums[wave][16 * j + r][4 * g + v] = acc[j][v];
        __syncthreads();
        for (int i = t; i < 16 * count; i += 512) {
            const int s = order[first + (i >> 4)];
            int32_t total = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) total += sums[w][i >> 4][i & 15];
            result[s][i & 15] = (float)total * scale[s] * a.scale2[(int64_t)e * a.H + min(n0 + (i & 15), a.H - 1)];
        }
    }
    __syncthreads();
    for (int i = t; i < 16 * a.tokens; i += 512) {
        const int tok = i >> 4;
        const int64_t n = n0 + (i & 15);
        if (n >= a.H) continue;
        float whole = 0.0f, y = 0.0f;
        for (int j = 0; j < a.top; ++j) whole += route[tok * a.top + j].weight;
        for (int j = 0; j < a.top; ++j)
            if (route[tok * a.top + j].weight > 0.0f) y = __fmaf_rn(route[tok * a.top + j].weight / whole, result[tok * a.top + j][i & 15], y);
        out[(int64_t)tok * a.ldo + n] = (T)(whole == whole ? y : whole);
    }
}

size_t round_up_256(size_t v) { return (v + 255) / 256 * 256; }
size_t route_bytes(int64_t tokens, int top) { return round_up_256((size_t)(tokens * top) * sizeof(Route)); }
size_t act_bytes(int64_t tokens, int top, int64_t F) { return round_up_256((size_t)(tokens * top) * (size_t)F * 4); }
size_t tops_bytes(int64_t tokens, int top, int64_t F) { return round_up_256((size_t)(tokens * top) * (size_t)ceil_div(F, 16) * 4); }

template <int kTiles>
int launch_moe(const MoeArgs &a, void *out, int type, hipStream_t s) {
    if (int rc = QNN_LAUNCH("int8_moe", moe_gate_up_kernel<kTiles>, dim3((unsigned)a.chunks, (unsigned)a.experts), dim3(256), 0, s, a)) return rc;
    return rows::with_type(type, [&](auto tag) {
        typedef decltype(tag) T;
        return QNN_LAUNCH("int8_moe", (moe_down_kernel<T, kTiles>), dim3((unsigned)ceil_div(a.H, 16)), dim3(512), 0, s, a, static_cast<T *>(out));
    });
}

}  // namespace
}  // namespace int8
}  // namespace qnn

using namespace qnn;

extern "C" size_t qnn_int8_moe_workspace_bytes(int64_t tokens, int top, int64_t F) {
    if (tokens < 1 || tokens > QNN_MOE_MAX_TOKENS || top < 1 || top > QNN_MOE_MAX_TOP || F < 1 || F > int8::kMostK) return 0;
    return int8::route_bytes(tokens, top) + int8::act_bytes(tokens, top, F) + int8::tops_bytes(tokens, top, F);
}

extern "C" int qnn_int8_moe(const int8_t *x, int64_t ldx, const float *scale_x, const float *logits, int64_t ld_logits, int64_t tokens, int experts,
                            int top, int64_t H, int64_t F, const int8_t *W1, int64_t ld_w1, const float *scale1, const int8_t *W2, int64_t ld_w2,
                            const float *scale2, void *out, int64_t ldo, int type, void *workspace, size_t workspace_bytes, void *stream) {
    if (tokens < 0 || experts < 1 || top < 1 || top > experts || H < 1 || F < 1)
        return fail(QNN_ERR_SHAPE, "int8_moe: tokens = %lld, experts = %d, top = %d, H = %lld, F = %lld", (long long)tokens, experts, top, (long long)H, (long long)F);
    if (!rows::known_type(type)) return fail(QNN_ERR_SHAPE, "int8_moe: type %d", type);
    if (ldx < H || ld_logits < experts || ld_w1 < H || ld_w2 < F || ldo < H) return fail(QNN_ERR_SHAPE, "int8_moe: leading dimension too small");
    if (tokens > QNN_MOE_MAX_TOKENS || top > QNN_MOE_MAX_TOP || experts > QNN_MOE_MAX_EXPERTS)
        return fail(QNN_ERR_UNSUPPORTED, "int8_moe: %lld tokens, top %d of %d experts (at most %d, %d, %d)", (long long)tokens, top, experts,
                    QNN_MOE_MAX_TOKENS, QNN_MOE_MAX_TOP, QNN_MOE_MAX_EXPERTS);
    if (H > int8::kMostK || F > int8::kMostK) return fail(QNN_ERR_OVERFLOW, "int8_moe: sums over H = %lld or F = %lld products of codes do not fit int32", (long long)H, (long long)F);
    if (tokens == 0) return QNN_OK;
    if (!x || !scale_x || !logits || !W1 || !scale1 || !W2 || !scale2 || !out) return fail(QNN_ERR_NULL, "int8_moe: NULL pointer");
    if (!rows::aligned_to(scale_x, 4) || !rows::aligned_to(logits, 4) || !rows::aligned_to(scale1, 4) || !rows::aligned_to(scale2, 4) ||
        !rows::aligned_to(out, rows::value_bytes(type)))
        return fail(QNN_ERR_ALIGN, "int8_moe: pointer not aligned to its type");
    const size_t need = qnn_int8_moe_workspace_bytes(tokens, top, F);
    if (!workspace || !rows::aligned_to(workspace, 256) || workspace_bytes < need)
        return fail(QNN_ERR_WORKSPACE, "int8_moe: workspace NULL, misaligned or smaller than %zu bytes", need);
    uint8_t *const ws = static_cast<uint8_t *>(workspace);
    const size_t r = int8::route_bytes(tokens, top), v = int8::act_bytes(tokens, top, F);
    const int8::MoeArgs a = {x, W1, W2, scale_x, logits, scale1, scale2, ldx, ld_logits, ld_w1, ld_w2, H, F, ldo, (int)tokens, experts, top,
                             reinterpret_cast<int8::Route *>(ws), reinterpret_cast<float *>(ws + r), reinterpret_cast<uint32_t *>(ws + r + v), ceil_div(F, 16)};
    hipStream_t s = static_cast<hipStream_t>(stream);
    return tokens <= 16 ? int8::launch_moe<1>(a, out, type, s) : int8::launch_moe<4>(a, out, type, s);
}
