// Mixture-of-experts layer on int8 codes for a few tokens, in two to four kernels.  What bounds it is reading the chosen experts' weights once.
//   moe_route_kernel, for many logits or experts: the choices.
//   moe_gate_up_kernel: a workgroup has 16 columns of one expert's inner width, that is 32 rows of W1, and all the tokens that chose the expert; which
//     tokens these are it otherwise finds itself from the logits.  The activation goes to the workspace in fp32, beside the largest magnitude of each token's 16
//     values; the expert's first workgroup also writes the tokens' weights.
//   quant_rows_kernel (qnn_rows.h), for more than a few choices: the activations to codes.
//   moe_down_kernel: a workgroup has 16 columns of the output, that is 16 rows of every expert's W2.  For a few choices it quantizes the activations itself
//     (a row's scale is known once the first kernel has ended).  It multiplies expert by expert and adds the weighted results in the order of the choices.
// Both products give 16 x 16 blocks of sums to the matrix cores, with the weights on the row side, and split k over their waves.
// One token, two of 8 experts of 4096 x 2048 (50 MB): 8.9 + 6.9 us, of which 2 and 3 pass before the weights flow; 20 tokens (201 MB): 29.5 + 4.2 + 16.6.
#include "qnn_int8.h"

namespace qnn {
namespace int8 {
namespace {

using rows::magnitude;
using rows::Quantizer;

static_assert(QNN_MOE_MAX_TOKENS == 64, "one lane a token");

// With more logits or experts the choices are found by a kernel of their own, not by every workgroup.  Per call, in every workgroup and in a kernel: one token,
// 8 experts 16.6 and 18.3 us; 32 tokens, 16 experts 44.6 and 46.2; one token, 128 experts 24.2 and 22.1; 8 tokens, 128 experts 178 and 82.
constexpr int kRoutedFrom = 512, kRoutedExperts = 64;

constexpr int kRingBytes = 72 * 1024;  // LDS of the first kernel's operands: two workgroups on a compute unit

struct Route {  // a choice of a token: `weight` is exp(logit - largest logit); NaN: the token's logits say nothing; 0: takes no part
    int32_t expert;
    float weight;
};

struct MoeArgs {
    const int8_t *x, *W1, *W2;
    const float *scale_x, *logits, *scale1, *scale2;
    int64_t ldx, ld_logits, ld_w1, ld_w2, H, F, ldo;
    int tokens, experts, top;
    // workspace: [tokens * top] routes, [tokens * top][F] activations, [tokens * top][ceil(F / 16)] largest magnitudes, then
    Route *route;
    float *act;
    uint32_t *tops;
    int64_t chunks;
    // (for more than a few choices) [tokens * top][ld_codes] activations as codes and [tokens * top] scales
    int8_t *codes;
    float *scales;
    int64_t ld_codes;
};

// Activations as they are, to codes (qnn_rows.h)
struct PlainSource {
    struct Kept {};
    const float *x;
    int64_t ld;
    template <bool kShort>
    __device__ __forceinline__ void load(int64_t row, const rows::Window &w, int64_t K, float (&v)[rows::kVec], Kept &) const {
        const rows::Raw<float> r = rows::load_raw<false, kShort>(x + row * ld, w, K);
#pragma unroll
        for (int i = 0; i < rows::kVec; ++i) v[i] = r.e[i];
    }
    __device__ __forceinline__ float add(const Kept &, int, float sum) const { return sum; }
    __device__ __forceinline__ float factor(float, int64_t) const { return 1.0f; }
    template <bool kShort>
    __device__ __forceinline__ void keep(int64_t, const rows::Window &, int64_t, const Kept &) const {}
};

// A logit as an unsigned integer in the order of the values: -0 counts as +0, NaN is above all
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);
    return v != v ? 0xFFFFFFFFu : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
constexpr uint32_t kKeyOfInf = 0xFF800000u, kKeyOfMinusInf = 0x007FFFFFu;
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key ^ (key >> 31 ? 0x80000000u : 0xFFFFFFFFu)); }

// Words of a token's keys in LDS: whole groups of four, an odd number of them (lanes that read a column meet different banks)
__host__ __device__ constexpr int keys_pitch(int experts) { return 4 * (((experts + 3) / 4) | 1); }

// Where expert e stands among the choices of a token with these keys (zeros from the last to a group of four), 0 the first (top or more: not chosen), and its
// weight
__device__ __forceinline__ int rank_of(const uint32_t *keys, int experts, int e, float &weight) {
    const uint32_t own = keys[e];
    int rank = 0;
    uint32_t top = 0u;
    for (int j = 0; j < experts; j += 4) {
        const v4i k = *reinterpret_cast<const v4i *>(keys + j);
#pragma unroll
        for (int i = 0; i < 4; ++i) rank += (uint32_t)k[i] > own || ((uint32_t)k[i] == own && j + i < e), top = max(top, (uint32_t)k[i]);
    }
    weight = top >= kKeyOfInf ? __uint_as_float(0x7FC00000u) : (top == kKeyOfMinusInf ? 0.0f : expf(value_of(own) - value_of(top)));
    return rank;
}

// The n-th (from 0) of the experts with a nonzero in any[], -1 if there are fewer; by a wave
__device__ __forceinline__ int nth_of(const int *any, int n) {
    const int lane = threadIdx.x & 63;
    for (int x0 = 0; x0 < QNN_MOE_MAX_EXPERTS; x0 += 64) {
        uint64_t who = __ballot(any[x0 + lane] != 0);
        const int here = __popcll(who);
        if (n < here) {
            for (; n > 0; --n) who &= who - 1ull;
            return __builtin_amdgcn_readfirstlane(x0 + __ffsll((unsigned long long)who) - 1);
        }
        n -= here;
    }
    return -1;
}

// Choices of a token, a workgroup each
__global__ __launch_bounds__(QNN_MOE_MAX_EXPERTS) void moe_route_kernel(const MoeArgs a) {
    __shared__ __attribute__((aligned(16))) uint32_t keys[QNN_MOE_MAX_EXPERTS];
    const int t = threadIdx.x, tok = blockIdx.x;
    keys[t] = t < a.experts ? key_of(a.logits[(int64_t)tok * a.ld_logits + t]) : 0u;
    __syncthreads();
    if (t >= a.experts) return;
    float weight;
    const int rank = rank_of(keys, a.experts, t, weight);
    if (rank < a.top) a.route[tok * a.top + rank] = Route{t, weight};
}

// kTiles of 16 tokens: what a workgroup of the first kernel does once it knows its tokens
template <int kTiles, Layout kLayout>
__device__ __forceinline__ void gate_up(const MoeArgs &a, int e, int chunk, const int *list, const int *slot_of, const float *scale_of, int count,
                                        uint8_t *lds) {
    constexpr int kWaves = 4, kStages = kTiles == 1 ? 3 : (kTiles == 2 ? 2 : 1);
    typedef Stream<2, kTiles, kStages, kLayout> S;
    static_assert(S::kBytes * kWaves <= kRingBytes && kWaves * 2 * 16 * kTiles * 17 * 4 <= kRingBytes, "");
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int64_t f0 = (int64_t)chunk * 16;
    // (the scales of this thread's column on their way before the weights, behind which they would wait)
    const float *const scales = a.scale1 + (int64_t)e * 2 * a.F + min(f0 + (threadIdx.x & 15), a.F - 1);
    const float scale_gate = scales[0], scale_up = scales[a.F];
    v4i acc[2][kTiles] = {};
    S s;
    s.lds = lds + wave * S::kBytes;
    s.x_base = a.x, s.K = (uint32_t)a.H;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int c = 0; c < 2; ++c) s.off[c][h] = (typename S::Offset)((c * a.F + min(f0 + 8 * h + (lane >> 3), a.F - 1)) * a.ld_w1);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) s.off[2 + t][h] = (typename S::Offset)(list[min(16 * t + 8 * h + (lane >> 3), count - 1)] * a.ldx);
    }
    s.sums(a.W1 + (int64_t)e * 2 * a.F * a.ld_w1, 128u * wave, 128u * kWaves, acc);
    __syncthreads();
    int32_t(*const sums)[2][16 * kTiles][17] = reinterpret_cast<int32_t(*)[2][16 * kTiles][17]>(lds);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) sums[wave][c][16 * t + r][4 * g + v] = acc[c][t][v];
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * count; i += 64 * kWaves) {  // (16 lanes of a wave share a token)
        const int m = i >> 4, c = i & 15;
        const int64_t f = f0 + c;
        float y = 0.0f;
        if (f < a.F) {
            int32_t s0 = 0, s1 = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) s0 += sums[w][0][m][c], s1 += sums[w][1][m][c];
            const float gate = (float)s0 * scale_of[m] * scale_gate, up = (float)s1 * scale_of[m] * scale_up;
            y = rows::silu(gate) * up;
            a.act[(int64_t)slot_of[m] * a.F + f] = y;
        }
        uint32_t top = magnitude(y);
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
        if (c == 0) a.tops[(int64_t)slot_of[m] * a.chunks + chunk] = top;
    }
}

// Grid: 16 columns of the inner width x as many experts as can be chosen.  Where those are fewer than there are, a workgroup finds the one that is its own
// among the chosen (a workgroup for each of them that ended at once: 11.4 us for one token and two of 8 experts of 4096 x 2048, 8.9 like this).
// kRouted: the choices are known; else every workgroup finds them from the logits
template <Layout kLayout, bool kRouted>
__global__ __launch_bounds__(256) void moe_gate_up_kernel(const MoeArgs a, int chosen_at_most) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[kRingBytes];
    __shared__ int list[64], slot_of[64], any[QNN_MOE_MAX_EXPERTS];
    __shared__ float scale_of[64];
    const int t = threadIdx.x, wave = t >> 6, lane = t & 63, chunk = (int)(blockIdx.x / (uint32_t)chosen_at_most);
    int e = (int)(blockIdx.x % (uint32_t)chosen_at_most);
    any[t] = 0;
    static_assert(QNN_MOE_MAX_EXPERTS == 256, "one thread an expert");
    bool chosen;
    int slot;
    float my_scale;
    if constexpr (kRouted) {
        constexpr int kSlots = QNN_MOE_MAX_TOKENS * QNN_MOE_MAX_TOP;
        static_assert(kSlots == 512, "");
        __shared__ int expert[kSlots], slot_at[64];
        const int slots = a.tokens * a.top;
        int mine[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const Route c = a.route[min(t + 256 * j, slots - 1)];
            mine[j] = t + 256 * j < slots && c.weight > 0.0f ? c.expert : -1;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            expert[t + 256 * j] = mine[j];
            if (mine[j] >= 0) any[mine[j]] = 1;
        }
        __syncthreads();
        e = nth_of(any, e);
        if (e < 0) return;
        int count = 0;
        for (int s0 = 0; s0 < slots; s0 += 64) {
            const bool is = expert[s0 + lane] == e;
            const uint64_t who = __ballot(is);
            if (wave == 0 && is) slot_at[count + __popcll(who & ((1ull << lane) - 1ull))] = s0 + lane;
            count += __popcll(who);
        }
        __syncthreads();
        chosen = lane < count;
        slot = chosen ? slot_at[lane] : 0;
        my_scale = a.scale_x[(uint32_t)slot / (uint32_t)a.top];
    } else {
        my_scale = a.scale_x[min(lane, a.tokens - 1)];
        uint32_t *const keys = reinterpret_cast<uint32_t *>(lds);
        const int pitch = keys_pitch(a.experts), padded = (a.experts + 3) / 4 * 4;
        static_assert(kRoutedFrom * 4 * 2 + QNN_MOE_MAX_TOKENS * 16 <= kRingBytes, "");
        for (int i = t; i < a.tokens * padded; i += 256) {
            const int tok = (int)((uint32_t)i / (uint32_t)padded), x = i - tok * padded;
            const float v = a.logits[(int64_t)tok * a.ld_logits + min(x, a.experts - 1)];
            keys[tok * pitch + x] = x < a.experts ? key_of(v) : 0u;
        }
        __syncthreads();
        float weight;
        if (chosen_at_most < a.experts) {
            for (int i = t; i < a.tokens * a.experts; i += 256) {
                const int tok = (int)((uint32_t)i / (uint32_t)a.experts), x = i - tok * a.experts;
                if (rank_of(keys + tok * pitch, a.experts, x, weight) < a.top) any[x] = 1;
            }
            __syncthreads();
            e = nth_of(any, e);
            if (e < 0) return;
        }
        const int rank = rank_of(keys + min(lane, a.tokens - 1) * pitch, a.experts, e, weight);
        const bool mine = lane < a.tokens && rank < a.top;
        if (mine && chunk == 0 && wave == 0) a.route[lane * a.top + rank] = Route{e, weight};
        chosen = mine && weight > 0.0f;
        slot = lane * a.top + rank;
    }
    const uint64_t who = __ballot(chosen);
    const int count = __popcll(who);
    if (count == 0) return;
    if (wave == 0 && chosen) {
        const int at = __popcll(who & ((1ull << lane) - 1ull));
        list[at] = (int)((uint32_t)slot / (uint32_t)a.top);
        slot_of[at] = slot;
        scale_of[at] = my_scale;
    }
    __syncthreads();  // (the keys' place is free too)
    if (count <= 16)
        gate_up<1, kLayout>(a, e, chunk, list, slot_of, scale_of, count, lds);
    else if (count <= 32)
        gate_up<2, kLayout>(a, e, chunk, list, slot_of, scale_of, count, lds);
    else
        gate_up<4, kLayout>(a, e, chunk, list, slot_of, scale_of, count, lds);
}

// The choices that take part, expert by expert: order[] of the choices, active[] experts, start[] of each in order[] and the end.  By one wave; returns the
// number of experts.  (Within an expert in any order: each choice has its own result.)
template <int kSlots>
__device__ __forceinline__ int in_order(const MoeArgs &a, Route *route, int slots, int *order, int *active, int *start, int *place) {
    constexpr int kPer = (kSlots + 63) / 64;
    typedef Stream<1, 0, 1, kPieces> S;
    const int lane = threadIdx.x & 63;
    int expert[kPer], at[kPer];
    *reinterpret_cast<v4i *>(&place[4 * lane]) = v4i{0, 0, 0, 0};
    static_assert(QNN_MOE_MAX_EXPERTS == 256, "four a lane");
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int s = 64 * j + lane;
        const Route c = a.route[min(s, slots - 1)];
        expert[j] = s < slots && c.weight > 0.0f ? c.expert : -1;
        if (s < slots) route[s] = Route{expert[j], c.weight};
    }
    S::in_wave();
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (expert[j] >= 0) at[j] = atomicAdd(&place[expert[j]], 1);
    S::in_wave();
    const v4i count = *reinterpret_cast<const v4i *>(&place[4 * lane]);
    // choices in the low half, experts in the high one
    uint32_t own = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) own += (uint32_t)count[i] + (count[i] > 0 ? 0x10000u : 0u);
    uint32_t before = own;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t other = (uint32_t)__shfl_up((int)before, d);
        before += lane >= d ? other : 0u;
    }
    const uint32_t whole = (uint32_t)__shfl((int)before, 63);
    before -= own;
    v4i places;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        places[i] = (int)(before & 0xFFFFu);
        if (count[i] > 0) active[before >> 16] = 4 * lane + i, start[before >> 16] = places[i];
        before += (uint32_t)count[i] + (count[i] > 0 ? 0x10000u : 0u);
    }
    *reinterpret_cast<v4i *>(&place[4 * lane]) = places;
    if (lane == 0) start[whole >> 16] = (int)(whole & 0xFFFFu);
    S::in_wave();
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (expert[j] >= 0) order[place[expert[j]] + at[j]] = 64 * j + lane;
    return (int)(whole >> 16);
}

// Activations lie in LDS as codes, `chunk` of the inner width at a time and as many experts at a time as have up to kCodes / (chunk + 16) choices together
// (mostly everything at once); then every wave goes through its steps of k of one expert after the other without a break in its loads, and adds what it has
// of an expert to the results in LDS (whole numbers: in any order).
// kQuantize: the codes are made here, from the first kernel's activations and maxima, all at once; else they and their scales are in memory.  The first
// saves a launch, but every workgroup reads four times as much and makes all the codes (7 tokens, three of 5 experts of 1000 x 700: 10.8 us where two
// kernels took 4.2 + 9.8; 20 tokens, two of 8 experts of 4096 x 2048: 24.6 where two took 4.3 + 18.6).
template <typename T, int kSlots, int kCodes, int kStages, Layout kLayout, bool kQuantize>
__global__ __launch_bounds__(512) void moe_down_kernel(const MoeArgs a, T *out, int chunk) {
    constexpr int kWaves = 8;
    constexpr bool kFactors = kSlots <= 128;  // what a result is multiplied with has room in LDS
    typedef Stream<1, 0, kStages, kLayout> S;
    __shared__ __attribute__((aligned(16))) uint8_t ring[kWaves * S::kBytes], codes[kCodes];
    __shared__ int32_t result[kSlots][16];
    __shared__ float factor[kFactors ? kSlots : 1][16];
    __shared__ Route route[kSlots];
    __shared__ float mul[kQuantize ? kSlots : 1], pre[kQuantize ? kSlots : 1], scale[kSlots];
    __shared__ __attribute__((aligned(16))) int place[QNN_MOE_MAX_EXPERTS];
    __shared__ int order[kSlots], active[QNN_MOE_MAX_EXPERTS], start[QNN_MOE_MAX_EXPERTS + 1], n_active;
    const int t = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(t >> 6), lane = t & 63, r = lane & 15, g = lane >> 4, slots = a.tokens * a.top;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const uint32_t F = (uint32_t)a.F;
    const int pitch = chunk + 16, most = kCodes / pitch;
    // everything at once: rows of codes are in the order of the choices, else in that of the experts
    const bool at_once = kQuantize || (slots <= most && F <= (uint32_t)chunk);
    // kQuantize: 256 activations of a row by a wave, a load of whole lines; the first kItems of a wave's are on their way from here on
    constexpr int kItems = 4;
    float v[kItems][4];
    const uint32_t parts = ((uint32_t)chunk + 255u) / 256u, items = (uint32_t)slots * parts;
    const uint32_t inverse = (65535u + parts) / parts;  // item / parts = item * inverse / 65536: up to 32 rows in 20 KB are less than 128 items
    auto row_of = [&](uint32_t item) __attribute__((always_inline)) { return (item * inverse) >> 16; };
    auto fetch = [&](float (&to)[4], uint32_t item) __attribute__((always_inline)) {  // (the rows are followed by more than they lack to a group of four)
        const uint32_t m = row_of(item), f = (item - m * parts) * 256u + 4u * lane;
        __builtin_memcpy(to, a.act + (int64_t)m * a.F + min(f, F - 1u), 16);
#pragma unroll
        for (uint32_t j = 0; j < 4u; ++j) to[j] = f + j < F ? to[j] : 0.0f;
    };
    if constexpr (kQuantize) {
#pragma unroll
        for (int j = 0; j < kItems; ++j) fetch(v[j], min((uint32_t)(wave + kWaves * j), items - 1u));
    }
    // One wave finds the order of the choices; the others how each activation is quantized (for a choice that takes no part: nothing that is used).
    if (wave == 0) {
        const int n = in_order<kSlots>(a, route, slots, order, active, start, place);
        if (lane == 0) n_active = n;
    } else {
        for (int i = t - 64; i < 16 * slots; i += 448) result[i >> 4][i & 15] = 0;
        if constexpr (kQuantize) {
            for (int s = (t - 64) >> 4; s < slots; s += 28) {  // 16 lanes each
                uint32_t top = 0u;
                const uint32_t *const from = a.tops + (int64_t)s * a.chunks;
                for (int64_t c0 = 0; c0 < a.chunks; c0 += 128) {
                    uint32_t w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = from[min(c0 + 16 * j + r, a.chunks - 1)];
#pragma unroll
                    for (int j = 0; j < 8; ++j) top = max(top, w[j]);
                }
#pragma unroll
                for (int d = 8; d >= 1; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
                const Quantizer q(top, 1.0f);
                if (r == 0) mul[s] = q.zero ? 0.0f : q.mul, pre[s] = q.zero ? 0.0f : q.pre, scale[s] = q.scale;
            }
        } else {
            for (int s = t - 64; s < slots; s += 448) scale[s] = a.scales[s];
        }
    }
    __syncthreads();
    const int experts = __builtin_amdgcn_readfirstlane(n_active);
    // share of a choice in its token's output and the scales of its product (whole: the sum of the weights, NaN where the logits say nothing)
    auto share = [&](int m, int64_t n, float whole) __attribute__((always_inline)) {
        return route[m].weight > 0.0f ? route[m].weight / whole * (scale[m] * a.scale2[(int64_t)route[m].expert * a.H + n]) : 0.0f;
    };
    auto sum_of = [&](int tok) __attribute__((always_inline)) {
        float whole = 0.0f;
        for (int j = 0; j < a.top; ++j) whole += route[tok * a.top + j].weight;
        return whole;
    };
    S s;
    s.lds = ring + wave * S::kBytes;
    s.K = F;
#pragma unroll
    for (int h = 0; h < 2; ++h) s.off[0][h] = (typename S::Offset)(min(n0 + 8 * h + (lane >> 3), a.H - 1) * a.ld_w2);
    for (int from = 0, to; from < experts; from = to) {
        // the experts whose activations are in LDS together
        const int first_row = __builtin_amdgcn_readfirstlane(start[from]);
        to = at_once ? experts : from + 1;
        while (to < experts && __builtin_amdgcn_readfirstlane(start[to + 1]) - first_row <= most) ++to;
        const int n_rows = __builtin_amdgcn_readfirstlane(start[to]) - first_row;
        for (uint32_t f0 = 0; f0 < F; f0 += (uint32_t)chunk) {
            // the steps of all experts here, expert by expert, blocks of 128 of them: a wave has every eighth; the loads' cursor and the products'
            const int blocks = (int)((min(F, f0 + (uint32_t)chunk) - f0 + 127u) / 128u), all = blocks * (to - from);
            const int steps = all > wave ? (all - wave - 1) / kWaves + 1 : 0;
            int send_x = from + wave / blocks, send_block = wave % blocks, x = send_x, block = send_block;
            auto next = [&](int &x, int &block) __attribute__((always_inline)) {
                block += kWaves;
                const bool other = block >= blocks;
                while (block >= blocks) block -= blocks, ++x;
                return other;
            };
            const int8_t *w_base = a.W2;
            bool send_other = true;
            auto base = [&](int) __attribute__((always_inline)) {
                if (send_other) w_base = a.W2 + (int64_t)__builtin_amdgcn_readfirstlane(active[send_x]) * a.H * a.ld_w2;
                return w_base;
            };
            auto at = [&](int) __attribute__((always_inline)) {  // (called after base)
                const uint32_t k = f0 + 128u * (uint32_t)send_block;
                send_other = next(send_x, send_block);
                return k;
            };
            s.start(steps, base, at);
            if constexpr (kQuantize) {  // zeros from an activation's end to a whole step
                for (uint32_t i0 = wave; i0 < items; i0 += kWaves * kItems) {
                    if (i0 != (uint32_t)wave) {
#pragma unroll
                        for (uint32_t j = 0; j < kItems; ++j) fetch(v[j], min(i0 + kWaves * j, items - 1u));
                    }
#pragma unroll
                    for (uint32_t j = 0; j < kItems; ++j) {
                        const uint32_t i = i0 + kWaves * j;
                        if (i >= items) break;
                        const uint32_t m = row_of(i), f = (i - m * parts) * 256u + 4u * lane;
                        Quantizer q(0u, 1.0f);
                        q.mul = mul[m], q.pre = pre[m], q.zero = pre[m] == 0.0f;
                        if (f < (uint32_t)chunk) *reinterpret_cast<uint32_t *>(&codes[m * pitch + f]) = q.four(v[j][0], v[j][1], v[j][2], v[j][3]);
                    }
                }
            } else {  // 16 codes a lane, whole rows of the part (what lies beyond the inner width meets zeros), eight loads under way
                const uint32_t per_row = min((uint32_t)chunk, (uint32_t)a.ld_codes - f0) / 16u, n = (uint32_t)(at_once ? slots : n_rows) * per_row;
                for (uint32_t i0 = t; i0 < n; i0 += 8u * 512u) {
                    v4i c[8];
#pragma unroll
                    for (uint32_t j = 0; j < 8u; ++j) {
                        const uint32_t i = min(i0 + 512u * j, n - 1u), row = i / per_row;
                        const int m = at_once ? (int)row : order[first_row + (int)row];
                        __builtin_memcpy(&c[j], a.codes + (int64_t)m * a.ld_codes + f0 + 16u * (i - row * per_row), 16);
                    }
#pragma unroll
                    for (uint32_t j = 0; j < 8u; ++j) {
                        const uint32_t i = min(i0 + 512u * j, n - 1u), row = i / per_row;
                        *reinterpret_cast<v4i *>(&codes[(int)row * pitch + 16 * (int)(i - row * per_row)]) = c[j];
                    }
                }
            }
            if (kFactors && from == 0 && f0 == 0u) {
                for (int i = t; i < 16 * slots; i += 512) factor[i >> 4][i & 15] = share(i >> 4, min(n0 + (i & 15), a.H - 1), sum_of((i >> 4) / a.top));
            }
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // (weights may still be on their way)
            constexpr int kBlocks = kSlots < 64 ? kSlots / 16 : 4;  // of 16 tokens of an expert
            v4i acc[kBlocks];
            int row[kBlocks], choice[kBlocks], count = 0;
            auto enter = [&]() __attribute__((always_inline)) {  // expert x: asked for at the end of the step before, so that LDS answers while its weights come in
                const int first = __builtin_amdgcn_readfirstlane(start[x]);
                count = __builtin_amdgcn_readfirstlane(start[x + 1]) - first;
#pragma unroll
                for (int j = 0; j < kBlocks; ++j) {
                    const int pos = first + min(16 * j + r, count - 1);
                    choice[j] = order[pos], row[j] = (at_once ? choice[j] : pos - first_row) * pitch, acc[j] = v4i{0, 0, 0, 0};
                }
            };
            if (steps > 0) enter();
            s.run(steps, base, at, [&](int i, const typename S::Operands &o) __attribute__((always_inline)) {
                const int k = 128 * block + 16 * g;
                const bool other = next(x, block);
#pragma unroll
                for (int j = 0; j < kBlocks; ++j)
                    if (16 * j < count) {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(o.w[h][0], *reinterpret_cast<const v4i *>(&codes[row[j] + k + 64 * h]), acc[j], 0, 0, 0);
                        if (other && 16 * j + r < count) {
#pragma unroll
                            for (int w = 0; w < 4; ++w) atomicAdd(&result[choice[j]][4 * g + w], acc[j][w]);
                        }
                    }
                if (other && i + 1 < steps) enter();
            });
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
    }
    for (int q = t; q < 16 * a.tokens; q += 512) {
        const int tok = q >> 4, c = q & 15;
        const int64_t n = n0 + c;
        if (n >= a.H) continue;
        const float whole = sum_of(tok);
        float y = 0.0f;
        for (int j = 0; j < a.top; ++j) {
            const int m = tok * a.top + j;
            if (route[m].weight > 0.0f) y = __fmaf_rn(kFactors ? factor[m][c] : share(m, n, whole), (float)result[m][c], y);
        }
        out[(int64_t)tok * a.ldo + n] = (T)(whole == whole ? y : whole);
    }
}

size_t round_up_256(size_t v) { return (v + 255) / 256 * 256; }
size_t route_bytes(int64_t tokens, int top) { return round_up_256((size_t)(tokens * top) * sizeof(Route)); }
size_t act_bytes(int64_t tokens, int top, int64_t F) { return round_up_256((size_t)(tokens * top) * (size_t)F * 4); }
size_t tops_bytes(int64_t tokens, int top, int64_t F) { return round_up_256((size_t)(tokens * top) * (size_t)ceil_div(F, 16) * 4 + 16); }  // (and see fetch)
int64_t codes_pitch(int64_t F) { return ceil_div(F, 128) * 128; }
size_t codes_bytes(int64_t tokens, int top, int64_t F) { return round_up_256((size_t)(tokens * top) * (size_t)codes_pitch(F)); }
size_t scales_bytes(int64_t tokens, int top) { return round_up_256((size_t)(tokens * top) * 4); }

int launch_moe(const MoeArgs &a, void *out, int type, hipStream_t s) {
    const int most = a.tokens * a.top < a.experts ? a.tokens * a.top : a.experts;
    const dim3 grid((unsigned)(a.chunks * most));
    const bool pieces1 = in_pieces(a.x, a.ldx, a.tokens, a.H) && in_pieces(a.W1, a.ld_w1, 2 * a.F, a.H), pieces2 = in_pieces(a.W2, a.ld_w2, a.H, a.F);
    const bool routed = a.tokens * a.experts > kRoutedFrom || a.experts > kRoutedExperts;
    // weights past the caches (20 tokens, two of 8 experts of 4096 x 2048, 201 MB: 56.3 -> 49.4 us; one token, 50 MB, which stay: 16.6 -> 17.4)
    const bool once = pieces1 && pieces2 && rows::beyond_caches(3.0 * most * (double)a.F * (double)a.H);
    auto up = [&](auto pieces, auto pieces_once, auto any, auto short_rows) {
        return pieces1 ? (once ? pieces_once : pieces) : (a.H >= 16 ? any : short_rows);
    };
    auto gate_up = routed ? up(moe_gate_up_kernel<kPieces, true>, moe_gate_up_kernel<kPiecesOnce, true>, moe_gate_up_kernel<kAny, true>,
                               moe_gate_up_kernel<kShortRows, true>)
                          : up(moe_gate_up_kernel<kPieces, false>, moe_gate_up_kernel<kPiecesOnce, false>, moe_gate_up_kernel<kAny, false>,
                               moe_gate_up_kernel<kShortRows, false>);
    if (routed)
        if (int rc = QNN_LAUNCH("int8_moe", moe_route_kernel, dim3((unsigned)a.tokens), dim3(QNN_MOE_MAX_EXPERTS), 0, s, a)) return rc;
    if (int rc = QNN_LAUNCH("int8_moe", gate_up, grid, dim3(256), 0, s, a, most)) return rc;
    const int64_t whole = codes_pitch(a.F);
    const int slots = a.tokens * a.top;
    // a few choices: codes are made by the second kernel, two workgroups on a compute unit; many: LDS holds the results of all and the codes of one expert's 64
    // tokens at least
    constexpr int kFew = 20 * 1024, kMore = 88 * 1024, kMost = 64 * (1024 + 16);
    const bool few = slots <= 32 && slots * (whole + 16) <= kFew;
    if (!few) {
        const PlainSource act = {a.act, a.F};
        if (int rc = rows::launch_quant_rows("int8_moe", act, slots, a.F, a.codes, a.ld_codes, a.scales, s)) return rc;
    }
    return rows::with_type(type, [&](auto tag) {
        typedef decltype(tag) T;
        const dim3 columns((unsigned)ceil_div(a.H, 16)), threads(512);
        T *const o = static_cast<T *>(out);
        auto launch = [&](auto pieces, auto pieces_once, auto any, auto short_rows, int chunk) {
            return QNN_LAUNCH("int8_moe", (pieces2 ? (once ? pieces_once : pieces) : (a.F >= 16 ? any : short_rows)), columns, threads, 0, s, a, o, chunk);
        };
        // (Few steps under way where there is little to do: each one more is code to fetch, which a short kernel waits for.  One token, two of 8 experts of
        // 4096 x 2048: 6.8 us, with a third 7.15, with four 7.45; rows of any length, 7 tokens, three of 5 experts of 1000 x 700: four 9.9 where one took 9.3.)
        if (few)
            return launch(moe_down_kernel<T, 32, kFew, 2, kPieces, true>, moe_down_kernel<T, 32, kFew, 2, kPiecesOnce, true>,
                          moe_down_kernel<T, 32, kFew, 1, kAny, true>, moe_down_kernel<T, 32, kFew, 1, kShortRows, true>, (int)whole);
        const int chunk = whole <= 1024 || (slots <= 128 && slots * (whole + 16) <= kMore) ? (int)whole : 1024;
        if (slots <= 128)
            return launch(moe_down_kernel<T, 128, kMore, 3, kPieces, false>, moe_down_kernel<T, 128, kMore, 3, kPiecesOnce, false>,
                          moe_down_kernel<T, 128, kMore, 1, kAny, false>, moe_down_kernel<T, 128, kMore, 1, kShortRows, false>, chunk);
        return launch(moe_down_kernel<T, 512, kMost, 2, kPieces, false>, moe_down_kernel<T, 512, kMost, 2, kPiecesOnce, false>,
                      moe_down_kernel<T, 512, kMost, 1, kAny, false>, moe_down_kernel<T, 512, kMost, 1, kShortRows, false>, chunk);
    });
}

}  // namespace
}  // namespace int8
}  // namespace qnn

using namespace qnn;

extern "C" size_t qnn_int8_moe_workspace_bytes(int64_t tokens, int top, int64_t F) {
    if (tokens < 1 || tokens > QNN_MOE_MAX_TOKENS || top < 1 || top > QNN_MOE_MAX_TOP || F < 1 || F > int8::kMostK) return 0;
    return int8::route_bytes(tokens, top) + int8::act_bytes(tokens, top, F) + int8::tops_bytes(tokens, top, F) + int8::codes_bytes(tokens, top, F) +
           int8::scales_bytes(tokens, top);
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
    const size_t r = int8::route_bytes(tokens, top), v = r + int8::act_bytes(tokens, top, F), c = v + int8::tops_bytes(tokens, top, F),
                 f = c + int8::codes_bytes(tokens, top, F);
    const int8::MoeArgs a = {x, W1, W2, scale_x, logits, scale1, scale2, ldx, ld_logits, ld_w1, ld_w2, H, F, ldo, (int)tokens, experts, top,
                             reinterpret_cast<int8::Route *>(ws), reinterpret_cast<float *>(ws + r), reinterpret_cast<uint32_t *>(ws + v), ceil_div(F, 16),
                             reinterpret_cast<int8_t *>(ws + c), reinterpret_cast<float *>(ws + f), int8::codes_pitch(F)};
    hipStream_t s = static_cast<hipStream_t>(stream);
    return int8::launch_moe(a, out, type, s);
}
