// Attention over the paged cache for few rows: a workgroup has 16 NB rows (queries of one sequence and the heads that share one of the cache), and its four waves
// take 32 keys at a time in turn; the grid splits long sequences further.  A wave's products are S^T = K Q^T and O^T = V^T P^T (16 x 16 x 32, float16): of the
// first result a lane has keys 4 g + 0 .. 3 of either 16 for query lane mod 16, which is the second's right operand as it is once the rows of V are taken in that
// order; the sums over keys of a query are per lane until the end.  Codes go from memory to registers, 16 bytes of K a lane and D / 16 of V (whole rows a load), and
// become float16 there; V's transposition is the choice of bytes in that step.
// Single tokens are bound by memory (64 sequences of up to 8192 tokens, 32 heads on 8 of 128, bf16: 618 MB in 126 us, and 5 for the join of four parts), of one sequence
// by latency: page numbers, scales, codes, one after the other, before the first product (10000 tokens, 21 MB: 11 us and 4).  Drafted trees and short prompts take some 750
// vector instructions, which make codes float16 and scores weights, a step of 32 rows, and 48 matrix instructions; what bounds them is the longest sequences' workgroups, for all
// sequences have the same number of parts (8 sequences of up to 4099 tokens, 40 drafted each, 16 heads on 4 of 128, fp16, capped: 44 us and 4.5 for the join, vector units
// 39 % busy).
#include "qnn_attention.h"

namespace qnn {
namespace attention {
namespace {

constexpr int kStep = 32, kWaves = 4;

// Keys of a step, as a wave needs them: by the lane in memory order, in LDS
struct __attribute__((aligned(16))) Keys {
    uint32_t row[kStep];
    float k_scale[kStep], v_scale[kStep];
    float bias[kStep];   // 0, or -infinity for a key that is not there
    float log_v[kStep];  // log2 of the values' scale, rounded up
    int32_t place[kStep];
};

template <int DP>
struct Codes {
    static constexpr int kV = DP / 64;  // words of V a lane and key: DP / 16 codes
    v4u k[2][DP / 64];
    uint32_t v[8][kV];
};

// A query's lanes: DP / 64 runs of 16 values, 64 c + 16 g + 0 .. 15 with g = lane / 16, as operands for the products with 16 bytes of code each
template <typename T, int DP>
struct Query {
    static constexpr int kParts = Parts<T>::kQuery;
    h8 part[kParts][DP / 64][2];
    float mult;
    T x[DP / 64][16];
    __device__ __forceinline__ void ask(const Args &a, const Row &row) {
        const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int c = 0; c < DP / 64; ++c) {
            const int d = 64 * c + 16 * g;
            __builtin_memcpy(x[c], static_cast<const T *>(a.q) + row.token * a.ld_q + row.head * a.step_q + (d < a.D ? d : 0), sizeof x[c]);
        }
    }
    __device__ __forceinline__ void make(const Args &a) {
        const int g = (threadIdx.x & 63) >> 4;
        uint32_t top = 0u;
#pragma unroll
        for (int c = 0; c < DP / 64; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[c][i] = 64 * c + 16 * g < a.D ? x[c][i] : (T)0.0f;
#pragma unroll
        for (int c = 0; c < DP / 64; ++c) {
#pragma unroll
            for (int i = 0; i < 16; ++i) top = max(top, rows::magnitude((float)x[c][i]));
        }
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        const Scaling scaling(top);
        mult = scaling.mult(a.scale);
#pragma unroll
        for (int c = 0; c < DP / 64; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                _Float16 y[kParts];
                split(scaling.of((float)x[c][i]), y);
#pragma unroll
                for (int p = 0; p < kParts; ++p) part[p][c][i >> 3][i & 7] = y[p];
            }
    }
};

// Waves that a SIMD is to hold: what is in flight grows with them.  (Heads of 64, 32 rows: three 62 us for two's 64, 16 sequences of up to 3000 tokens with 40 drafted, bf16; 41 for
// 46, 4 sequences with 100 new tokens, fp16.  With a cap or a bias registers would be spilled.)
constexpr int waves_of(int DP, int NB, int parts, bool more) {
    return DP == 64 ? (NB == 1 ? 4 : (parts == 2 || more ? 2 : 3)) : (DP == 128 && NB == 1 ? 3 : (parts == 2 ? 1 : 2));
}

// kKind: 0 plain scores, 1 a bias by distance or a cap, 2 a cap that is close
template <typename T, int DP, int NB, int kKind>
__global__ __launch_bounds__(64 * kWaves, waves_of(DP, NB, Parts<T>::kQuery, kKind > 0)) void few_rows_kernel(const Args a) {
    constexpr bool kMore = kKind > 0, kClose = kKind == 2;
    constexpr int kRows = 16 * NB, kPitch = DP + 4, kV = DP / 64, kQuery = Parts<T>::kQuery, kWeight = Parts<T>::kWeight;
    __shared__ Keys keys[kWaves][2];
    __shared__ float2 states[kWaves][kRows];
    __shared__ __attribute__((aligned(16))) float sums[2][kRows][kPitch];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    uint32_t head, split, block, b;
    {
        const uint32_t id = rows::block_number();
        uint32_t rest = quotient(id, a.pages.heads, a.heads_inverse, head);
        rest = quotient(rest, (uint32_t)a.splits, a.splits_inverse, split);
        b = quotient(rest, (uint32_t)a.blocks, a.blocks_inverse, block);
    }
    if ((int64_t)b >= a.sequences) return;  // (of the launch's last line)
    const Sequence s = sequence_at(a, b);
    const uint32_t n_rows = (uint32_t)s.fresh * (uint32_t)a.group;
    if (a.short_rows > 0 && n_rows > (uint32_t)a.short_rows) return;
    for (uint32_t first = block * kRows; first < n_rows; first += (uint32_t)a.blocks * kRows) {
        uint32_t in_group;
        const uint32_t last = min(first + kRows, n_rows) - 1u;
        const int32_t i0 = (int32_t)quotient(first, (uint32_t)a.group, a.group_inverse, in_group), i1 = (int32_t)quotient(last, (uint32_t)a.group, a.group_inverse, in_group);
        // keys below `end` are looked at, those below `open` are seen by all rows
        const int32_t end = min(a.tree ? s.n : max(s.base + i1 + 1, 0), s.in_table), open = a.tree ? s.base : s.base + i0 + 1;
        const int64_t steps = (end + (int64_t)kStep - 1) / kStep;
        const int32_t lo = (int32_t)(steps * split / a.splits), hi = (int32_t)(steps * (split + 1) / a.splits);

        const Cap cap = kClose || (kMore && !kAlwaysClose<T> && a.cap > 0.0f) ? cap_of<kClose>(a) : Cap{};
        Query<T, DP> query[NB];
        Sight sight[NB];
        v4f out[DP / 16][NB] = {};
        float level[NB], total[NB];  // R; the sum of 2^(t - R) over this lane's keys
#pragma unroll
        for (int n = 0; n < NB; ++n) level[n] = -INFINITY, total[n] = 0.0f;

        // ---- loads.  Of a step: the page numbers, then rows and scales, then codes
        const int at = lane & 31;
        struct Ahead {
            uint32_t row;
            float k_scale, v_scale;
            int32_t place;
        };
        auto find = [&](int32_t step) __attribute__((always_inline)) -> paged::Place {
            const int32_t key = step * kStep + at;
            return step < hi && key < end ? paged::place_of(a.pages, b, (uint32_t)key) : paged::Place{paged::kNoRow, 0u};
        };
        auto scales = [&](int32_t step, const paged::Place &place, Ahead &x) __attribute__((always_inline)) {
            const uint32_t row = paged::row_of(a.pages, place, head);
            x.row = row;
            x.k_scale = row != paged::kNoRow ? a.k_scale[row] : 0.0f, x.v_scale = row != paged::kNoRow ? a.v_scale[row] : 0.0f;
            x.place = step * kStep + at;
            if (kMore && a.tree && x.place >= s.base && row != paged::kNoRow && x.place - s.base < s.fresh)
                x.place = s.base - 1 + __popcll(a.tree[s.first + (x.place - s.base)]);
        };
        auto note = [&](const Ahead &x, Keys &k) __attribute__((always_inline)) -> bool {  // whether all are there
            const bool there = x.row != paged::kNoRow;
            if (lane < kStep) {
                k.row[at] = there ? x.row : 0u;
                k.k_scale[at] = x.k_scale, k.v_scale[at] = x.v_scale;
                k.bias[at] = there ? 0.0f : -INFINITY;
                k.log_v[at] = log_scale(x.v_scale);
                if constexpr (kMore) k.place[at] = x.place;
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            return __all(there);
        };
        Codes<DP> c;
        auto fetch_k = [&](const Keys &k) __attribute__((always_inline)) {
            const int lane = opaque(threadIdx.x & 63), r = lane & 15, g = lane >> 4;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int8_t *const from = a.k + (int64_t)k.row[16 * h + r] * a.D;
#pragma unroll
                for (int i = 0; i < DP / 64; ++i) {
                    const int d = 64 * i + 16 * g;
                    c.k[h][i] = *reinterpret_cast<const v4u *>(from + (d < a.D ? d : 0));  // (beyond the head the query is zero)
                }
            }
        };
        auto fetch_v = [&](const Keys &k) __attribute__((always_inline)) {
            const int lane = opaque(threadIdx.x & 63), r = lane & 15, g = lane >> 4;
            const int d = r * (DP / 16) < a.D ? r * (DP / 16) : 0;  // (beyond the head nothing is stored)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int8_t *const from = a.v + (int64_t)k.row[16 * (e >> 2) + 4 * g + (e & 3)] * a.D + d;
                __builtin_memcpy(c.v[e], __builtin_assume_aligned(from, 4 * kV), 4 * kV);
            }
        };
        v4f dots[2][NB];
        auto use_k = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int n = 0; n < NB; ++n) dots[h][n] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < DP / 64; ++i)
#pragma unroll
                for (int f = 0; f < 2; ++f)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const h8 codes = eight_codes(c.k[h][i][2 * f], c.k[h][i][2 * f + 1]);
#pragma unroll
                        for (int n = 0; n < NB; ++n)
#pragma unroll
                            for (int p = 0; p < kQuery; ++p)
                                dots[h][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes, query[n].part[p][i][f], dots[h][n], 0, 0, 0);
                    }
        };
        auto use_v = [&](int32_t step, const Keys &k, bool all_there) __attribute__((always_inline)) {
            const int g = opaque(threadIdx.x & 63) >> 4;
            v4f k_scale[2], v_scale[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int from = 16 * h + 4 * g;
                k_scale[h] = *reinterpret_cast<const v4f *>(&k.k_scale[from]), v_scale[h] = *reinterpret_cast<const v4f *>(&k.v_scale[from]);
            }
            const bool masked = (step + 1) * (int64_t)kStep > open || !all_there;
            h8 weights[NB][kWeight];
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                float t[2][4];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float x = dots[h][n][e] * (query[n].mult * k_scale[h][e]);
                        if constexpr (kMore) {
                            if (kClose || (!kAlwaysClose<T> && a.cap > 0.0f)) x = capped<kClose>(cap, x);
                            if (a.slopes) x = __fmaf_rn(sight[n].slope, (float)(k.place[16 * h + 4 * g + e] - sight[n].place), x);
                        }
                        t[h][e] = x;
                    }
                auto mask = [&](auto tree) __attribute__((always_inline)) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const v4f bias = *reinterpret_cast<const v4f *>(&k.bias[16 * h + 4 * g]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const bool sees = sight[n].template sees<decltype(tree)::value>(s, step * kStep + 16 * h + 4 * g + e) & (bias[e] == 0.0f);
                            t[h][e] = sees ? t[h][e] : -INFINITY;
                        }
                    }
                };
                if (masked) {
                    if (a.tree)
                        mask(std::true_type{});
                    else
                        mask(std::false_type{});
                }
                float sum, largest;
                auto weigh = [&]() __attribute__((always_inline)) {
                    const float from = level[n] == -INFINITY ? 0.0f : level[n];
                    sum = 0.0f, largest = 0.0f;
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float p = __builtin_amdgcn_exp2f(t[h][e] - from), w = t[h][e] == -INFINITY ? 0.0f : p * v_scale[h][e];
                            sum += p, largest = fmaxf(largest, fabsf(w));  // (and a scale that is NaN is only for those who see it)
                            _Float16 x[kWeight];
                            attention::split(w, x);
#pragma unroll
                            for (int i = 0; i < kWeight; ++i) weights[n][i][4 * h + e] = x[i];
                        }
                };
                weigh();
                largest = fmaxf(largest, sum * kOfSum);
                if (__any(level[n] == -INFINITY || largest > 32768.0f)) {
                    float most = -INFINITY;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const v4f log_v = *reinterpret_cast<const v4f *>(&k.log_v[16 * h + 4 * g]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) most = fmaxf(most, t[h][e] + log_v[e]);
                    }
                    most = fmaxf(most, __shfl_xor(most, 16));
                    most = fmaxf(most, __shfl_xor(most, 32));
                    largest = fmaxf(largest, __shfl_xor(largest, 16));
                    largest = fmaxf(largest, __shfl_xor(largest, 32));
                    // (whether a query's R moves depends on that query alone)
                    const bool moves = (level[n] == -INFINITY || largest > 32768.0f) && most > level[n];
                    const float now = moves ? most - 8.0f : level[n], root = level[n] == now ? 1.0f : root_of(level[n], now), factor = root * root;
                    level[n] = now;
                    total[n] = total[n] * root * root;
#pragma unroll
                    for (int d = 0; d < DP / 16; ++d) out[d][n] *= factor;
                    weigh();
                }
                total[n] += sum;
            }
            // V: byte d mod 4 of word d / 4 of the eight keys' rows
#pragma unroll
            for (int x = 0; x < kV; ++x)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    h2 codes[2][4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t pair = __builtin_amdgcn_perm(c.v[2 * e + 1][x] ^ kBias, c.v[2 * e][x] ^ kBias, half ? 0x07030602u : 0x05010400u);
                        codes[0][e] = halves(__builtin_amdgcn_perm(kExponents, pair, 0x04010400u));
                        codes[1][e] = halves(__builtin_amdgcn_perm(kExponents, pair, 0x04030402u));
                    }
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const h8 operand = {codes[y][0][0], codes[y][0][1], codes[y][1][0], codes[y][1][1], codes[y][2][0], codes[y][2][1], codes[y][3][0], codes[y][3][1]};
                        const int d = 4 * x + 2 * half + y;
#pragma unroll
                        for (int n = 0; n < NB; ++n)
#pragma unroll
                            for (int p = 0; p < kWeight; ++p) out[d][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand, weights[n][p], out[d][n], 0, 0, 0);
                    }
                }
        };

        // ---- steps lo + wave, lo + wave + 4, ...: of the next one, K's codes are asked for as soon as this one's are used, and V's likewise; scales two steps ahead,
        // page numbers three
        {
            Ahead ahead;
            const int32_t step0 = lo + wave;
            paged::Place row = find(step0);
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const Row of = row_at(a, s, min(first + 16u * n + r, last), head);
                query[n].ask(a, of);
                sight[n].load(a, s, of);
            }
            scales(step0, row, ahead);
            row = find(step0 + kWaves);
            bool all_there = true;
            if (step0 < hi) {
                all_there = note(ahead, keys[wave][0]);
                fetch_k(keys[wave][0]);
                fetch_v(keys[wave][0]);
            }
            scales(step0 + kWaves, row, ahead);
            row = find(step0 + 2 * kWaves);
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                query[n].make(a);
                query[n].mult *= kClose || (kMore && !kAlwaysClose<T> && a.cap > 0.0f) ? cap.before : kLog2e;
            }
            int turn = 0;
            for (int32_t step = step0; step < hi; step += kWaves) {
                use_k();
                const bool next_there = note(ahead, keys[wave][turn ^ 1]);
                if (step + kWaves < hi) fetch_k(keys[wave][turn ^ 1]);
                use_v(step, keys[wave][turn], all_there);
                all_there = next_there;
                turn ^= 1;
                if (step + kWaves < hi) fetch_v(keys[wave][turn]);
                scales(step + 2 * kWaves, row, ahead);
                row = find(step + 3 * kWaves);
            }
        }

        // ---- the waves' sums
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            total[n] += __shfl_xor(total[n], 16);
            total[n] += __shfl_xor(total[n], 32);
            if (g == 0) states[wave][16 * n + r] = make_float2(level[n], total[n]);
        }
        __syncthreads();
        auto most_of = [&](int row) __attribute__((always_inline)) {
            float most = states[0][row].x;
#pragma unroll
            for (int w = 1; w < kWaves; ++w) most = fmaxf(most, states[w][row].x);
            return most;
        };
        auto put = [&](bool add) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const float root = root_of(level[n], most_of(16 * n + r)), f = root * root;
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int d4 = 0; d4 < DP / 64; ++d4) {
                        v4f *const to = reinterpret_cast<v4f *>(&sums[wave & 1][16 * n + r][(4 * g + e) * (DP / 16) + 4 * d4]);
                        v4f x = {out[4 * d4][n][e] * f, out[4 * d4 + 1][n][e] * f, out[4 * d4 + 2][n][e] * f, out[4 * d4 + 3][n][e] * f};
                        if (add) x += *to;
                        *to = x;
                    }
            }
        };
        if (wave >= 2) put(false);
        __syncthreads();
        if (wave < 2) put(true);
        __syncthreads();
        for (uint32_t x = threadIdx.x; x < (uint32_t)(kRows * (DP / 8)); x += 64 * kWaves) {
            const uint32_t row = x / (DP / 8), d = x % (DP / 8) * 8;
            if (first + row > last || (int32_t)d >= a.D) continue;
            const Row at_row = row_at(a, s, first + row, head);
            const float most = most_of(row);
            float sum = 0.0f, y[8];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float root = root_of(states[w][row].x, most);
                sum += states[w][row].y * root * root;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = sums[0][row][d + e] + sums[1][row][d + e];
            if (a.splits == 1) {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = sum == 0.0f ? 0.0f : y[e] / sum;
                store_eight<T>(a.out, at_row.token * a.ld_out + at_row.head * a.step_out + d, y);
            } else {
                const int64_t to = ((int64_t)split * a.tokens + at_row.token) * a.heads_q + at_row.head;
                if (d == 0) a.state[to] = make_float2(most, sum);
                if (!(sum == 0.0f)) {
                    float *const p = a.part + to * a.D + d;
                    __builtin_memcpy(p, y, sizeof y);
                }
            }
        }
        __syncthreads();  // (before the next rows)
    }
}

// Parts of the keys joined.  32 lanes (64 where a head is longer than 128) take a query and head, 4 values a lane: up to 8 parts, all asked for at once.  Where there
// are more, 256 / kLanes groups of lanes share them, 16 parts each at most.  (2 parts of 32768 rows of 128: 10.7 us, and 49.7 with a workgroup for each row.)
template <typename T>
__device__ __forceinline__ void store_joined(const Args &a, int64_t token, int64_t head, int at, const v4f &y, float total) {
    if (4 * at >= a.D) return;
    struct Four {
        T e[4];
    } four;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float x = total == 0.0f ? 0.0f : y[e] / total;
        if constexpr (std::is_same<T, rows::f16>::value) asm("" : "+v"(x));  // (rounded from the value in fp32)
        four.e[e] = (T)x;
    }
    __builtin_memcpy(static_cast<T *>(a.out) + token * a.ld_out + head * a.step_out + 4 * at, &four, sizeof four);
}
template <typename T, int kLanes, int kParts>
__global__ __launch_bounds__(256) void join_few_kernel(const Args a) {
    const int at = threadIdx.x % kLanes;
    const int64_t all = a.tokens * a.heads_q, id = (int64_t)rows::block_number() * (256 / kLanes) + threadIdx.x / kLanes;
    if (id >= all) return;
    uint32_t head;
    const int64_t token = quotient((uint32_t)id, (uint32_t)a.heads_q, a.heads_q_inverse, head);
    const float *const from = a.part + id * a.D + (4 * at < a.D ? 4 * at : 0);
    float2 state[kParts];
    v4f part[kParts];
    // (parts beyond the last are the last again, and take no part; what was not written, because nothing was seen, neither)
#pragma unroll
    for (int s = 0; s < kParts; ++s) {
        const int64_t from_part = min(s, a.splits - 1) * all;
        state[s] = a.state[from_part + id], part[s] = *reinterpret_cast<const v4f *>(from + from_part * a.D);
    }
    if (token < a.starts[0] || token >= a.starts[a.sequences]) return;
    float top = -INFINITY, total = 0.0f;
    v4f y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < kParts; ++s) top = fmaxf(top, state[s].x);
#pragma unroll
    for (int s = 0; s < kParts; ++s) {
        const float root = s < a.splits ? root_of(state[s].x, top) : 0.0f, factor = root * root;
        const bool none = s >= a.splits || state[s].y == 0.0f;
        total = none ? total : __fmaf_rn(state[s].y * root, root, total);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = none ? y[e] : __fmaf_rn(factor, part[s][e], y[e]);
    }
    store_joined<T>(a, token, head, at, y, total);
}

template <typename T, int kLanes>
__global__ __launch_bounds__(256) void join_many_kernel(const Args a) {
    constexpr int kTeams = 256 / kLanes, kPer = kMostSplits / kTeams;
    __shared__ v4f sums[kTeams][kLanes];
    const int lane = threadIdx.x & 63, at = threadIdx.x % kLanes, team = threadIdx.x / kLanes;
    const int64_t all = a.tokens * a.heads_q, id = rows::block_number();
    if (id >= all) return;
    uint32_t head;
    const int64_t token = quotient((uint32_t)id, (uint32_t)a.heads_q, a.heads_q_inverse, head);
    // every wave reads all states, two a lane
    float2 state[2];
    v4f part[kPer];
    const float *const from = a.part + id * a.D + (4 * at < a.D ? 4 * at : 0);
#pragma unroll
    for (int i = 0; i < 2; ++i) state[i] = lane + 64 * i < a.splits ? a.state[(lane + 64 * i) * all + id] : make_float2(-INFINITY, 0.0f);
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (team + kTeams * i < a.splits) part[i] = *reinterpret_cast<const v4f *>(from + (team + kTeams * i) * all * a.D);
    if (token < a.starts[0] || token >= a.starts[a.sequences]) return;
    float top = fmaxf(state[0].x, state[1].x);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    float factor[2], total = 0.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float root = root_of(state[i].x, top);
        factor[i] = root * root;
        total = __fmaf_rn(state[i].y * root, root, total);
        if (state[i].y == 0.0f) factor[i] = -1.0f;  // (nothing there)
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) total += __shfl_xor(total, d);
    v4f y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int s = team + kTeams * i;
        const float f = s < 64 ? __shfl(factor[0], s & 63) : __shfl(factor[1], s & 63);
        if (s < a.splits && !(f < 0.0f)) y += f * part[i];
    }
    sums[team][at] = y;
    __syncthreads();
    if (team != 0) return;
#pragma unroll
    for (int t = 1; t < kTeams; ++t) y += sums[t][at];
    store_joined<T>(a, token, head, at, y, total);
}

template <typename T>
int launch_join(const Args &a, hipStream_t s) {
    auto launch = [&](auto kernel, int rows) { return QNN_LAUNCH("cache_attention", kernel, rows::grid_of(ceil_div(a.tokens * a.heads_q, rows)), dim3(256), 0, s, a); };
    auto few = [&](auto two, auto four, auto eight, int rows) { return launch(a.splits <= 2 ? two : (a.splits <= 4 ? four : eight), rows); };
    if (a.splits > 8) return a.D <= 128 ? launch(join_many_kernel<T, 32>, 1) : launch(join_many_kernel<T, 64>, 1);
    if (a.D <= 128) return few(join_few_kernel<T, 32, 2>, join_few_kernel<T, 32, 4>, join_few_kernel<T, 32, 8>, 8);
    return few(join_few_kernel<T, 64, 2>, join_few_kernel<T, 64, 4>, join_few_kernel<T, 64, 8>, 4);
}

// Few rows (up to 768 of a sequence and head of the cache): 16 or 32 a workgroup, and as many parts of the keys as fill the card, each the same number of steps for
// every wave.  (us, bf16, 32 heads on 8 of 128: 8 sequences of up to 4000 tokens in 11 parts each 22, in one 55; one of 10000 in 79 parts 17, in 16 parts 20.)  Where there is
// work for every unit without: parts of 8 turns of the waves at least, for their joining takes 5 us (64 sequences of up to 500 tokens in one part each 17, in two 22),
// and where a sequence has one workgroup's rows, 2.5 times what the card holds, so that long sequences and short ones come out even (64 of up to 8192 in one part 163, in
// two 146, in four 138; 128 of up to 4096 in one 156, in two 145).
// Many rows: 128 or 256 a workgroup, one on a compute unit, and parts only as far as all are resident (1500 of up to 6000 tokens, 16 heads on 4 of 64: 96 workgroups in
// 2 parts 140, in 3 171), but 2 where they are more than half as many, for sequences of different lengths (3 of up to 2500 with 700 new ones: 84, in one part 121).
// (us on the kernel for few and on the one for many, sequences of up to: 16 of 2000 with 256 rows each 67 and 74, 512 rows 109 and 106; 2 of 5000 with 640 rows 65 and 70, 800 rows 77 and 80; one of 8192 with 512 rows 59 and 65, 1024 rows 99 and 79; heads of 256: 4 of 4000
// with 400 rows 108 and 166, one of 4096 with 1024 rows 111 and 110, 2048 rows 191 and 178.)
Plan plan_of(int64_t sequences, int64_t heads_q, int64_t heads, int64_t D, int type, int64_t most_new, int64_t longest) {
    Plan p;
    const int64_t rows = most_new * (heads_q / heads);
    const bool few = rows <= 768 || !takes_many(D, type);
    p.rows = few ? (rows <= 16 || D > 128 ? 16 : 32) : many_rows(D);
    p.blocks = ceil_div(rows, p.rows);
    const int64_t on_unit = few ? waves_of(D <= 64 ? 64 : (D <= 128 ? 128 : 256), p.rows / 16, 1, false) : 1;
    const double blocks = (double)sequences * (double)heads * (double)p.blocks;
    const int64_t units = compute_units(), wanted = blocks < 1e12 ? (int64_t)blocks : (int64_t)1e12, per_turn = few ? kStep * kWaves : 256, turns = ceil_div(longest, per_turn);
    int64_t want = few || units / wanted < 2 ? ceil_div(on_unit * units, wanted) : units / wanted;
    if (few && wanted >= units) {
        if (p.blocks == 1) want = ceil_div(on_unit * units * 5 / 2, wanted);
        want = want < turns / 8 ? want : (turns >= 8 ? turns / 8 : 1);
    }
    p.splits = ceil_div(turns, ceil_div(turns, want < kMostSplits ? want : kMostSplits));
    return p;
}
bool plannable(int64_t tokens, int64_t sequences, int64_t heads_q, int64_t heads, int64_t D, int64_t most_new, int64_t longest) {
    return tokens >= 1 && tokens <= 0x7FFFFFFF && sequences >= 1 && sequences <= 0x3FFFFFFF && heads >= 1 && heads_q >= 1 && heads_q % heads == 0 &&
           heads_q <= 65535 && D >= 16 && D <= paged::kMostD && most_new >= 1 && longest >= 1;
}
// Rows (queries and heads) times parts that a call has at most: what its workspace is for.  More tokens or longer sequences never have less, so that a workspace made for the most
// serves all calls.  No plan for the tokens that sequences can have (sequences * most_new) comes to the second bound: two parts or more are made of fewer workgroups than 7.5 a unit
// with 32 rows each, or than one a unit with 256, and there is at most one part more than that many workgroups in all give.  Calls of more tokens, nobody's for the most part, are
// split into fewer.
int64_t most_rows(int64_t rows, int64_t longest) {
    const int64_t turns = ceil_div(longest, kStep * kWaves), parts = turns < kMostSplits ? turns : kMostSplits, most = 512 * (int64_t)compute_units();
    return parts == 1 ? 0 : (rows * parts < most ? rows * parts : most);
}
// (numbers above what there can be do no more than these)
int64_t at_most(int64_t x, int64_t limit) { return x < limit ? x : limit; }
// From so many sequences on, those with up to 16 rows, or one token, are left to the kernel for few where the call is the kernel's for many: tokens beside a prompt.  (us with and
// without, 32 heads on 8 of 128, bf16: 2048 of 8192 tokens and one of each of 63 sequences of up to 8192 507 and 1454, 1024 of 4096 and 31 of up to 4096 250 and 403, and 15 of them 247 and
// 279; with 7 sequences it goes either way: 512 of 2000 and 7 of up to 32768 594 and 916, a prompt of 1024 and 7 of up to 8000 174 and 231, but 1024 of 8000 and 7 of up to 8000 453
// and 327, 512 of 2000 and 7 of up to 4000 155 and 122; 8 sequences of 600 with 300 each 74 and 73.)
constexpr int64_t kMixed = 8;

template <typename T, int DP, int kKind>
int launch_few(const Args &a, int rows, dim3 grid, hipStream_t s) {
    if (DP > 128 || rows == 16) return QNN_LAUNCH("cache_attention", (few_rows_kernel<T, DP, 1, kKind>), grid, dim3(64 * kWaves), 0, s, a);
    if constexpr (DP <= 128) return QNN_LAUNCH("cache_attention", (few_rows_kernel<T, DP, 2, kKind>), grid, dim3(64 * kWaves), 0, s, a);
}
template <typename T, int DP>
int launch_few(const Args &a, int rows, dim3 grid, hipStream_t s) {
    if (a.cap > (kAlwaysClose<T> ? 0.0f : kCloseFrom)) return launch_few<T, DP, 2>(a, rows, grid, s);
    return a.cap > 0.0f || a.slopes ? launch_few<T, DP, 1>(a, rows, grid, s) : launch_few<T, DP, 0>(a, rows, grid, s);
}
template <typename T>
int launch_few(const Args &a, int rows, dim3 grid, hipStream_t s) {
    if (a.D <= 64) return launch_few<T, 64>(a, rows, grid, s);
    return a.D <= 128 ? launch_few<T, 128>(a, rows, grid, s) : launch_few<T, 256>(a, rows, grid, s);
}

}  // namespace
}  // namespace attention
}  // namespace qnn

using namespace qnn;

extern "C" size_t qnn_cache_attention_workspace_bytes(int64_t tokens, int64_t sequences, int64_t heads_q, int64_t heads, int64_t D, int64_t most_new,
                                                      int64_t longest) {
    if (!attention::plannable(tokens, sequences, heads_q, heads, D, most_new, longest)) return 0;
    return (size_t)attention::most_rows(tokens * heads_q, attention::at_most(longest, 0x7FFFFFFF)) * ((size_t)D * 4 + 8);
}

extern "C" int qnn_cache_attention(const qnn_paged_cache *cache, const void *q, int64_t ld_q, int64_t step_q, int64_t heads_q, int type, float scale, float cap,
                                   const float *slopes, const uint64_t *tree, int64_t tokens, int64_t most_new, int64_t longest, void *out, int64_t ld_out,
                                   int64_t step_out, void *workspace, size_t workspace_bytes, void *stream) {
    const char *const what = "cache_attention";
    if (int rc = paged::check_cache(what, cache)) return rc;
    const int64_t D = cache->D;
    if (tokens < 0 || tokens > 0x7FFFFFFF || heads_q < 1 || heads_q > 65535 || heads_q % cache->heads || most_new < 1 || longest < 1)
        return fail(QNN_ERR_SHAPE, "%s: %lld tokens, %lld heads on %lld of the cache, most_new = %lld, longest = %lld", what, (long long)tokens, (long long)heads_q,
                    (long long)cache->heads, (long long)most_new, (long long)longest);
    if (!rows::known_type(type)) return fail(QNN_ERR_SHAPE, "%s: type %d", what, type);
    if (!(cap == 0.0f || (cap >= 1e-30f && cap <= 3.0e38f)) || !(scale >= -3.0e38f && scale <= 3.0e38f)) return fail(QNN_ERR_SHAPE, "%s: scale = %g, cap = %g", what, (double)scale, (double)cap);
    if (tokens == 0 || cache->sequences == 0) return QNN_OK;
    if ((double)tokens * (double)(heads_q / cache->heads) > 2147483647.0) return fail(QNN_ERR_UNSUPPORTED, "%s: %lld tokens", what, (long long)tokens);
    if (!paged::heads_fit(ld_q, step_q, heads_q, D, tokens) || !paged::heads_fit(ld_out, step_out, heads_q, D, tokens))
        return fail(QNN_ERR_SHAPE, "%s: heads of %lld values at strides %lld, %lld or %lld, %lld overlap", what, (long long)D, (long long)ld_q, (long long)step_q,
                    (long long)ld_out, (long long)step_out);
    if (!q || !out) return fail(QNN_ERR_NULL, "%s: NULL pointer", what);
    if (int rc = paged::check_cache_pointers(what, cache)) return rc;
    const int w = rows::value_bytes(type);
    if (!rows::aligned_to(q, w) || !rows::aligned_to(out, w) || !rows::aligned_to(slopes, 4) || !rows::aligned_to(tree, 8))
        return fail(QNN_ERR_ALIGN, "%s: pointer not aligned to its type", what);
    most_new = attention::at_most(most_new, tokens), longest = attention::at_most(longest, 0x7FFFFFFF);
    attention::Plan p = attention::plan_of(cache->sequences, heads_q, cache->heads, D, type, most_new, longest);
    const int64_t parts = attention::most_rows(tokens * heads_q, longest) / (tokens * heads_q);
    p.splits = p.splits <= parts ? p.splits : (parts > 1 ? parts : 1);
    const size_t need = p.splits == 1 ? 0 : qnn_cache_attention_workspace_bytes(tokens, cache->sequences, heads_q, cache->heads, D, most_new, longest);
    if (need > 0 && (!workspace || !rows::aligned_to(workspace, 256) || workspace_bytes < need))
        return fail(QNN_ERR_WORKSPACE, "%s: workspace NULL, misaligned or smaller than %zu bytes", what, need);
    const double blocks = (double)cache->sequences * (double)cache->heads * (double)p.blocks * (double)p.splits;
    if (blocks > 1073741823.0 || (double)tokens * (double)heads_q > 2147483647.0) return fail(QNN_ERR_UNSUPPORTED, "%s: %.0f workgroups", what, blocks);
    const int64_t queries = tokens * heads_q;
    float *const part = static_cast<float *>(workspace);
    attention::Args a = {};
    a.q = q, a.out = out, a.ld_q = ld_q, a.step_q = step_q, a.ld_out = ld_out, a.step_out = step_out;
    a.k = cache->k, a.v = cache->v, a.k_scale = cache->k_scale, a.v_scale = cache->v_scale;
    a.pages = paged::pages_of(*cache), a.starts = cache->starts, a.lengths = cache->lengths, a.slopes = slopes, a.tree = tree, a.scale = scale, a.cap = cap;
    a.tokens = tokens, a.sequences = cache->sequences, a.D = (int32_t)D, a.heads_q = (int32_t)heads_q;
    a.group = (int32_t)(heads_q / cache->heads), a.splits = (int32_t)p.splits, a.blocks = (int32_t)p.blocks;
    a.group_inverse = inverse_of(a.group), a.heads_inverse = inverse_of(cache->heads), a.heads_q_inverse = inverse_of(heads_q), a.splits_inverse = inverse_of(p.splits), a.blocks_inverse = inverse_of(p.blocks);
    a.part = part, a.state = reinterpret_cast<float2 *>(part + p.splits * queries * D);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 grid = rows::grid_of((int64_t)blocks);
    const auto few = [&](const attention::Args &a, int rows, dim3 grid) {
        return rows::with_type(type, [&](auto tag) { return attention::launch_few<decltype(tag)>(a, rows, grid, s); });
    };
    int rc;
    if (p.rows > 32) {
        a.short_rows = cache->sequences >= attention::kMixed && a.group <= 64 ? (a.group > 16 ? a.group : 16) : 0;
        rc = attention::launch_many(a, type, grid, s);
        if (rc == QNN_OK && a.short_rows > 0) {
            const int rows = a.short_rows <= 16 || D > 128 ? 16 : 32;
            a.blocks = (int32_t)ceil_div(a.short_rows, rows), a.blocks_inverse = inverse_of(a.blocks);  // (at most 4, and those of many rows more)
            rc = few(a, rows, rows::grid_of(cache->sequences * cache->heads * p.splits * a.blocks));
        }
    } else {
        rc = few(a, p.rows, grid);
    }
    if (rc || p.splits == 1) return rc;
    return rows::with_type(type, [&](auto tag) { return attention::launch_join<decltype(tag)>(a, s); });
}
