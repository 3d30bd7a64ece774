// Attention over the paged cache for many rows (drafted trees, prompts): a workgroup has 32 rows a wave, and all its waves meet the same 64 keys at a time, whose codes
// the workgroup brings from memory to registers two tiles ahead, makes float16 once for all waves and lays into LDS as the matrix instructions (32 x 32 x 16) take them.
// S^T = K Q^T and O^T = V^T P^T: of the first result a lane has keys 8 a + 4 g + 0 .. 3 (a = 0 .. 3, g = lane / 32) of its query lane mod 32, which is the second's
// right operand as it is, with the rows of V^T's operand in that order of keys.
// Bound by what a wave's matrix instructions and vector ones take together and by the card's power: the last 2048 of 8192 tokens, 32 heads on 8 of 128, bf16, take 342 to
// 390 us (0.62 to 0.70 Pop/s; 155 at the rate of a large matrix product), matrix cores 27 % of the time busy, vector ones 61 %; on codes that are all zero, with the same
// instructions, 312.  A quarter more vector instructions (a bias by distance whose slopes are zero) cost 1 to 3 %.
#include "qnn_attention.h"

namespace qnn {
namespace attention {
namespace {

typedef float v16f __attribute__((ext_vector_type(16)));

constexpr int kTile = 64;  // keys

// K: [key][DP] in pieces of 8 float16, piece p of key r at p xor (r mod 8; mod 16 where a row has as many pieces: 1 % less time).  V: rows of 64 keys, value d at row (d mod 4) (DP / 4) + d / 4: a block of 32 rows is what
// one quarter of the lanes' words holds; piece 2 s + g has keys 16 s + 4 g + 0 .. 3 and 16 s + 8 + 4 g + 0 .. 3, and lies at (2 s + g) xor (row mod 8).
template <int DP>
struct Tile {
    uint8_t k[kTile * DP * 2];
    uint8_t v[kTile * DP * 2];
};
struct __attribute__((aligned(16))) Scales {
    float k[kTile], v[kTile], log_v[kTile], bias[kTile];  // log_v: log2 of v, rounded up; bias: 0, or -infinity for a key that is not there
    float place[kTile];  // from the tile's first key's on
    int32_t all_there;
};

// kKind: 0 plain scores, 1 a bias by distance, 2 capped, with a bias or not, 3 by a cap that is close
template <typename T, int DP, int kWaves, int kKind>
__global__ __launch_bounds__(64 * kWaves, kWaves / 4) void many_rows_kernel(const Args a) {
    constexpr int kThreads = 64 * kWaves, kRows = 32 * kWaves, kQuery = Parts<T>::kQuery, kWeight = Parts<T>::kWeight;
    constexpr int kUnitsK = kTile * DP / 16, kUnitsV = kTile / 4 * (DP / 4), kLoadsK = (kUnitsK + kThreads - 1) / kThreads, kLoadsV = (kUnitsV + kThreads - 1) / kThreads;
    constexpr int kTurnK = DP >= 128 ? 15 : 7;  // pieces of a row of K change places by its number
    __shared__ __attribute__((aligned(16))) Tile<DP> tiles[2];
    __shared__ __attribute__((aligned(16))) Scales scales[2];
    __shared__ uint32_t rows_of[2][kTile];
    __shared__ __attribute__((aligned(16))) float ones[kTile];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 31, g = lane >> 5;
    uint32_t head, split, block, b;
    {
        const uint32_t id = rows::block_number();
        uint32_t rest = quotient(id, a.pages.heads, a.heads_inverse, head);
        rest = quotient(rest, (uint32_t)a.splits, a.splits_inverse, split);
        b = quotient(rest, (uint32_t)a.blocks, a.blocks_inverse, block);
        block = (uint32_t)a.blocks - 1u - block;  // (the last rows see the most keys: long work first.  4096 tokens' prompt, 32 heads of 128: 293 us -> 238)
    }
    if ((int64_t)b >= a.sequences) return;  // (of the launch's last line)
    if (tid < kTile) ones[tid] = 1.0f;
    const Sequence s = sequence_at(a, b);
    const uint32_t n_rows = (uint32_t)s.fresh * (uint32_t)a.group;
    if (n_rows <= (uint32_t)a.short_rows) return;
    for (uint32_t first = block * kRows; first < n_rows; first += (uint32_t)a.blocks * kRows) {
        uint32_t in_group;
        const uint32_t last = min(first + kRows, n_rows) - 1u;
        const int32_t i0 = (int32_t)quotient(first, (uint32_t)a.group, a.group_inverse, in_group), i1 = (int32_t)quotient(last, (uint32_t)a.group, a.group_inverse, in_group);
        // keys below `end` are looked at, those below `open` are seen by all rows
        const int32_t end = min(a.tree ? s.n : max(s.base + i1 + 1, 0), s.in_table), open = a.tree ? s.base : s.base + i0 + 1;
        const int64_t steps = (end + (int64_t)kTile - 1) / kTile;
        const int32_t lo = (int32_t)(steps * split / a.splits), hi = (int32_t)(steps * (split + 1) / a.splits);
        const bool busy = first + 32u * wave <= last;  // (other waves bring codes only)
        const Row row = row_at(a, s, min(first + 32u * wave + r, last), head);

        // ---- the query: DP / 16 steps of 16 values, 8 g + 0 .. 7 of each in this lane
        h8 query[kQuery][DP / 16];
        float mult;
        const Cap cap = kKind >= 2 ? cap_of<kKind == 3>(a) : Cap{};
        Sight sight;
        {
            T x[DP / 16][8];
            uint32_t top = 0u;
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) {
                __builtin_memcpy(x[c], static_cast<const T *>(a.q) + row.token * a.ld_q + row.head * a.step_q + (16 * c < a.D ? 16 * c + 8 * g : 0), sizeof x[c]);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[c][i] = 16 * c < a.D ? x[c][i] : (T)0.0f;
            }
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) {
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, rows::magnitude((float)x[c][i]));
            }
            top = max(top, (uint32_t)__shfl_xor((int)top, 32));
            const Scaling scaling(top);
            mult = scaling.mult(a.scale) * (kKind >= 2 ? cap.before : kLog2e);
#pragma unroll
            for (int c = 0; c < DP / 16; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    _Float16 y[kQuery];
                    attention::split(scaling.of((float)x[c][i]), y);
#pragma unroll
                    for (int p = 0; p < kQuery; ++p) query[p][c][i] = y[p];
                }
            sight.load(a, s, row);
        }
        v16f out[DP / 32] = {};
        float level = -INFINITY, total = 0.0f;

        // ---- codes: page numbers four tiles ahead, rows and scales three, codes two, float16 one.  Tiles are taken from the last on (tile_at): the keys next to a
        // query weigh most, all the more with a bias by distance, and R, which follows the largest, moves once.  (From the first on half as
        // long again, 607 us and 416 when that was tried: 2048 of 8192 tokens, 32 heads of 128, half of whose slopes are above 2^-4.)
        auto tile_at = [&](int32_t t) __attribute__((always_inline)) { return lo + hi - 1 - t; };
        auto find = [&](int32_t t) __attribute__((always_inline)) -> paged::Place {  // (threads below kTile)
            const int32_t key = tile_at(t) * kTile + tid;
            return t < hi && key < end ? paged::place_of(a.pages, b, (uint32_t)key) : paged::Place{paged::kNoRow, 0u};
        };
        struct Ahead {
            uint32_t row;
            float k, v;
            int32_t place;
        };
        auto ask = [&](int32_t t, const paged::Place &place, Ahead &x) __attribute__((always_inline)) {
            const uint32_t at = paged::row_of(a.pages, place, head);
            rows_of[(t - lo) & 1][tid] = at == paged::kNoRow ? 0u : at;
            x.row = at;
            x.k = at != paged::kNoRow ? a.k_scale[at] : 0.0f, x.v = at != paged::kNoRow ? a.v_scale[at] : 0.0f;
            x.place = tile_at(t) * kTile + tid;
            if (kKind > 0 && a.tree && x.place >= s.base && at != paged::kNoRow && x.place - s.base < s.fresh)
                x.place = s.base - 1 + __popcll(a.tree[s.first + (x.place - s.base)]);
        };
        auto note = [&](int32_t t, const Ahead &x) __attribute__((always_inline)) {
            Scales &to = scales[(t - lo) & 1];
            const bool there = x.row != paged::kNoRow;
            // (a scale of values that is not finite becomes a score that is NaN, for those who see it)
            const bool fine = rows::magnitude(x.v) < 0x7F800000u;
            to.k[tid] = fine ? x.k : __uint_as_float(0x7FC00000u), to.v[tid] = fine ? x.v : 0.0f, to.bias[tid] = there ? 0.0f : -INFINITY;
            to.log_v[tid] = log_scale(x.v);
            if constexpr (kKind > 0) to.place[tid] = (float)(x.place - tile_at(t) * kTile);
            const bool all = __all(there);
            if (tid == 0) to.all_there = all;
        };
        v4u raw_k[kLoadsK];
        uint32_t raw_v[kLoadsV][4];
        auto fetch = [&](int32_t t) __attribute__((always_inline)) {
            const int tid = opaque(threadIdx.x);
            const uint32_t *const at = rows_of[(t - lo) & 1];
#pragma unroll
            for (int i = 0; i < kLoadsK; ++i) {
                const int u = tid + kThreads * i, key = u / (DP / 16), d = u % (DP / 16) * 16;
                if (kUnitsK % kThreads == 0 || u < kUnitsK) raw_k[i] = *reinterpret_cast<const v4u *>(a.k + (int64_t)at[key] * a.D + (d < a.D ? d : 0));
            }
#pragma unroll
            for (int i = 0; i < kLoadsV; ++i) {
                const int u = tid + kThreads * i, four = u / (DP / 4), d = u % (DP / 4) * 4;
                if (kUnitsV % kThreads == 0 || u < kUnitsV) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) raw_v[i][e] = *reinterpret_cast<const uint32_t *>(a.v + (int64_t)at[4 * four + e] * a.D + (d < a.D ? d : 0));
                }
            }
        };
        auto put = [&](int32_t t) __attribute__((always_inline)) {
            const int tid = opaque(threadIdx.x);
            Tile<DP> &to = tiles[(t - lo) & 1];
#pragma unroll
            for (int i = 0; i < kLoadsK; ++i) {
                const int u = tid + kThreads * i, key = u / (DP / 16), piece = u % (DP / 16) * 2;
                if (kUnitsK % kThreads == 0 || u < kUnitsK) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        *reinterpret_cast<h8 *>(to.k + key * DP * 2 + 16 * ((piece + h) ^ (key & kTurnK))) = eight_codes(raw_k[i][2 * h], raw_k[i][2 * h + 1]);
                }
            }
#pragma unroll
            for (int i = 0; i < kLoadsV; ++i) {
                const int u = tid + kThreads * i, four = u / (DP / 4), at = u % (DP / 4);
                if (kUnitsV % kThreads == 0 || u < kUnitsV) {
                    h2 codes[4][2];
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const uint32_t pair = __builtin_amdgcn_perm(raw_v[i][2 * e + 1] ^ kBias, raw_v[i][2 * e] ^ kBias, half ? 0x07030602u : 0x05010400u);
                            codes[2 * half][e] = halves(__builtin_amdgcn_perm(kExponents, pair, 0x04010400u));
                            codes[2 * half + 1][e] = halves(__builtin_amdgcn_perm(kExponents, pair, 0x04030402u));
                        }
                    // keys 4 four .. + 3 = 16 s + 8 h + 4 g + ..
                    const int piece = (four >> 2) * 2 + (four & 1), h = four >> 1 & 1;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int at_row = j * (DP / 4) + at;
                        *reinterpret_cast<h4 *>(to.v + at_row * kTile * 2 + 16 * (piece ^ (at_row & 7)) + 8 * h) = h4{codes[j][0][0], codes[j][0][1], codes[j][1][0], codes[j][1][1]};
                    }
                }
            }
        };

        // ---- a tile's products.  Operands are read from LDS a group ahead; of a tile's two halves (32 keys each) the second's product with K runs beside the first's
        // weights, the first's product with V beside the second's: a wave's matrix instructions and its vector ones take turns, since the two waves of a SIMD, which
        // meet at a barrier every tile, would do the same at the same time.
        constexpr int kOperands = DP / 16, kOfK = kOperands * kQuery, kOfV = kOperands * kWeight;  // of K, of V, for 32 keys; products
        constexpr int kAhead = kQuery == 2 || DP > 128 ? 2 : 4;                                    // as many as registers allow
        auto use = [&](int32_t number) __attribute__((always_inline)) {
            const int32_t tile = tile_at(number);
            const int lane = opaque(threadIdx.x & 63), r = lane & 31, g = lane >> 5;
            const Tile<DP> &t = tiles[(number - lo) & 1];
            const Scales &sc = scales[(number - lo) & 1];
            const bool masked = (tile + 1) * (int64_t)kTile > open || !sc.all_there;  // some rows do not see some keys
            // products are scaled on the way to the exponent, unless they had to be before
            const bool scaled = kKind > 0 || masked;
            const float *const rest_k = scaled ? ones : sc.k;
            const float rest = scaled ? 1.0f : mult;
            // operands: K's number c of half h at place (h kOperands + c) mod kAhead, V's likewise
            h8 of_k[kAhead], of_v[kAhead];
            auto read_k = [&](int n) __attribute__((always_inline)) {
                const int h = n / kOperands, c = n % kOperands;
                if (n < 2 * kOperands) of_k[n % kAhead] = *reinterpret_cast<const h8 *>(t.k + (32 * h + r) * DP * 2 + 16 * ((2 * c + g) ^ (r & kTurnK)));
            };
            auto read_v = [&](int n) __attribute__((always_inline)) {  // step c of 16 keys, rows 32 d on
                const int h = n / kOperands, c = n % kOperands / (DP / 32), d = n % (DP / 32);
                if (n < 2 * kOperands) of_v[n % kAhead] = *reinterpret_cast<const h8 *>(t.v + (32 * d + r) * kTile * 2 + 16 * ((2 * (2 * h + c) + g) ^ (r & 7)));
            };
            v16f dots[2];  // key 32 h + 8 e + 4 g + i is value 4 e + i of half h
            h8 weights[2][kWeight][2];
            float sum, largest;
            auto four = [&](const float *from, int h, int e) __attribute__((always_inline)) { return *reinterpret_cast<const v4f *>(from + 32 * h + 8 * e + 4 * g); };
            // the j-th eighth of the products of half h
            auto with_k = [&](int h, int j) __attribute__((always_inline)) {
#pragma unroll
                for (int m = kOfK * j / 8; m < kOfK * (j + 1) / 8; ++m) {
                    const int n = h * kOperands + m / kQuery, p = m % kQuery;
                    if (m == 0) dots[h] = v16f{};
                    dots[h] = __builtin_amdgcn_mfma_f32_32x32x16_f16(of_k[n % kAhead], query[p][n % kOperands], dots[h], 0, 0, 0);
                    if (p == kQuery - 1) read_k(n + kAhead);
                }
            };
            auto with_v = [&](int h, int j) __attribute__((always_inline)) {
#pragma unroll
                for (int m = kOfV * j / 8; m < kOfV * (j + 1) / 8; ++m) {
                    const int n = h * kOperands + m / kWeight, q = m % kWeight, d = n % (DP / 32);
                    out[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(of_v[n % kAhead], weights[h][q][n % kOperands / (DP / 32)], out[d], 0, 0, 0);
                    if (q == kWeight - 1) read_v(n + kAhead);
                }
            };
            auto scale = [&](int h) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const v4f k = four(sc.k, h, e);
#pragma unroll
                    for (int i = 0; i < 4; ++i) dots[h][4 * e + i] *= mult * k[i];
                }
            };
            // scores times log2(e), -infinity where a row does not see a key
            auto score = [&](int h) __attribute__((always_inline)) {
                if constexpr (kKind > 0) scale(h);
                if constexpr (kKind >= 2) {
#pragma unroll
                    for (int x = 0; x < 16; ++x) dots[h][x] = capped<kKind == 3>(cap, dots[h][x]);
                }
                if (kKind == 1 || (kKind >= 2 && a.slopes)) {
                    const float place = (float)(sight.place - tile * kTile);  // (from the tile's beginning: whole numbers, exact)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const v4f of = four(sc.place, h, e);
#pragma unroll
                        for (int i = 0; i < 4; ++i) dots[h][4 * e + i] = __fmaf_rn(sight.slope, of[i] - place, dots[h][4 * e + i]);
                    }
                }
                if (masked) {
                    asm volatile("" ::: "memory");  // (keeps the branch a branch, here and below)
                    if constexpr (kKind == 0) scale(h);
                    auto mask = [&](auto tree) __attribute__((always_inline)) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const v4f bias = four(sc.bias, h, e);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const bool sees = sight.template sees<decltype(tree)::value>(s, tile * kTile + 32 * h + 8 * e + 4 * g + i) & (bias[i] == 0.0f);
                                dots[h][4 * e + i] = sees ? dots[h][4 * e + i] : -INFINITY;
                            }
                        }
                    };
                    if (a.tree) {
                        asm volatile("" ::: "memory");
                        mask(std::true_type{});
                    } else {
                        asm volatile("" ::: "memory");
                        mask(std::false_type{});
                    }
                }
            };
            // weights from R on, their sum without the values' scales, and the largest: the j-th eighth, two of a lane
            float from;
            auto begin = [&]() __attribute__((always_inline)) { from = level == -INFINITY ? 0.0f : level, sum = 0.0f, largest = 0.0f; };
            auto weigh = [&](int h, int j) __attribute__((always_inline)) {
                const int e = j / 2;
                const v4f v = four(sc.v, h, e);
                v4f k;
                if constexpr (kKind == 0) k = four(rest_k, h, e);
#pragma unroll
                for (int i = 2 * (j & 1); i < 2 * (j & 1) + 2; ++i) {
                    const float x = dots[h][4 * e + i], p = __builtin_amdgcn_exp2f(kKind == 0 ? __fmaf_rn(x, rest * k[i], -from) : x - from);
                    const float w = p * v[i];
                    sum += p, largest = fmaxf(largest, fabsf(w));
                    _Float16 y[kWeight];
                    attention::split(w, y);
#pragma unroll
                    for (int q = 0; q < kWeight; ++q) weights[h][q][e >> 1][4 * (e & 1) + i] = y[q];
                }
            };
            // moves R where a weight would be too large, which is seldom, and takes the half's sum in
            auto settle = [&](int h) __attribute__((always_inline)) {
                largest = fmaxf(largest, sum * kOfSum);
                if (__any(level == -INFINITY || largest > 32768.0f)) {
                    asm volatile("" ::: "memory");
                    float most = -INFINITY;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const v4f v = four(sc.log_v, h, e), k = four(rest_k, h, e);
#pragma unroll
                        for (int i = 0; i < 4; ++i) most = fmaxf(most, dots[h][4 * e + i] * (rest * k[i]) + v[i]);
                    }
                    most = fmaxf(most, __shfl_xor(most, 32)), largest = fmaxf(largest, __shfl_xor(largest, 32));
                    // (whether a query's R moves, and what it gets, depends on that query alone)
                    const bool moves = (level == -INFINITY || largest > 32768.0f) && most > level;
                    const float now = moves ? most - 8.0f : level, root = level == now ? 1.0f : root_of(level, now), factor = root * root;
                    level = now;
                    total = total * root * root;
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) out[d] *= factor;
                    begin();
#pragma unroll
                    for (int j = 0; j < 8; ++j) weigh(h, j);
                }
                total += sum;
            };
#pragma unroll
            for (int n = 0; n < kAhead; ++n) read_k(n);
#pragma unroll
            for (int j = 0; j < 8; ++j) with_k(0, j);
#pragma unroll
            for (int n = 0; n < kAhead; ++n) read_v(n);
            score(0);
            __builtin_amdgcn_sched_barrier(0);
            begin();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                with_k(1, j);
                weigh(0, j);
            }
            settle(0);
            score(1);
            __builtin_amdgcn_sched_barrier(0);
            begin();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                with_v(0, j);
                weigh(1, j);
            }
            settle(1);
#pragma unroll
            for (int j = 0; j < 8; ++j) with_v(1, j);
        };

        __syncthreads();  // (the rows before are done with LDS)
        if (lo < hi) {
            Ahead even, odd;  // scales of tiles lo, lo + 2, .. and lo + 1, lo + 3, ..
            paged::Place at = {paged::kNoRow, 0u};
            if (tid < kTile) {
                ask(lo, find(lo), even);
                ask(lo + 1, find(lo + 1), odd);
                note(lo, even);
                at = find(lo + 2);
            }
            __syncthreads();
            fetch(lo);
            put(lo);
            fetch(lo + 1);
            __syncthreads();
            if (tid < kTile) {
                ask(lo + 2, at, even);
                at = find(lo + 3);
            }
            __syncthreads();
            // at the top: tile t in LDS, the codes of t + 1 and scales of t + 1, t + 2 under way.  (Behind the last tile rows are 0: loads that nobody uses.)
            for (int32_t t = lo; t < hi; ++t) {
                put(t + 1);
                fetch(t + 2);
                if (tid < kTile) {
                    note(t + 1, odd);
                    ask(t + 3, at, odd);
                    at = find(t + 4);
                    const Ahead swap = odd;
                    odd = even, even = swap;
                }
                if (busy) use(t);
                __syncthreads();
            }
        }

        if (busy) {
            const int g = opaque(threadIdx.x & 63) >> 5;
            total += __shfl_xor(total, 32);
            const bool mine = first + 32u * wave + r <= last;
            const float inverse = total == 0.0f ? 0.0f : 1.0f / total;
            const int64_t to = ((int64_t)split * a.tokens + row.token) * a.heads_q + row.head;
            if (mine && a.splits > 1 && g == 0) a.state[to] = make_float2(level, total);
            // four values 4 x + 0 .. 3 are at rows x, x + DP / 4, ..; of them this lane has x = 8 e + 4 g + 0 .. 3
#pragma unroll
            for (int e = 0; e < DP / 32; ++e)
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    float y[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int at_row = (j & 3) * (DP / 4) + 8 * e;
                        y[j] = out[at_row / 32][at_row % 32 / 8 * 4 + i + (j >> 2)];
                    }
                    const int d = 4 * (8 * e + 4 * g + i);
                    if (mine && d < a.D) {
                        if (a.splits == 1) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) y[j] = total == 0.0f ? 0.0f : y[j] * inverse;
                            store_eight<T>(a.out, row.token * a.ld_out + row.head * a.step_out + d, y);
                        } else if (!(total == 0.0f)) {
                            __builtin_memcpy(a.part + to * a.D + d, y, sizeof y);
                        }
                    }
                }
        }
    }
}

template <typename T, int DP, int kWaves>
int launch(const Args &a, dim3 grid, hipStream_t s) {
    auto kernel = a.cap > 0.0f ? (a.cap > kCloseFrom ? many_rows_kernel<T, DP, kWaves, 3> : many_rows_kernel<T, DP, kWaves, kAlwaysClose<T> ? 3 : 2>)
                               : (a.slopes ? many_rows_kernel<T, DP, kWaves, 1> : many_rows_kernel<T, DP, kWaves, 0>);
    return QNN_LAUNCH("cache_attention", kernel, grid, dim3(64 * kWaves), 0, s, a);
}

}  // namespace

int launch_many(const Args &a, int type, dim3 grid, hipStream_t s) {
    return rows::with_type(type, [&](auto tag) {
        typedef decltype(tag) T;
        if (a.D <= 64) return launch<T, 64, 8>(a, grid, s);
        if (a.D <= 128) return launch<T, 128, 8>(a, grid, s);
        if constexpr (!std::is_same<T, float>::value) return launch<T, 256, 4>(a, grid, s);
        return fail(QNN_ERR_UNSUPPORTED, "cache_attention: no kernel");  // (as takes_many says)
    });
}

}  // namespace attention
}  // namespace qnn
