// Matrix product of int8 codes with one scale for each row of either operand: out[m][n] = scaleA[m] scaleW[n] sum_k A[m][k] W[n][k] + bias[n], written as
// fp32, fp16 or bf16.  The sums are exact int32 (v_mfma_i32_*_i8); the scales and the bias are applied in fp32 on the way out, rounded once.
#include <cmath>

#include "qnn_int8_panel.h"

namespace qnn {
namespace int8 {
namespace {

using rows::bf16;
using rows::f16;
using rows::kVec;

// 16 kCols weight rows against 16 kTiles rows of A a workgroup, its waves every kWaves-th step of 128 codes, each through its own ring in LDS
template <typename T, int kCols, int kTiles, int kWaves, int kStages, Layout kLayout>
__global__ __launch_bounds__(64 * kWaves) void gemm_stream_kernel(const Args<T> a, const Tiles tiles) {
    typedef Stream<kCols, kTiles, kStages, kLayout> S;
    constexpr int kRows = 16 * kTiles, kColumns = 16 * kCols, kPitch = kColumns + 4, kHalf = kWaves / 2 > 0 ? kWaves / 2 : 1;
    constexpr int kJoin = kHalf * kRows * kPitch * 4, kLds = S::kBytes * kWaves > kJoin ? S::kBytes * kWaves : kJoin;
    __shared__ __attribute__((aligned(16))) uint8_t lds[kLds];
    uint32_t tm, tn;
    tile_of_block(blockIdx.x, tiles, tm, tn);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int64_t m0 = (int64_t)tm * kRows, n0 = (int64_t)tn * kColumns;
    S s;
    s.lds = lds + wave * S::kBytes;
    s.x_base = a.A, s.K = (uint32_t)a.K;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int c = 0; c < kCols; ++c) s.off[c][h] = (typename S::Offset)(min(n0 + 16 * c + 8 * h + (lane >> 3), a.N - 1) * a.ldw);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) s.off[kCols + t][h] = (typename S::Offset)(min(m0 + 16 * t + 8 * h + (lane >> 3), a.M - 1) * a.lda);
    }
    v4i acc[kCols][kTiles] = {};
    s.sums(a.W, 128u * wave, 128u * kWaves, acc);
    __syncthreads();  // (every wave is done with its ring)
    int32_t(*const sums)[kRows][kPitch] = reinterpret_cast<int32_t(*)[kRows][kPitch]>(lds);
    auto put = [&](int at) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
            for (int t = 0; t < kTiles; ++t) *reinterpret_cast<v4i *>(&sums[at][16 * t + r][16 * c + 4 * g]) = acc[c][t];
    };
    // the upper half of the waves hands its sums to the lower half, and the sums of these are added where they are written
    if (wave >= kHalf) put(wave - kHalf);
    __syncthreads();
    if (wave < kHalf) {
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
            for (int t = 0; t < kTiles; ++t) acc[c][t] += *reinterpret_cast<const v4i *>(&sums[wave][16 * t + r][16 * c + 4 * g]);
        put(wave);
    }
    __syncthreads();
    constexpr int kFours = kColumns / 4;  // four columns a lane
    for (int i = threadIdx.x; i < kRows * kFours; i += 64 * kWaves) {
        const int row = i / kFours, col = 4 * (i % kFours);
        const int64_t m = m0 + row, n = n0 + col, here = a.N - n;
        if (m >= a.M || here <= 0) continue;
        v4i sum = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kHalf; ++w) sum += *reinterpret_cast<const v4i *>(&sums[w][row][col]);
        const float sa = a.scaleA[m];
        struct Four {
            T e[4];
        } four;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t at = min(n + e, a.N - 1);
            four.e[e] = (T)((float)sum[e] * sa * a.scaleW[at] + (a.bias ? a.bias[at] : 0.0f));
        }
        T *const to = a.out + m * a.ldo + n;
        if (here >= 4) {
            __builtin_memcpy(to, &four, sizeof four);
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < here) to[e] = four.e[e];
        }
    }
}

// 128 x 128 on four waves of 64 x 64, two workgroups on a compute unit; groups of 128 codes through registers to LDS, two buffers; rows of any length at
// any address (K >= 16).  A group's loads are sent two groups ahead (one ahead, their latency was half of the time: 1999 x 3001 x 2500 38.2 us, and 34.4).
// 16-byte piece c of row r sits at piece c xor (r / 2 mod 8): the 16 rows that a read serves at a time lie on different banks.
constexpr int kTile = 128, kGroup = 128, kPanel = kTile * kGroup;

template <typename T>
__global__ __launch_bounds__(256, 2) void gemm_tile_kernel(const Args<T> a, const Tiles tiles) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][2 * kPanel];
    uint32_t tm, tn;
    tile_of_block(blockIdx.x, tiles, tm, tn);
    const int t = threadIdx.x, wave = t >> 6, lane = t & 63, wm = wave >> 1, wn = wave & 1;
    const int64_t m0 = (int64_t)tm * kTile, n0 = (int64_t)tn * kTile;
    // a thread loads piece t mod 8 of rows t / 8 + 32 i
    const int piece = t & 7;
    const int8_t *src[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        src[i] = a.A + min(m0 + (t >> 3) + 32 * i, a.M - 1) * a.lda;
        src[4 + i] = a.W + min(n0 + (t >> 3) + 32 * i, a.N - 1) * a.ldw;
    }
    auto fetch = [&](int64_t k, v4i (&in)[8]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) in[i] = load_window(src[i], k + 16 * piece, a.K);
    };
    auto put = [&](int buf, v4i (&in)[8], int64_t k) __attribute__((always_inline)) {
        if (k + kGroup > a.K) {
#pragma unroll
            for (int i = 0; i < 8; ++i) in[i] = in_place(in[i], k + 16 * piece, a.K);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = (t >> 3) + 32 * (i & 3);
            *reinterpret_cast<v4i *>(&lds[buf][(i >> 2) * kPanel + row * kGroup + 16 * (piece ^ ((row >> 1) & 7))]) = in[i];
        }
    };
    v4i acc[4][4] = {};  // [n block][m block] of 16 x 16
    const int r = lane & 15, g = lane >> 4;
    auto multiply = [&](int buf) __attribute__((always_inline)) {
        v4i x[2][4], w[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = r * kGroup + 16 * ((4 * h + g) ^ ((r >> 1) & 7));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[h][i] = *reinterpret_cast<const v4i *>(&lds[buf][(64 * wm + 16 * i) * kGroup + at]);
                w[h][i] = *reinterpret_cast<const v4i *>(&lds[buf][kPanel + (64 * wn + 16 * i) * kGroup + at]);
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[h][i], x[h][j], acc[i][j], 0, 0, 0);
    };
    v4i even[8], odd[8];
    fetch(0, even);
    fetch(kGroup, odd);
    put(0, even, 0);
    auto turn = []() __attribute__((always_inline)) {  // (written and, the other buffer, read; loads stay under way)
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    // at the top: group k in buffer 0, the loads of the next in `odd` under way
    int64_t k = 0;
    for (; k + 2 * kGroup < a.K; k += 2 * kGroup) {
        turn();
        fetch(k + 2 * kGroup, even);
        multiply(0);
        put(1, odd, k + kGroup);
        turn();
        fetch(k + 3 * kGroup, odd);
        multiply(1);
        put(0, even, k + 2 * kGroup);
    }
    turn();
    multiply(0);
    if (k + kGroup < a.K) {
        put(1, odd, k + kGroup);
        turn();
        multiply(1);
    }
    __syncthreads();
    // A wave's sums of 32 rows pass through its part of LDS and leave as rows of 64 columns, 8 columns a lane
    constexpr int kPitch = 64 + 4;
    float *const stage = reinterpret_cast<float *>(&lds[0][0]) + wave * 32 * kPitch;
    static_assert(4 * 32 * kPitch * 4 <= sizeof lds, "");
    const int64_t n = n0 + 64 * wn + 8 * (lane & 7), n_here = a.N - n;
    float sw[kVec], bias[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
        sw[e] = e < n_here ? a.scaleW[n + e] : 0.0f;
        bias[e] = a.bias && e < n_here ? a.bias[n + e] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float *const to = stage + (16 * h + r) * kPitch + 16 * i + 4 * g;
#pragma unroll
                for (int e = 0; e < 4; ++e) to[e] = (float)acc[i][2 * j + h][e];
            }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 8 * i + (lane >> 3);
            const int64_t m = m0 + 64 * wm + 32 * j + row;
            if (m < a.M && n_here > 0) {
                const float sa = a.scaleA[m];
                float y[kVec];
#pragma unroll
                for (int e = 0; e < kVec; ++e) y[e] = stage[row * kPitch + 8 * (lane & 7) + e] * sa * sw[e] + bias[e];
                T *const to = a.out + m * a.ldo + n;
                rows::Raw<T> out;
#pragma unroll
                for (int e = 0; e < kVec; ++e) out.e[e] = (T)y[e];
                if (n_here >= kVec) {
                    __builtin_memcpy(to, &out, sizeof out);
                } else {
#pragma unroll
                    for (int e = 0; e < kVec; ++e)
                        if (e < n_here) to[e] = out.e[e];
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
}

// The ways a product can go, by rows and columns of a workgroup's tile.  The least start + more (R - 1) + k R K / 1024 is taken, with R the rounds of `side` tiles
// a compute unit: formed like a time in us, but it only ranks the ways (one round or many, and what overlaps, share one line; 2000 x 4096 x 4096 on the pairs comes
// out as 28 and takes 35).  Fitted to products of all three kinds of rows, judged on others: 200 of each kind drawn over 1 .. 20000 rows, 64 .. 12000 columns and
// K of 16 .. 9000, where the way that comes out ahead takes in the mean 1.6 % (pieces), 1.8 % (words) and 0.7 % (any rows) longer than the fastest of all, and 22,
// 32 and 31 % at most.  (us at N = K = 4096, bf16 out, inputs in the caches: M = 16: 16 x 16 3.8, 64 x 16 5.3; 64: 64 x 16 6.1, 64 x 32 6.5, 16 x 16 8.3;
// 128: 64 x 32 6.9, 64 x 64 9.1, 64 x 16 10.1; 256: 64 x 64 10.5, panels of 64 x 64 11.1, 64 x 32 12.2; 512: panels of 64 x 64 15.3, of 128 x 128 on eight waves
// 16.9 and in pairs 22.3, streams 19.3; 1024: 29.4, 21.5, 26.1; 2000: 56.1, 39.6, 35.1, 256 x 256 42.2; 5000: 137, 95, 86, 89; 8192 x 8192 x 8192: 824, 553, 507,
// 386.)  The pairs are two workgroups on a compute unit: counted as one round of two tiles, since with rounds of one the choice costs 3.9 % where this costs 1.9.
enum WayId { kStream16x16, kStream64x16, kStream64x32, kStream64x64, kPanel64, kPanel128, kPanel128Pairs, kPanel256, kTile128 };
struct Way {
    WayId id;
    int rows, columns, side;
    double start, more, k;
};
constexpr Way kWaysOfPieces[] = {{kStream16x16, 16, 16, 1, 2.7, 0.56, 0.276},     {kStream64x16, 64, 16, 1, 3.1, 1.95, 0.743}, {kStream64x32, 64, 32, 1, 3.3, 2.37, 0.924},
                                 {kStream64x64, 64, 64, 1, 4.3, 3.93, 1.306},     {kPanel64, 64, 64, 1, 3.6, 0.80, 1.600},     {kPanel128, 128, 128, 1, 4.7, 2.51, 4.068},
                                 {kPanel128Pairs, 128, 128, 2, 4.7, 8.98, 5.945}, {kPanel256, 256, 256, 1, 6.4, 9.10, 8.518}};
// Rows at any address
constexpr Way kWaysOfAny[] = {{kStream16x16, 16, 16, 1, 2.8, 0.33, 0.671},
                              {kStream64x16, 64, 16, 1, 3.4, 1.04, 1.610},
                              {kStream64x32, 64, 32, 1, 3.9, 3.11, 2.022},
                              {kStream64x64, 64, 64, 1, 5.2, 4.72, 2.982},
                              {kTile128, 128, 128, 1, 6.2, 4.49, 7.015}};
// Rows of whole words: streams as above, panels.  (300 x 4100 x 3004: panels of 64 x 64 16.7 us, streams of 64 x 64 18.0; 4000 x 4000 x 4004: 256 x 256 69,
// 128 x 128 96; 1999 x 3001 x 2500: 128 x 128 29.5, 256 x 256 43.6.  Counting the pairs two tiles a round changes nothing here: 2.6 and 2.5 %.)
constexpr Way kWaysOfWords[] = {{kStream16x16, 16, 16, 1, 2.8, 0.33, 0.671}, {kStream64x16, 64, 16, 1, 3.4, 1.04, 1.610},
                                {kStream64x32, 64, 32, 1, 3.9, 3.11, 2.022}, {kStream64x64, 64, 64, 1, 5.2, 4.72, 2.982},
                                {kPanel64, 64, 64, 1, 5.4, 0.80, 2.486},     {kPanel128Pairs, 128, 128, 1, 6.8, 1.21, 5.749},
                                {kPanel256, 256, 256, 1, 9.8, 11.65, 12.12}};
template <int kCount>
const Way &fastest(const Way (&ways)[kCount], int64_t M, int64_t N, int64_t K) {
    const Way *best = nullptr;
    double least = 0.0;
    for (const Way &w : ways) {
        const double rounds = std::ceil((double)ceil_div(M, w.rows) * (double)ceil_div(N, w.columns) / (compute_units() * w.side));
        const double us = w.start + w.more * (rounds - 1.0) + w.k * rounds * (double)K / 1024.0;
        if (!best || us < least) best = &w, least = us;
    }
    return *best;
}

constexpr int64_t kMostTiles = 1 << 22;  // of 512 threads: HIP launches fewer than 2^32 along a dimension

template <typename T>
int launch(const Args<T> &a, hipStream_t s) {
    const bool pieces = in_pieces(a.A, a.lda, a.M, a.K) && in_pieces(a.W, a.ldw, a.N, a.K), any = !pieces && a.K >= 16;
    const bool words = any && in_words(a.A, a.lda, a.M, a.K) && in_words(a.W, a.ldw, a.N, a.K);
    const Way &w = pieces  ? fastest(kWaysOfPieces, a.M, a.N, a.K)
                   : words ? fastest(kWaysOfWords, a.M, a.N, a.K)
                   : any   ? fastest(kWaysOfAny, a.M, a.N, a.K)
                           : kWaysOfAny[0];
    const int64_t tm = ceil_div(a.M, w.rows), tn = ceil_div(a.N, w.columns);
    if ((double)tm * (double)tn > kMostTiles) {  // in two parts
        Args<T> one = a, two = a;
        if (tm >= tn) {
            const int64_t m = tm / 2 * w.rows;
            one.M = m, two.M -= m, two.A += m * a.lda, two.scaleA += m, two.out += m * a.ldo;
        } else {
            const int64_t n = tn / 2 * w.columns;
            one.N = n, two.N -= n, two.W += n * a.ldw, two.scaleW += n, two.bias += a.bias ? n : 0, two.out += n;
        }
        const int rc = launch(one, s);
        return rc ? rc : launch(two, s);
    }
    const Tiles tiles = make_tiles(tm, tn);
    const dim3 grid((unsigned)(tm * tn));
    auto stream = [&](auto on_pieces, auto on_any) { return QNN_LAUNCH("int8_gemm", (pieces ? on_pieces : on_any), grid, dim3(512), 0, s, a, tiles); };
    auto panels_of = [&](auto shape) {
        typedef decltype(shape) S;
        const int64_t most = (int64_t)compute_units() * S::kPerUnit;
        return QNN_LAUNCH("int8_gemm", (panel::gemm_panel_kernel<T, S>), dim3((unsigned)(tm * tn < most ? tm * tn : most)), dim3(S::kThreads), 0, s, a, tiles,
                          (uint32_t)ceil_div(a.K, panel::kRow));
    };
    auto panels = [&](auto shape, auto shape_of_words) { return words ? panels_of(shape_of_words) : panels_of(shape); };
    if (!pieces && !any) return QNN_LAUNCH("int8_gemm", (gemm_stream_kernel<T, 1, 1, 8, 1, kShortRows>), grid, dim3(512), 0, s, a, tiles);
    switch (w.id) {
    case kStream16x16: return stream(gemm_stream_kernel<T, 1, 1, 8, 2, kPieces>, gemm_stream_kernel<T, 1, 1, 8, 2, kAny>);
    case kStream64x16: return stream(gemm_stream_kernel<T, 1, 4, 8, 2, kPieces>, gemm_stream_kernel<T, 1, 4, 8, 1, kAny>);
    case kStream64x32: return stream(gemm_stream_kernel<T, 2, 4, 8, 1, kPieces>, gemm_stream_kernel<T, 2, 4, 8, 1, kAny>);
    case kStream64x64: return stream(gemm_stream_kernel<T, 4, 4, 8, 1, kPieces>, gemm_stream_kernel<T, 4, 4, 8, 1, kAny>);
    case kPanel64: return panels(panel::Tiny(), panel::TinyWords());
    case kPanel128: return panels_of(panel::Eight());
    case kPanel128Pairs: return panels(panel::Small(), panel::SmallWords());
    case kPanel256: return panels(panel::Large(), panel::LargeWords());
    case kTile128: return QNN_LAUNCH("int8_gemm", gemm_tile_kernel<T>, grid, dim3(256), 0, s, a, tiles);
    }
    return fail(QNN_ERR_UNSUPPORTED, "int8_gemm: no way");
}

}  // namespace
}  // namespace int8
}  // namespace qnn

using namespace qnn;

extern "C" int qnn_int8_gemm(const int8_t *A, int64_t lda, const float *scaleA, const int8_t *W, int64_t ldw, const float *scaleW, const float *bias,
                             void *out, int64_t ldo, int type, int64_t M, int64_t N, int64_t K, void *stream) {
    if (M < 0 || N < 0 || K < 1) return fail(QNN_ERR_SHAPE, "int8_gemm: M = %lld, N = %lld, K = %lld", (long long)M, (long long)N, (long long)K);
    if (!rows::known_type(type)) return fail(QNN_ERR_SHAPE, "int8_gemm: type %d", type);
    if (lda < K || ldw < K || ldo < N) return fail(QNN_ERR_SHAPE, "int8_gemm: leading dimension too small");
    if (K > int8::kMostK) return fail(QNN_ERR_OVERFLOW, "int8_gemm: sums of K = %lld products of codes do not fit int32", (long long)K);
    if (M == 0 || N == 0) return QNN_OK;
    if (!A || !scaleA || !W || !scaleW || !out) return fail(QNN_ERR_NULL, "int8_gemm: NULL pointer");
    if (!rows::aligned_to(scaleA, 4) || !rows::aligned_to(scaleW, 4) || !rows::aligned_to(bias, 4) || !rows::aligned_to(out, rows::value_bytes(type)))
        return fail(QNN_ERR_ALIGN, "int8_gemm: pointer not aligned to its type");
    return rows::with_type(type, [&](auto tag) {
        typedef decltype(tag) T;
        return int8::launch(int8::Args<T>{A, W, scaleA, scaleW, bias, static_cast<T *>(out), lda, ldw, ldo, M, N, K}, static_cast<hipStream_t>(stream));
    });
}
