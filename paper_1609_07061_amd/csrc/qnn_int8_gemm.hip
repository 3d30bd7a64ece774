// Matrix product of int8 codes with one scale for each row of either operand: out[m][n] = scaleA[m] scaleW[n] sum_k A[m][k] W[n][k] + bias[n], written as
// fp32, fp16 or bf16.  The sums are exact int32 (v_mfma_i32_*_i8); the scales and the bias are applied in fp32 on the way out, rounded once.
#include "qnn_int8.h"

namespace qnn {
namespace int8 {
namespace {

using rows::bf16;
using rows::f16;
using rows::kVec;

template <typename T>
struct Args {
    const int8_t *A, *W;
    const float *scaleA, *scaleW, *bias;  // bias may be null
    T *out;
    int64_t lda, ldw, ldo, M, N, K;
};

// ---------------------------------------------------------------------------------------------------------------- few rows
// Up to 16 kTiles rows of A: a workgroup has 16 weight rows, its waves every kWaves-th step of 64 codes, and adds its waves' sums in LDS.
template <typename T, int kTiles, int kWaves>
__global__ __launch_bounds__(64 * kWaves) void gemm_few_kernel(const Args<T> a) {
    __shared__ int32_t sums[kWaves][16 * kTiles][17];
    const int wave = threadIdx.x >> 6, r = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * (16 * kTiles);
    const int8_t *w_row[1], *x_row[kTiles];
    w_row[0] = a.W + min(n0 + r, a.N - 1) * a.ldw;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) x_row[t] = a.A + min(m0 + 16 * t + r, a.M - 1) * a.lda;
    v4i acc[1][kTiles] = {};
    multiply_rows<1, kTiles, 4>(w_row, x_row, a.K, 64 * wave, 64 * kWaves, acc);
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v) sums[wave][16 * t + r][4 * g + v] = acc[0][t][v];
    __syncthreads();
    for (int i = threadIdx.x; i < 256 * kTiles; i += 64 * kWaves) {
        const int64_t m = m0 + (i >> 4), n = n0 + (i & 15);
        if (m >= a.M || n >= a.N) continue;
        int32_t s = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) s += sums[w][i >> 4][i & 15];
        float y = (float)s * a.scaleA[m] * a.scaleW[n];
        if (a.bias) y += a.bias[n];
        a.out[m * a.ldo + n] = (T)y;
    }
}

// ---------------------------------------------------------------------------------------------------------------- tiles
// 128 x 128 on four waves of 64 x 64; groups of 128 codes through registers to LDS, two buffers; rows of any length at any address.  16-byte piece c of
// row r sits at piece c xor (r / 2 mod 8): the 16 rows that a read serves at a time lie on different banks.
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
    v4i in[8];
    auto fetch = [&](int64_t k) __attribute__((always_inline)) {
        if (k + kGroup <= a.K) {
#pragma unroll
            for (int i = 0; i < 8; ++i) __builtin_memcpy(&in[i], src[i] + k + 16 * piece, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) in[i] = load16(src[i], k + 16 * piece, a.K);
        }
    };
    auto put = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = (t >> 3) + 32 * (i & 3);
            *reinterpret_cast<v4i *>(&lds[buf][(i >> 2) * kPanel + r * kGroup + 16 * (piece ^ ((r >> 1) & 7))]) = in[i];
        }
    };
    v16i acc[2][2] = {};
    const int r = lane & 31, kg = lane >> 5;
    fetch(0);
    put(0);
    __syncthreads();
    int buf = 0;
    for (int64_t k = 0; k < a.K; k += kGroup, buf ^= 1) {
        const bool more = k + kGroup < a.K;
        if (more) fetch(k + kGroup);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            v4i x[2], w[2];
            const int at = 16 * ((2 * s + kg) ^ ((r >> 1) & 7));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[i] = *reinterpret_cast<const v4i *>(&lds[buf][(64 * wm + 32 * i + r) * kGroup + at]);
                w[i] = *reinterpret_cast<const v4i *>(&lds[buf][kPanel + (64 * wn + 32 * i + r) * kGroup + at]);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[i], x[j], acc[i][j], 0, 0, 0);
        }
        if (more) put(buf ^ 1);
        __syncthreads();
    }
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
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int v = 0; v < 16; v += 4) {
                float *const to = stage + r * kPitch + 32 * i + 2 * v + 4 * kg;
#pragma unroll
                for (int e = 0; e < 4; ++e) to[e] = (float)acc[i][j][v + e];
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
                rows::store_values(a.out + m * a.ldo + n, y, n_here);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
}

template <typename T>
int launch(const Args<T> &a, hipStream_t s) {
    if (a.M <= 64) {
        const int64_t blocks = ceil_div(a.N, 16);
        if (blocks > 0x7FFFFFFFLL) return fail(QNN_ERR_SHAPE, "int8_gemm: N = %lld", (long long)a.N);
        const dim3 grid((unsigned)blocks);
        if (a.M <= 16) return QNN_LAUNCH("int8_gemm", (gemm_few_kernel<T, 1, 8>), grid, dim3(512), 0, s, a);
        if (a.M <= 32) return QNN_LAUNCH("int8_gemm", (gemm_few_kernel<T, 2, 8>), grid, dim3(512), 0, s, a);
        return QNN_LAUNCH("int8_gemm", (gemm_few_kernel<T, 4, 8>), grid, dim3(512), 0, s, a);
    }
    const int64_t tm = ceil_div(a.M, kTile), tn = ceil_div(a.N, kTile);
    if (tm > 0x7FFFFFFFLL || tn > 0x7FFFFFFLL || tm * tn > 0x7FFFFFFFLL) return fail(QNN_ERR_SHAPE, "int8_gemm: M = %lld, N = %lld", (long long)a.M, (long long)a.N);
    return QNN_LAUNCH("int8_gemm", gemm_tile_kernel<T>, dim3((unsigned)(tm * tn)), dim3(256), 0, s, a, make_tiles(tm, tn));
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
