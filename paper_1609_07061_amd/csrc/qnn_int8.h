// Shared by the kernels on int8 codes (qnn_int8_gemm.hip, qnn_int8_moe.hip): operands of the matrix cores from rows of codes at any address and of any
// length, and the small product of a few rows whose waves share k.
#pragma once
#include "qnn_rows.h"

namespace qnn {
namespace int8 {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));

// Codes k0 .. k0 + 15 of a row of K, zero beyond it; nothing beyond the row is read.  (One operand's zeros are enough for a product.)
__device__ __forceinline__ v4i load16(const int8_t *row, int64_t k0, int64_t K) {
    v4i v = {0, 0, 0, 0};
    if (k0 + 16 <= K) {
        __builtin_memcpy(&v, row + k0, 16);
    } else if (k0 < K) {
        if (K >= 16) {  // the row's last 16 codes, moved down
            uint64_t w[2];
            __builtin_memcpy(w, row + K - 16, 16);
            const int shift = 8 * (int)(k0 + 16 - K);  // 8 .. 120
            const uint64_t lo = shift < 64 ? (w[0] >> shift) | (w[1] << (64 - shift)) : w[1] >> (shift - 64), hi = shift < 64 ? w[1] >> shift : 0u;
            v = v4i{(int)lo, (int)(lo >> 32), (int)hi, (int)(hi >> 32)};
        } else {
            uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < 15; ++i)
                if (k0 + i < K) w[i >> 2] |= (uint32_t)(uint8_t)row[k0 + i] << (8 * (i & 3));
            v = v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
        }
    }
    return v;
}

// Sums of a wave's share of k: up to 16 kCols weight rows against 16 kTiles rows of codes.  Lane l of an operand holds 16 codes of row l mod 16, the
// four groups of 16 lanes consecutive ones; acc[c][t][v] is weight row 16 c + 4 (l / 16) + v and code row 16 t + l mod 16.
// w_row[c], x_row[t]: this lane's rows.  Steps of 64 codes first, first + stride, ... below K; kAhead steps' loads are sent before they are needed.
template <int kCols, int kTiles, int kAhead>
__device__ __forceinline__ void multiply_rows(const int8_t *const (&w_row)[kCols], const int8_t *const (&x_row)[kTiles], int64_t K, int64_t first,
                                              int64_t stride, v4i (&acc)[kCols][kTiles]) {
    const int64_t at = 16 * ((threadIdx.x & 63) >> 4);
    for (int64_t k = first; k < K; k += stride * kAhead) {
        v4i w[kAhead][kCols], x[kAhead][kTiles];
        if (k + stride * (kAhead - 1) + 64 <= K) {
#pragma unroll
            for (int s = 0; s < kAhead; ++s) {
#pragma unroll
                for (int c = 0; c < kCols; ++c) __builtin_memcpy(&w[s][c], w_row[c] + k + s * stride + at, 16);
#pragma unroll
                for (int t = 0; t < kTiles; ++t) __builtin_memcpy(&x[s][t], x_row[t] + k + s * stride + at, 16);
            }
        } else {
#pragma unroll
            for (int s = 0; s < kAhead; ++s) {
#pragma unroll
                for (int c = 0; c < kCols; ++c) w[s][c] = load16(w_row[c], k + s * stride + at, K);
#pragma unroll
                for (int t = 0; t < kTiles; ++t) x[s][t] = load16(x_row[t], k + s * stride + at, K);
            }
        }
#pragma unroll
        for (int s = 0; s < kAhead; ++s)
#pragma unroll
            for (int c = 0; c < kCols; ++c)
#pragma unroll
                for (int t = 0; t < kTiles; ++t) acc[c][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[s][c], x[s][t], acc[c][t], 0, 0, 0);
    }
}

// Products with K codes of at most 128 in magnitude are exact in int32
constexpr int64_t kMostK = 131071;

}  // namespace int8
}  // namespace qnn
