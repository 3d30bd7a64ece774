// Shared by the kernels on int8 codes (qnn_int8_gemm.hip, qnn_int8_moe.hip): operands of the matrix cores from rows of codes at any address and of any
// length, and the small product of a few rows whose waves share k.
#pragma once
#include <type_traits>

#include "qnn_rows.h"

namespace qnn {
namespace int8 {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));

// Codes k .. k + 15 of a row of K >= 16, zero beyond it, in two steps: the load, of the row's last 16 codes where it would go beyond them, and, once it has
// come in, the shift into place.  (A load that depended on a branch would be waited for at the branch's end.)  Nothing beyond the row is read.
__device__ __forceinline__ v4i load_window(const int8_t *row, int64_t k, int64_t K) {
    v4i v;
    __builtin_memcpy(&v, row + min(k, K - 16), 16);
    return v;
}
__device__ __forceinline__ v4i in_place(const v4i &v, int64_t k, int64_t K) {
    // codes to leave out: a shift by as many bytes, words first, without a branch (1356 x 384 x 767: 8.7 us with branches, 7.7 so)
    const int64_t over = k + 16 - K;
    const uint32_t bytes = (uint32_t)(over < 0 ? 0 : (over > 16 ? 16 : over));
    uint32_t x[5] = {(uint32_t)v[0], (uint32_t)v[1], (uint32_t)v[2], (uint32_t)v[3], 0u};
    const bool four = (bytes & 16u) != 0u, two = (bytes & 8u) != 0u, one = (bytes & 4u) != 0u;
    x[0] = two ? x[2] : x[0], x[1] = two ? x[3] : x[1], x[2] = two ? 0u : x[2], x[3] = two ? 0u : x[3];
    x[0] = one ? x[1] : x[0], x[1] = one ? x[2] : x[1], x[2] = one ? x[3] : x[2], x[3] = one ? 0u : x[3];
    v4i out;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = four ? 0 : (int)__builtin_amdgcn_alignbyte(x[i + 1], x[i], bytes);
    return out;
}
// The same for a row of fewer than 16 codes
__device__ __forceinline__ v4i load_short(const int8_t *row, int64_t k, int64_t K) {
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 15; ++i)
        if (k + i < K) w[i >> 2] |= (uint32_t)(uint8_t)row[k + i] << (8 * (i & 3));
    return v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
}
// How rows of codes are loaded: kPieces: whole 16-byte pieces at 16-byte aligned addresses, within 4 GiB; kPiecesOnce: the same, and the weights past the
// caches; kAny; kShortRows: fewer than 16 codes
enum Layout { kPieces, kPiecesOnce, kAny, kShortRows };

// A wave's own stream of operands: steps of 128 codes of 16 kCols weight rows and 16 kTiles rows of codes, brought to LDS in whole lines (8 rows of 128
// bytes a load) and read from there as the matrix cores take them.  Loaded straight into place, lane l of an operand having 16 codes of row l mod 16,
// neighbouring lanes are different rows and the 64 pieces of a load are taken one by one: 16 bytes a cycle and compute unit, against 64 in whole lines (4096
// codes of 128 x 4096 rows: 18.8 us, and 8.3 like this).  Nobody waits for another wave.  Piece c of row r is at piece c xor (r / 2 mod 8): the 16 rows
// that a read serves at a time lie on different banks.
// Pieces: loads straight to LDS, kStages steps there.  Otherwise kStages steps in registers, which pass through one place in LDS.
template <int kCols, int kTiles, int kStages, Layout kLayout>
struct Stream {
    static constexpr bool kRing = kLayout == kPieces || kLayout == kPiecesOnce;
    static constexpr int kRows = kCols + kTiles, kLoads = 2 * kRows, kStage = 1024 * kLoads, kBytes = (kRing ? kStages : 1) * kStage;
    static_assert(kStages <= 4 && (kStages - 1) * kLoads <= 63, "a count of loads that s_waitcnt can name");
    typedef std::conditional_t<kRing, uint32_t, int64_t> Offset;
    struct Operands {
        v4i w[2][kCols], x[2][kTiles > 0 ? kTiles : 1];  // codes 0 .. 63 and 64 .. 127 of a step
    };

    uint8_t *lds;          // this wave's part
    const int8_t *x_base;  // (the weights' may change from step to step)
    Offset off[kRows][2];  // of the rows this lane loads, 8 h + lane / 8 of a block; weights first
    uint32_t K;
    v4i held[kRing ? 1 : kStages][kRing ? 1 : kLoads];
    uint32_t under_way[kStages];  // where the steps in the stages begin

    // sends the loads of the step at k0 to stage s
    __device__ __forceinline__ void send(const int s, const int8_t *w_base, uint32_t k0) {
        const uint32_t lane = threadIdx.x & 63u;
        under_way[s] = k0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t k = k0 + (((lane & 7u) ^ ((4u * h + (lane >> 4)) & 7u)) << 4);
            if constexpr (kRing) k = k < K ? k : 0u;  // beyond the rows: their beginning
#pragma unroll
            for (int b = 0; b < kRows; ++b) {
                const int8_t *const base = b < kCols ? w_base : x_base;
                if constexpr (kRing) {
                    const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t *)lds)) +
                                        (uint32_t)(s * kStage + 2048 * b + 1024 * h);
                    if (kLayout == kPiecesOnce && b < kCols)
                        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" : : "s"(to), "v"(off[b][h] + k), "s"(base) : "memory");
                    else
                        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(off[b][h] + k), "s"(base) : "memory");
                } else {
                    held[s][2 * b + h] = kLayout == kAny ? load_window(base + off[b][h], k, K) : load_short(base + off[b][h], k, K);
                }
            }
        }
    }
    // the operands of the step at k0, in stage s; `after` steps are under way behind it
    __device__ __forceinline__ void take(const int s, uint32_t k0, int after, Operands &o) {
        const uint32_t lane = threadIdx.x & 63u, r = lane & 15u, g = lane >> 4;
        uint8_t *const at = lds + (kRing ? s * kStage : 0);
        if constexpr (kRing) {
            if (kStages > 3 && after >= 3)
                asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kStages > 3 ? 3 * kLoads : 0) : "memory");
            else if (kStages > 2 && after >= 2)
                asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kStages > 2 ? 2 * kLoads : 0) : "memory");
            else if (kStages > 1 && after >= 1)
                asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kStages > 1 ? kLoads : 0) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        } else {
            if (kLayout == kAny && k0 + 128u > K) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) held[s][i] = in_place(held[s][i], k0 + (((lane & 7u) ^ ((4u * (i & 1) + (lane >> 4)) & 7u)) << 4), K);
            }
#pragma unroll
            for (int i = 0; i < kLoads; ++i) *reinterpret_cast<v4i *>(at + 1024 * i + 16 * lane) = held[s][i];
            in_wave();
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t piece = r * 128u + (((4u * h + g) ^ ((r >> 1) & 7u)) << 4);
#pragma unroll
            for (int c = 0; c < kCols; ++c) o.w[h][c] = *reinterpret_cast<const v4i *>(at + 2048 * c + piece);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) o.x[h][t] = *reinterpret_cast<const v4i *>(at + 2048 * (kCols + t) + piece);
        }
        if (kRing && k0 + 128u > K) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (k0 + 64u * h + 16u * g >= K) {
#pragma unroll
                    for (int c = 0; c < kCols; ++c) o.w[h][c] = v4i{0, 0, 0, 0};
                }
        }
        if constexpr (kRing)
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // read before it is overwritten
        else
            in_wave();
    }
    // what a wave has written to LDS is there for its own reads (its LDS operations are done in order)
    __device__ __forceinline__ static void in_wave() {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
    // n steps: step i's weights are at base(i), its codes from at(i) on, asked in this order; use(i, operands).  start() before, which may be well before.
    template <typename Base, typename At>
    __device__ __forceinline__ void start(int n, Base base, At at) {
#pragma unroll
        for (int s = 0; s < kStages; ++s)
            if (s < n) {
                const int8_t *const from = base(s);
                send(s, from, at(s));
            }
    }
    template <typename Base, typename At, typename Use>
    __device__ __forceinline__ void run(int n, Base base, At at, Use use) {
        for (int i = 0; i < n; i += kStages) {
#pragma unroll
            for (int s = 0; s < kStages; ++s)
                if (i + s < n) {
                    Operands o;
                    take(s, under_way[s], n - 1 - i - s, o);
                    if (i + s + kStages < n) {
                        const int8_t *const from = base(i + s + kStages);
                        send(s, from, at(i + s + kStages));
                    }
                    use(i + s, o);
                }
        }
    }
    // all steps of a wave's share of k: those at first, first + stride, ... below K
    __device__ __forceinline__ void sums(const int8_t *w_base, uint32_t first, uint32_t stride, v4i (&acc)[kCols][kTiles > 0 ? kTiles : 1]) {
        const int n = K > first ? (int)((K - first - 1u) / stride) + 1 : 0;
        auto base = [&](int) __attribute__((always_inline)) { return w_base; };
        auto at = [&](int i) __attribute__((always_inline)) { return first + (uint32_t)i * stride; };
        start(n, base, at);
        run(n, base, at, [&](int, const Operands &o) __attribute__((always_inline)) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int c = 0; c < kCols; ++c) acc[c][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(o.w[h][c], o.x[h][t], acc[c][t], 0, 0, 0);
        });
    }
};

inline bool in_pieces(const int8_t *p, int64_t ld, int64_t n_rows, int64_t K) {
    return K % 16 == 0 && ld % 16 == 0 && rows::aligned_to(p, 16) && (long double)n_rows * ld < 4294967296.0L;
}

// Rows of whole 4-byte words at 4-byte aligned addresses, within 4 GiB
inline bool in_words(const int8_t *p, int64_t ld, int64_t n_rows, int64_t K) {
    return K % 4 == 0 && ld % 4 == 0 && rows::aligned_to(p, 4) && (long double)n_rows * ld < 4294967296.0L;
}

// Products with K codes of at most 128 in magnitude are exact in int32
constexpr int64_t kMostK = 131071;

}  // namespace int8
}  // namespace qnn
