// Large products of int8 codes with scales: both operands through LDS in whole 128-byte lines (global_load_lds), sums on the matrix cores
// (v_mfma_i32_16x16x64_i8), scales and rounding on the way out.  Rows of whole 16-byte pieces at 16-byte aligned addresses, or of 4-byte words.
//
// As in gemm_bytes_panel_kernel, a group of 128 codes of k is in an LDS buffer while others are loaded, 16-byte piece c of row r at piece c xor (r / 2 mod 8),
// and a persistent workgroup runs from tile to tile, its loads as many groups ahead of its products as there are buffers, so that a tile's end has the next
// one's operands in flight.  What is different is the way out (floats, half as wide or as wide as the sums) and that nothing pads the operands: codes of k
// beyond the rows are loaded from the rows' beginning and zeroed on one side behind LDS.
//
// What bounds it: at 8192 x 8192 x 8192 the card's power (codes of a normal distribution: 386 - 417 us, 2.6 - 2.8 P op/s, the matrix cores busy 73 % of
// 710 k cycles at 1.76 GHz; all zeros run at 2.44 GHz).  16 x 16 x 64 instead of 32 x 32 x 32 matrix instructions: half as many updates of sums a product,
// 484 -> 425 us.  At middle sizes the fixed part and LDS: 64 x 64 sums a wave read 64 KB and write 32 KB of LDS for 512 cycles of matrix instructions.
#pragma once
#include "qnn_int8.h"

namespace qnn {
namespace int8 {

template <typename T>
struct Args {
    const int8_t *A, *W;
    const float *scaleA, *scaleW, *bias;  // bias may be null
    T *out;
    int64_t lda, ldw, ldo, M, N, K;
};

namespace panel {

constexpr int kRow = 128;  // codes of a row in a group

// WM x WN waves, each with 32 BA rows of A and 32 BW rows of W; kRing groups in LDS; kPerUnit workgroups on a compute unit.  (1024 x 4096 x 4096 on 128 x 128:
// four waves 26.1 us, eight waves and four groups 21.5; two teams of four on alternate groups of k, or four groups in LDS for four waves, lay between.)
template <int WM_, int WN_, int BA_, int BW_, int kRing_, int kPerUnit_, bool kWords_ = false>
struct Shape {
    static constexpr int WM = WM_, WN = WN_, BA = BA_, BW = BW_, kRing = kRing_, kPerUnit = kPerUnit_;
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves, kRowsA = 32 * BA * WM, kRowsW = 32 * BW * WN;
    static constexpr bool kWords = kWords_;  // rows of whole 4-byte words at 4-byte aligned addresses, loaded word by word
    static constexpr int kPart = kWords ? 4 : 1;  // loads of 8 rows
    static constexpr int kLoadsA = kPart * kRowsA / (8 * kWaves), kLoadsW = kPart * kRowsW / (8 * kWaves), kLoads = kLoadsA + kLoadsW;  // a wave's of a group
    static constexpr int kGroup = (kRowsA + kRowsW) * kRow, kStage = 4096;  // bytes of a group; of a wave's part of the way out
    static constexpr int kLds = kRing * kGroup + kWaves * kStage;
    static_assert(kRowsA % (8 * kWaves) == 0 && kRowsW % (8 * kWaves) == 0 && kWaves % 2 == 0 && kLds * kPerUnit <= 160 * 1024, "");
    static_assert(kRing >= 2 && (kRing - 1) * kLoads <= 63, "a count of loads that s_waitcnt can name");
};

template <typename T, typename S>
__global__ __launch_bounds__(S::kThreads, S::kThreads / 256 * S::kPerUnit) void gemm_panel_kernel(const Args<T> a, const Tiles tiles, uint32_t ngroups) {
    constexpr int BA = S::BA, BW = S::BW;
    __shared__ __attribute__((aligned(16))) uint8_t lds[S::kLds];
    const uint32_t tid = threadIdx.x;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / S::WN, wn = wave % S::WN;
    const uint32_t lds_base = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t *)lds);
    uint8_t *const stage = lds + S::kRing * S::kGroup + wave * S::kStage;
    const uint32_t K = (uint32_t)a.K, lda = (uint32_t)a.lda, ldw = (uint32_t)a.ldw, last_m = (uint32_t)(a.M - 1), last_n = (uint32_t)(a.N - 1);
    // (address arithmetic that the compiler would work out once before the loops ends up spilled)
    auto opaque = [](uint32_t x) __attribute__((always_inline)) {
        asm volatile("" : "+v"(x));
        return x;
    };

    // ---- loads.  The cursor (tile p_vb, group p_G) runs kRing groups ahead.  The waves have 8 rows each in turn.  Pieces: a load brings 8 rows, lane l lands
    // in piece l mod 8 of row l / 8 and fetches piece (l mod 8) xor (row / 2 mod 8).  Words: a load brings 2 rows, lane l lands in word l mod 32 of row l / 32.
    const uint32_t n_mine = (tiles.total - blockIdx.x + gridDim.x - 1u) / gridDim.x;
    constexpr int kPart = S::kPart;
    uint32_t p_vb = blockIdx.x, p_G = 0, p_item = 0, p_k[kPart];
    uint32_t off_a[S::kLoadsA], off_w[S::kLoadsW];
    auto p_locate = [&]() __attribute__((always_inline)) {
        uint32_t tm, tn;
        tile_of_block(p_vb, tiles, tm, tn);
        const uint32_t lane = opaque(tid) & 63u, row = 8u * wave + (S::kWords ? lane >> 5 : lane >> 3);
        auto row_of = [&](int i) { return row + (uint32_t)(8 * S::kWaves * (i / kPart) + 2 * (i % kPart)); };
#pragma unroll
        for (int i = 0; i < S::kLoadsA; ++i) off_a[i] = min(tm * (uint32_t)S::kRowsA + row_of(i), last_m) * lda;
#pragma unroll
        for (int i = 0; i < S::kLoadsW; ++i) off_w[i] = min(tn * (uint32_t)S::kRowsW + row_of(i), last_n) * ldw;
    };
    auto p_piece = [&]() __attribute__((always_inline)) {
        const uint32_t t = opaque(tid);
#pragma unroll
        for (int j = 0; j < kPart; ++j) {
            // (row / 2 mod 8: of rows t / 8 and, words, 8 wave + 2 j + ..; more by multiples of 16)
            const uint32_t in = S::kWords ? (((((t & 31u) >> 2) ^ ((4u * wave + j) & 7u)) << 4) | ((t & 3u) << 2)) : (((t & 7u) ^ ((t >> 4) & 7u)) << 4);
            const uint32_t k = p_G * (uint32_t)kRow + in;
            p_k[j] = k < K ? k : 0u;  // beyond the rows: their beginning
        }
    };
    auto p_advance = [&]() __attribute__((always_inline)) {
        ++p_G;
        if (p_G == ngroups) {
            asm volatile("" ::: "memory");  // keeps the branch a branch
            p_G = 0;
            ++p_item;
            if (p_item < n_mine) p_vb = blockIdx.x + p_item * gridDim.x;  // (after the last tile the loads are repeated and never used)
            p_locate();
        }
        p_piece();
    };
    auto load_to_lds = [](const void *base, uint32_t voff, uint32_t vadd, uint32_t lds_addr) __attribute__((always_inline)) {
        uint32_t tmp;
        if constexpr (S::kWords)
            asm volatile("s_mov_b32 m0, %1\n\tv_add_u32 %0, %2, %3\n\tglobal_load_lds_dword %0, %4"
                         : "=&v"(tmp)
                         : "s"(lds_addr), "v"(voff), "v"(vadd), "s"(base)
                         : "memory");
        else
            asm volatile("s_mov_b32 m0, %1\n\tv_add_u32 %0, %2, %3\n\tglobal_load_lds_dwordx4 %0, %4"
                         : "=&v"(tmp)
                         : "s"(lds_addr), "v"(voff), "v"(vadd), "s"(base)
                         : "memory");
    };
    constexpr int kLoads = S::kLoads;
    auto load = [&](const int i, const uint32_t buf) __attribute__((always_inline)) {
        const uint32_t dst = lds_base + buf + wave * (8u * kRow);
        auto at = [](int i) { return (uint32_t)(i / kPart * 8 * S::kWaves * kRow + i % kPart * 2 * kRow); };
        if (i < S::kLoadsA)
            load_to_lds(a.A, off_a[i < S::kLoadsA ? i : 0], p_k[i % kPart], dst + at(i));
        else
            load_to_lds(a.W, off_w[i < S::kLoadsA ? 0 : i - S::kLoadsA], p_k[i % kPart], dst + (uint32_t)(S::kRowsA * kRow) + at(i - S::kLoadsA));
    };

    // ---- products: blocks of 16 x 16, 64 codes at a time (step 0, 1 of a group)
    constexpr int NX = 2 * BA, NW = 2 * BW;
    v4i x[NX], w[2][NW];
    v4i acc[NW][NX];
    auto place = [&](const int s, const uint32_t buf) __attribute__((always_inline)) {
        const uint32_t lane = opaque(tid) & 63u, r = lane & 15u, g = lane >> 4;
        return buf + r * (uint32_t)kRow + ((((uint32_t)(4 * s) + g) ^ ((r >> 1) & 7u)) << 4);
    };
    auto fetch_w = [&](const int i, const uint32_t at, v4i (&to)[NW]) __attribute__((always_inline)) {
        to[i] = *reinterpret_cast<const v4i *>(lds + at + (S::kRowsA + wn * 32u * BW) * kRow + 16 * i * kRow);
    };
    auto fetch_x = [&](const int i, const uint32_t at) __attribute__((always_inline)) {
        x[i] = *reinterpret_cast<const v4i *>(lds + at + wm * 32u * BA * kRow + 16 * i * kRow);
    };
    constexpr int kHold = NX >= 4 ? 2 : 1;  // rows of codes multiplied before the barrier, whose operands are on their way
    auto multiply = [&](const int j, v4i (&now)[NW]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NW; ++i) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(now[i], x[j], acc[i][j], 0, 0, 0);
    };
    auto clear_beyond = [&](v4i (&f)[NW], const uint32_t k_end, const int s) __attribute__((always_inline)) {
        const uint32_t k = k_end - (uint32_t)kRow + 64u * s + 16u * ((opaque(tid) & 63u) >> 4);
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            if constexpr (S::kWords) {
#pragma unroll
                for (int e = 0; e < 4; ++e) f[i][e] = k + 4u * e < K ? f[i][e] : 0;
            } else {
                if (k >= K) f[i] = v4i{0, 0, 0, 0};
            }
        }
    };

    // ---- a tile's way out: 32 rows x 128 bytes at a time through the wave's part of LDS, rows of 128 bytes leave as they are
    auto finish = [&](const uint32_t tm, const uint32_t tn) __attribute__((always_inline)) {
        constexpr int kPer = 32 * BW * (int)sizeof(T) < 128 ? BW : 128 / (int)sizeof(T) / 32;  // blocks of 32 columns that leave together
        constexpr int kLine = kPer * 32 * (int)sizeof(T), kUnit = 16 / (int)sizeof(T), kUnits = kLine / 16;  // 128 bytes (64) in 16-byte units
        const uint32_t lane = opaque(tid) & 63u, r = lane & 15u, g = lane >> 4;
        const int64_t m0 = (int64_t)tm * S::kRowsA + wm * 32u * BA, n0 = (int64_t)tn * S::kRowsW + wn * 32u * BW;
        float sa[NX];
#pragma unroll
        for (int j = 0; j < NX; ++j) sa[j] = a.scaleA[min(m0 + 16 * j + r, a.M - 1)];
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const int32_t n = (int32_t)(n0 + 16 * i) + 4 * (int32_t)g;
            float sw[4], bias[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t at = min((uint32_t)(n + e), last_n);
                sw[e] = a.scaleW[at];
                bias[e] = a.bias ? a.bias[at] : 0.0f;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < NX; ++j) acc[i][j][e] = __float_as_int((float)acc[i][j][e] * sa[j] * sw[e] + bias[e]);
            __builtin_amdgcn_sched_barrier(0);  // (all these loads at once would take the registers of the sums)
        }
#pragma unroll
        for (int i0 = 0; i0 < BW; i0 += kPer) {
#pragma unroll
            for (int j = 0; j < BA; ++j) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 2 * kPer; ++i) {
                        struct Four {
                            T e[4];
                        } four;
#pragma unroll
                        for (int e = 0; e < 4; ++e) four.e[e] = (T)__int_as_float(acc[2 * i0 + i][2 * j + h][e]);
                        // values 16 i + 4 g .. + 3 of a row, in units swizzled with the row
                        const uint32_t at = (uint32_t)(16 * i) + 4u * g, unit = at / kUnit, in = at % kUnit, row = 16u * h + r;
                        __builtin_memcpy(__builtin_assume_aligned(stage + row * kLine + ((unit ^ (row & (kUnits - 1u))) << 4) + in * sizeof(T), 4 * sizeof(T)),
                                         &four, sizeof four);
                    }
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                const int64_t n = n0 + 32 * i0 + kUnit * (int64_t)(lane % kUnits), here = a.N - n;
#pragma unroll
                for (int q = 0; q < kUnits / 2; ++q) {
                    const uint32_t row = (64u / kUnits) * q + lane / kUnits;
                    const v4i line = *reinterpret_cast<const v4i *>(stage + row * kLine + (((lane ^ row) & (kUnits - 1u)) << 4));
                    const int64_t m = m0 + 32 * j + row;
                    if (m < a.M && here > 0) {
                        T *const to = a.out + m * a.ldo + n;
                        if (here >= kUnit) {
                            __builtin_memcpy(to, &line, 16);
                        } else {
                            T e[kUnit];
                            __builtin_memcpy(e, &line, 16);
#pragma unroll
                            for (int x = 0; x < kUnit; ++x)
                                if (x < here) to[x] = e[x];
                        }
                    }
                }
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            }
        }
    };

    p_locate();
    p_piece();
#pragma unroll
    for (int q = 0; q < S::kRing; ++q) {
        if (q > 0) p_advance();
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load(i, (uint32_t)(q * S::kGroup));
    }
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((S::kRing - 1) * kLoads) : "memory");

    uint32_t rd = 0u;
    {
        const uint32_t at = place(0, 0u);
#pragma unroll
        for (int i = 0; i < NW; ++i) fetch_w(i, at, w[0]);
#pragma unroll
        for (int i = 0; i < NX; ++i) fetch_x(i, at);
    }
    for (uint32_t item = 0; item < n_mine; ++item) {
#pragma unroll
        for (int i = 0; i < NW; ++i)
#pragma unroll
            for (int j = 0; j < NX; ++j) acc[i][j] = v4i{0, 0, 0, 0};
        for (uint32_t G = 0; G < ngroups; ++G) {
            const uint32_t other = rd == (uint32_t)((S::kRing - 1) * S::kGroup) ? 0u : rd + (uint32_t)S::kGroup;
            uint32_t k_end = (G + 1u) * (uint32_t)kRow;
            asm volatile("" : "+s"(k_end));
            const bool beyond = k_end > K;
            p_advance();
            if (beyond) clear_beyond(w[0], k_end, 0);
            {
                const uint32_t at = place(1, rd);
#pragma unroll
                for (int j = 0; j < NX; ++j) {
#pragma unroll
                    for (int i = 0; i < NW; ++i)
                        if (i * NX / NW == j) fetch_w(i, at, w[1]);
                    multiply(j, w[0]);
                    fetch_x(j, at);
                }
            }
            if (beyond) clear_beyond(w[1], k_end, 1);
            {
                const uint32_t at = place(0, other);
#pragma unroll
                for (int j = 0; j < kHold; ++j) multiply(j, w[1]);
                // The next group has landed (kRing - 2 groups' loads were sent after it, and perhaps a tile's stores), and every wave holds its last
                // operands of this one: the buffer is free.
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((S::kRing - 2) * kLoads) : "memory");
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = kHold; j < NX; ++j) {
#pragma unroll
                    for (int i = 0; i < kLoads; ++i)
                        if (kHold + i * (NX - kHold) / kLoads == j) load(i, rd);
#pragma unroll
                    for (int i = 0; i < NW; ++i)
                        if (kHold + i * (NX - kHold) / NW == j) fetch_w(i, at, w[0]);
                    if (j - kHold < kHold) fetch_x(j - kHold, at);
                    multiply(j, w[1]);
                    fetch_x(j, at);
                }
            }
            rd = other;
        }
#pragma unroll
        for (int i = 0; i < NW; ++i)
#pragma unroll
            for (int j = 0; j < NX; ++j) asm volatile("" : "+v"(acc[i][j]));
        uint32_t tm, tn;
        tile_of_block(blockIdx.x + item * gridDim.x, tiles, tm, tn);
        finish(tm, tn);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (the loads beyond the last tile)
}

typedef Shape<2, 4, 4, 2, 2, 1> Large;  // 256 x 256
typedef Shape<2, 2, 2, 2, 2, 2> Small;  // 128 x 128, two workgroups on a compute unit
typedef Shape<2, 4, 2, 1, 4, 1> Eight;  // 128 x 128 on eight waves
typedef Shape<2, 2, 1, 1, 4, 2> Tiny;   // 64 x 64
// the same for words (a line of 256 bytes a load: slower by half, but 4000 x 4000 x 4004 104 us through registers, 69 like this; the largest spills 7 to 9 registers in the
// way out, none in the loop over k)
typedef Shape<2, 4, 4, 2, 2, 1, true> LargeWords;
typedef Shape<2, 2, 2, 2, 2, 2, true> SmallWords;
typedef Shape<2, 2, 1, 1, 4, 2, true> TinyWords;

}  // namespace panel
}  // namespace int8
}  // namespace qnn
