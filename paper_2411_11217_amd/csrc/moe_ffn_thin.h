// a3 for a handful of tokens, on the matrix cores (moe_ffn_op.h: bf16 operands with fp32 sums, or 8-bit integers with scales).  Few experts have rows then, and
// a block of moe_ffn_rows.h with its 64 or 128 columns leaves compute units without weights to stream (one token of
// the Mixtral-8x7B shape: 64 blocks in the down launch, 82 us for 235 MB).
//
// Here a wavefront is on its own: 16 columns (MODE 0: 16 features, gate and up), one row tile, no LDS and no barrier.  Its weights
// (1 KiB in a row per half-tile, one MFMA operand) and its activations (16 rows x 64 bytes, from the L2 after the first
// wavefront) go straight into registers, D k-steps ahead, all loads the compiler's own and in one order.  With at most 16 tokens an
// expert has at most 16 rows (others, from offsets that no routing made, take several row tiles).  us for the launch, D = 8 / 12 / 16:
// down of the Mixtral-8x7B shape, one token 45 / 46 / 45 (rows kernel 82), two tokens 74 / 79 / - (96); four wavefronts to a block
// instead of one 55.  Every output is the same chain of MFMAs along k as in the other kernels: the same bits.
#pragma once

#include <type_traits>

#include "moe_ffn_common.h"
#include "moe_ffn_op.h"

namespace moe {
namespace {


// CW: wavefronts of a block, side by side along the columns
template <class Op, int MODE, int CW>
__global__ __launch_bounds__(64 * CW) void ffn_thin(const GemmParams p) {
    constexpr int D = 8;                             // k-steps under way
    constexpr int BM = 16, NB = MODE == 0 ? 2 : 1, kCols = 16 * CW, kColTiles = 128 / kCols;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;

    RowsTile tc;
    if (!locate_rows_tile<BM>(p, tc)) return;
    const int nt = tc.nt, row0 = tc.row0, rows_here = tc.rows_here, KT = p.KT;
    const int32_t* trow = p.table + (size_t)(p.table_row_mod ? tc.e % p.table_row_mod : tc.e) * p.ppe + p.group_base;
    int bad = 0, page[NB], within[NB];
    const char* tile[NB];
    auto page_addr = [&](int pg) __attribute__((always_inline)) -> const char* {
        int slot = __builtin_amdgcn_readfirstlane(trow[pg]);
        if ((unsigned)slot >= (unsigned)p.pool_pages) {   // never follow an entry outside the pool
            bad = 1;
            slot = 0;
        }
        return p.pool + (int64_t)slot * p.page_bytes;
    };
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int t0 = ((nt / kColTiles) * NB + b) * KT;
        page[b] = t0 / p.tpp;
        within[b] = t0 - page[b] * p.tpp;
        tile[b] = page_addr(page[b]) + (int64_t)within[b] * kTileBytes;
    }
    const uint32_t b_off = ((nt % kColTiles) * kCols + wave * 16 + r) * 64 + ((g ^ ((r >> 2) & 2)) << 4);
    const int row = min(r, rows_here - 1);
    const int src = p.a_gather ? min(max(p.a_gather[row0 + row] / p.a_div, 0), p.a_rows - 1) : row;
    const uint32_t a_off = (uint32_t)src * (uint32_t)p.lda_bytes + g * 16;
    const char* a_base = p.a_gather ? p.A : p.A + (int64_t)row0 * p.lda_bytes;

    // scales: of row r (lane r, handed round at the end), and of column nt * kCols + wave * 16 + r of each matrix
    float row_scale = 0.f, col_scale[NB];
    if constexpr (Op::kScaled) {
        row_scale = p.a_scale[p.a_gather ? src : row0 + row];
        if (MODE == 1 && p.row_w) row_scale *= p.row_w[row0 + row];
#pragma unroll
        for (int b = 0; b < NB; ++b) col_scale[b] = (b ? p.w_scale_up : p.w_scale)[(int64_t)tc.e * p.n_cols + nt * kCols + wave * 16 + r];
    }

    typename Op::Acc acc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b] = typename Op::Acc{0, 0, 0, 0};
    auto main_loop = [&](auto stream_c) __attribute__((always_inline)) {
        i32x4 areg[D][2], breg[D][2][NB];
        auto load = [&](int s, int slot) __attribute__((always_inline)) {        // k-step s, s in order
#pragma unroll
            for (int hp = 0; hp < 2; ++hp) {
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const i32x4* src = (const i32x4*)(tile[b] + hp * kHalfTileBytes + b_off);
                    if constexpr (decltype(stream_c)::value) breg[slot][hp][b] = __builtin_nontemporal_load(src);
                    else breg[slot][hp][b] = *src;
                }
                areg[slot][hp] = *(const i32x4*)(a_base + (int64_t)s * 128 + hp * 64 + a_off);
            }
            if (s + 1 < KT) {
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    tile[b] += kTileBytes;
                    if (__builtin_expect(++within[b] == p.tpp, 0)) {
                        within[b] = 0;
                        tile[b] = page_addr(++page[b]);
                    }
                }
            }
        };
        auto multiply = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
            for (int hp = 0; hp < 2; ++hp)
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    acc[b] = Op::mfma(areg[slot][hp], breg[slot][hp][b], acc[b]);
        };
#pragma unroll
        for (int u = 0; u < D; ++u)
            if (u < KT) load(u, u);
        int s = 0;
        for (; s + 2 * D <= KT; s += D)
#pragma unroll
            for (int u = 0; u < D; ++u) {
                multiply(u);
                load(s + u + D, u);
            }
        // fewer than 2 D k-steps are left, the next D of them loaded
#pragma unroll
        for (int u = 0; u < D; ++u)
            if (s + u < KT) {
                multiply(u);
                if (s + u + D < KT) load(s + u + D, u);
            }
#pragma unroll
        for (int u = 0; u < D; ++u)
            if (s + u + D < KT) multiply(u);
    };
    if (p.stream && tc.mtiles == 1) main_loop(std::true_type{});
    else main_loop(std::false_type{});

    const int col = nt * kCols + wave * 16 + r;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int orow = g * 4 + v;
        if constexpr (Op::kScaled) {
            const float s = __shfl(row_scale, orow, 64);
            if (orow >= rows_here) continue;
            const int64_t o = (int64_t)(row0 + orow) * p.ldo + col;
            if constexpr (MODE == 0) ((__bf16*)p.out)[o] = (__bf16)silu_mul_i8(acc[0][v], acc[NB - 1][v], col_scale[0] * kGateFactor, col_scale[NB - 1] * kUpFactor, s);
            else ((typename Op::Out*)p.out)[o] = (typename Op::Out)((float)acc[0][v] * col_scale[0] * s);
            continue;
        }
        if (orow >= rows_here) continue;
        const int64_t o = (int64_t)(row0 + orow) * p.ldo + col;
        if constexpr (MODE == 0) ((__bf16*)p.out)[o] = (__bf16)silu_mul_bf16(acc[0][v], acc[1][v]);
        else ((float*)p.out)[o] = acc[0][v] * (p.row_w ? p.row_w[row0 + orow] : 1.0f);
    }
    if (bad && lane == 0 && p.status) atomicOr(p.status, 1);
}

template <class Op, int MODE, int CW>
int launch_thin(GemmParams& p, int cols, int R, int n_exp, hipStream_t st) {
    p.NT = cols / (16 * CW);
    hipLaunchKernelGGL((ffn_thin<Op, MODE, CW>), dim3(rows_grid(p.NT, R, 16, n_exp)), dim3(64 * CW), 0, st, p);
    MOE_HIP_TRY(hipGetLastError());
    return MOE_OK;
}

}  // namespace
}  // namespace moe
