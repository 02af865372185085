// a3 and the dense linear map for launches with few rows per expert, on the matrix cores (moe_ffn_op.h: bf16 operands with fp32 sums,
// or 8-bit integers with scales).  The launch is bound by reading every weight once, and what counts is how many bytes are under
// way and how short a block's way to its first load is.
//
// A block owns a row tile (16 * RT rows) x 16 * CW * FC columns (MODE 0: features, gate and up).  The CW wavefronts split the
// columns; a wavefront's 16 weight rows of a half-tile are 1 KiB in a row in the page, exactly one 16-byte load per lane and
// exactly its MFMA operand, so the weights go from the page straight into registers, D k-steps ahead (p.stream: with the
// non-temporal hint).  The activations, which all wavefronts share, are loaded as far ahead into registers and pass through a
// double-buffered LDS stage (one k-step, 128-byte rows, the chunk swizzle of moe_ffn_gemm.h), one barrier per k-step.
// All loads are the compiler's own, in one order, so its counted waits keep D - 1 k-steps under way across the barriers.
// Rows beyond the tile's last pair of 16-row MFMA tiles are neither loaded nor multiplied (a copy of the loop per pair:
// branches inside it would put an LDS latency in front of every MFMA).  Few registers and little LDS: two or more blocks share
// a compute unit and cover each other's start and end.
//
// FC = 1 in the linear map: a block's groups of 16 columns need not be a page tile's, every wavefront walks the tile of its own.
// RG > 1 (linear map): RG groups of CW wavefronts share the columns and split the row tiles.  Every output is the same chain of
// MFMAs along k as in moe_ffn_gemm.h: the same bits.
#pragma once

#include "moe_ffn_common.h"
#include "moe_ffn_op.h"

namespace moe {
namespace {

constexpr int kComputeUnits = 256;                   // MI355X

template <int N>
struct Num {
    static constexpr int value = N;
};

// FC: fragments of 16 columns per wavefront (MODE 0: of 16 features, gate and up)
// KG (the linear map of integers; for the experts' down launch two teams won nothing): KG teams of CW * RG wavefronts, each with a part of k; their whole numbers are added up at the end, which is exact in any order.
template <class Op, int MODE, int RT, int CW, int FC, int RG, int D, int KG = 1>
__global__ __launch_bounds__(64 * CW * RG * KG) void ffn_rows(const GemmParams p) {
    constexpr int BM = 16 * RT, NB = MODE == 0 ? 2 * FC : FC, kCols = 16 * CW * FC;
    constexpr int kPass = 8 * CW * RG;               // rows that one load instruction per thread fetches
    constexpr int AJ = (BM + kPass - 1) / kPass, kStage = AJ * kPass * 128;
    static_assert(RT % 2 == 0 && RT <= 8 && (128 % kCols == 0 || FC == 1) && (kPass <= BM || RG == 1 || kPass >= 16 * RG), "");
    constexpr int kOutRow = kCols * 2 + 16;          // MODE 0: bytes of a row of h in LDS, 16 of padding
    constexpr int kTeam = CW * RG, kPartial = kTeam * ((RT + RG - 1) / RG) * NB * 1024;      // wavefronts of a team, bytes of its sums
    constexpr int kSmem = MODE == 0 && BM * kOutRow > 2 * kStage ? BM * kOutRow : KG * 2 * kStage;
    static_assert(MODE == 1 || RG == 1, "the row groups are the linear map's");
    static_assert(KG == 1 || (MODE == 1 && Op::kScaled && (KG - 1) * kPartial <= kSmem), "teams add up whole numbers");
    __shared__ __attribute__((aligned(1024))) char smem[kSmem];
    __shared__ float row_scales[Op::kScaled ? BM : 1];
    const int lane = threadIdx.x & 63;
    const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kg = KG == 1 ? 0 : wave_all / kTeam, wave = KG == 1 ? wave_all : wave_all % kTeam;
    const int tid = KG == 1 ? threadIdx.x : wave * 64 + lane;        // in the team
    const int cw = RG == 1 ? wave : wave % CW, rg = RG == 1 ? 0 : wave / CW;
    const int r = lane & 15, g = lane >> 4;

    RowsTile tc;
    if (!locate_rows_tile<BM>(p, tc)) return;
    // diagnostic: some blocks report the shader clock they saw, as in moe_ffn_gemm.h
    const bool clock_probe = p.status && (blockIdx.x & 511) == 256 && threadIdx.x == 0;
    long long probe_c = 0, probe_w = 0;
    if (clock_probe) {
        probe_c = clock64();
        probe_w = wall_clock64();
    }
    const int nt = tc.nt, row0 = tc.row0, rows_here = tc.rows_here;
    const int32_t* trow = p.table + (size_t)(p.table_row_mod ? tc.e % p.table_row_mod : tc.e) * p.ppe + p.group_base;

    // activations: 16 bytes of rows tid / 8 + kPass * j
    uint32_t a_off[AJ];
#pragma unroll
    for (int j = 0; j < AJ; ++j) {
        const int row = min(j * kPass + (tid >> 3), rows_here - 1);
        const int src = p.a_gather ? min(max(p.a_gather[row0 + row] / p.a_div, 0), p.a_rows - 1) : row;
        a_off[j] = (uint32_t)src * (uint32_t)p.lda_bytes + (tid & 7) * 16;
    }
    // the team's k-steps; every team takes as many turns of the loop as the longest
    const int k0 = KG == 1 ? 0 : p.KT * kg / KG, KT = KG == 1 ? p.KT : p.KT * (kg + 1) / KG - k0, turns = KG == 1 ? p.KT : (p.KT + KG - 1) / KG;
    const char* a_base = (p.a_gather ? p.A : p.A + (int64_t)row0 * p.lda_bytes) + (KG == 1 ? 0 : k0 * 128);
    const int a_wr0 = (tid >> 3) * 128 + (((tid & 7) ^ ((tid >> 4) & 7)) << 4);
    auto a_wr = [&](int j) __attribute__((always_inline)) { return (kPass % 16 ? a_wr0 ^ ((j & 1) << 6) : a_wr0) + j * kPass * 128; };     // kPass / 2 is 4 modulo 8 or 0
    const int a_rd[2] = {r * 128 + ((g ^ ((r >> 1) & 7)) << 4), r * 128 + (((4 + g) ^ ((r >> 1) & 7)) << 4)};

    // weights: one page tile is walked along k, MODE 0 two (the W1 and the W3 tile of the same features)
    int bad = 0, page, within, page1 = 0, within1 = 0;
    const char* tile[MODE == 0 ? 2 : 1];
    auto page_addr = [&](int pg) __attribute__((always_inline)) -> const char* {
        int slot = __builtin_amdgcn_readfirstlane(trow[pg]);
        if ((unsigned)slot >= (unsigned)p.pool_pages) {   // never follow an entry outside the pool
            bad = 1;
            slot = 0;
        }
        return p.pool + (int64_t)slot * p.page_bytes;
    };
    // MODE 1 with FC = 1, and columns that are no part of a page tile: each wavefront has the page tile of its own 16 columns (a block may begin in one and end in the next)
    constexpr bool kOwn = FC == 1 && (MODE == 1 || 128 % kCols != 0);
    constexpr int kColTiles = kOwn ? 1 : 128 / kCols;     // blocks per page tile along the columns
    const int group = kOwn ? min(nt * CW + cw, p.n_cols / 16 - 1) : 0;       // the last block may have wavefronts too many
    {
        const int t0 = (kOwn ? (group >> 3) * (MODE == 0 ? 2 : 1) * p.KT : (nt / kColTiles) * (MODE == 0 ? 2 : 1) * p.KT) + k0;
        page = t0 / p.tpp;
        within = t0 - page * p.tpp;
        tile[0] = page_addr(page) + (int64_t)within * kTileBytes;
        if (MODE == 0) {
            page1 = (t0 + p.KT) / p.tpp;
            within1 = t0 + p.KT - page1 * p.tpp;
            tile[MODE == 0] = page_addr(page1) + (int64_t)within1 * kTileBytes;
        }
    }
    auto advance = [&]() __attribute__((always_inline)) {
        tile[0] += kTileBytes;
        if (++within == p.tpp) {
            within = 0;
            tile[0] = page_addr(++page);
        }
        if (MODE == 0) {
            tile[MODE == 0] += kTileBytes;
            if (++within1 == p.tpp) {
                within1 = 0;
                tile[MODE == 0] = page_addr(++page1);
            }
        }
    };
    const uint32_t b_off = ((kOwn ? (group & 7) * 16 : (nt % kColTiles) * kCols + cw * 16 * FC) + r) * 64 + ((g ^ ((r >> 2) & 2)) << 4);

    // the scales of the block's rows, one per thread, and of the wavefront's columns: on their way before the operands, wanted after them
    float row_scale = 0.f, col_scale[NB];
    if constexpr (Op::kScaled) {
        static_assert(BM <= 64 * CW * RG, "a row to a thread");
        if (tid < BM) {
            const int row = min(tid, rows_here - 1);
            const int64_t src = p.a_gather ? min(max(p.a_gather[row0 + row] / p.a_div, 0), p.a_rows - 1) : row0 + row;
            row_scale = p.a_scale[src];
            if (MODE == 1 && p.row_w) row_scale *= p.row_w[row0 + row];
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int c = min(nt * kCols + cw * 16 * FC + (b % FC) * 16 + r, p.n_cols - 1);
            col_scale[b] = (MODE == 0 && b >= FC ? p.w_scale_up : p.w_scale)[(int64_t)tc.e * p.n_cols + c];
        }
    }

    // row group rg: row tiles rg * (NRT / RG) ..
    constexpr int TPW = (RT + RG - 1) / RG;
    typename Op::Acc acc[TPW][NB];
#pragma unroll
    for (int i = 0; i < TPW; ++i)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[i][b] = typename Op::Acc{0, 0, 0, 0};
    int tile0 = 0, tiles_mine = TPW;                 // this wavefront's first row tile and their number

    // the loop for NRT row tiles: rows beyond them are neither loaded nor multiplied
    auto main_loop = [&](auto stream_c, auto nrt_c) __attribute__((always_inline)) {
        constexpr bool STREAM = decltype(stream_c)::value;
        constexpr int NRT = decltype(nrt_c)::value, NA = (16 * NRT + kPass - 1) / kPass, NT = (NRT + RG - 1) / RG;
        static_assert(RG * NT * 16 <= AJ * kPass, "every row tile that is multiplied lies inside the stage");
        tile0 = rg * NT;
        tiles_mine = NT;
        // Integers, blocks of few columns: rows that the tile does not have are zeros instead of its last row again (us, in a graph: 4096 x 6144 1 row 8.7 / 7.9, 36: 10.8 / 10.1; blocks
        // of 64 columns, 100 rows 12.9 / 13.2, which are left as they were).
        constexpr bool kSkip = Op::kScaled && (RG > 1 || BM == 32);
        i32x4 areg[D][NA], breg[D][2][NB];
        if constexpr (kSkip)
#pragma unroll
            for (int u = 0; u < D; ++u)
#pragma unroll
                for (int j = 0; j < NA; ++j) areg[u][j] = i32x4{0, 0, 0, 0};
        int kt_load = 0;                             // k-step that the next load_b fetches
        auto load_a = [&](int s, int slot) __attribute__((always_inline)) {
            const char* base = a_base + (int64_t)(KG == 1 ? min(s, KT - 1) : max(min(s, KT - 1), 0)) * 128;      // a team may have no step of its own
#pragma unroll
            for (int j = 0; j < NA; ++j)
                if (!kSkip || j * kPass + (tid >> 3) < rows_here) areg[slot][j] = *(const i32x4*)(base + a_off[j]);
        };
        auto load_b = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
            for (int hp = 0; hp < 2; ++hp)
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const i32x4* src = (const i32x4*)(tile[MODE == 0 ? b / FC : 0] + (MODE == 0 ? b % FC : b) * 1024 + hp * kHalfTileBytes + b_off);
                    if constexpr (STREAM) breg[slot][hp][b] = __builtin_nontemporal_load(src);
                    else breg[slot][hp][b] = *src;
                }
            if (++kt_load < KT) advance();
        };
        int buf = 0;
        auto step = [&](int s, int slot, bool more) __attribute__((always_inline)) {     // slot: known at compile time
            char* st = smem + (KG == 1 ? 0 : kg * 2 * kStage) + buf;
#pragma unroll
            for (int j = 0; j < NA; ++j) *(i32x4*)(st + a_wr(j)) = areg[slot][j];
            __syncthreads();
            if (more) load_a(s + D, slot);
            i32x4 a[2][NT];
#pragma unroll
            for (int hp = 0; hp < 2; ++hp)
#pragma unroll
                for (int i = 0; i < NT; ++i) a[hp][i] = *(const i32x4*)(st + a_rd[hp] + (tile0 + i) * 2048);
#pragma unroll
            for (int hp = 0; hp < 2; ++hp)
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int b = 0; b < NB; ++b)
                        if (KG == 1 || s < KT) acc[i][b] = Op::mfma(a[hp][i], breg[slot][hp][b], acc[i][b]);
            if (more) load_b(slot);
            buf ^= kStage;
        };
#pragma unroll
        for (int u = 0; u < D; ++u) {
            load_a(u, u);
            load_b(u);
        }
        int s = 0;
        for (; s + 2 * D <= turns; s += D)
#pragma unroll
            for (int u = 0; u < D; ++u) step(s + u, u, true);
#pragma unroll
        for (int u = 0; u < 2 * D - 1; ++u)
            if (s + u < turns) step(s + u, u % D, s + u + D < turns);
    };
    auto run = [&](auto stream_c) __attribute__((always_inline)) {
        if (RT > 6 && rows_here > 96) main_loop(stream_c, Num<RT>{});
        else if (RT > 4 && rows_here > 64) main_loop(stream_c, Num<RT < 6 ? RT : 6>{});
        else if (RT > 2 && rows_here > 32) main_loop(stream_c, Num<RT < 4 ? RT : 4>{});
        else main_loop(stream_c, Num<2>{});
    };
    if (RG == 1 && p.stream && tc.mtiles == 1) run(Num<RG == 1>{});        // RG > 1: the linear map, never streamed
    else run(Num<0>{});

    if constexpr (Op::kScaled) {
        if (KG > 1) __syncthreads();                 // everyone has read the last stages
        if (kg == 0 && tid < BM) row_scales[tid] = row_scale;
        if constexpr (KG > 1) {
            i32x4* const part = (i32x4*)(smem + (kg - 1) * kPartial) + wave * TPW * NB * 64 + lane;
            if (kg > 0)
#pragma unroll
                for (int i = 0; i < TPW; ++i)
#pragma unroll
                    for (int b = 0; b < NB; ++b) part[(i * NB + b) * 64] = acc[i][b];
        }
        if (MODE == 1) __syncthreads();
        if constexpr (KG > 1) {
            if (kg == 0)
#pragma unroll
                for (int o = 0; o < KG - 1; ++o)
#pragma unroll
                    for (int i = 0; i < TPW; ++i)
#pragma unroll
                        for (int b = 0; b < NB; ++b) acc[i][b] += ((const i32x4*)(smem + o * kPartial))[(wave * TPW * NB + i * NB + b) * 64 + lane];
        }
    }

    if constexpr (MODE == 0) {
        // h leaves through LDS in whole lines, 16 bytes a lane, in part past the L2 (see kStreamRows)
        __syncthreads();                             // everyone has read the last stage
#pragma unroll
        for (int i = 0; i < TPW; ++i)
            if (i * 16 < rows_here)
#pragma unroll
                for (int v = 0; v < 4; ++v)
#pragma unroll
                    for (int f = 0; f < FC; ++f) {
                        const int row = i * 16 + g * 4 + v;
                        float y;
                        if constexpr (Op::kScaled) y = silu_mul_i8(acc[i][f][v], acc[i][NB - FC + f][v], col_scale[f] * kGateFactor, col_scale[NB - FC + f] * kUpFactor, row_scales[row]);
                        else y = silu_mul_bf16(acc[i][f][v], acc[i][NB - FC + f][v]);
                        *(__bf16*)(smem + row * kOutRow + (cw * 16 * FC + f * 16 + r) * 2) = (__bf16)y;
                    }
        __syncthreads();
        constexpr int kChunks = kCols / 8;           // 16-byte chunks of a row
        char* o = (char*)p.out + ((int64_t)row0 * p.ldo + nt * kCols) * 2;
        auto store_rows = [&](auto past_l2) __attribute__((always_inline)) {
            for (int c = tid; c < rows_here * kChunks; c += 64 * CW * RG) {
                const int row = c / kChunks, ch = c % kChunks;
                if (kOwn && nt * kCols + ch * 8 >= p.n_cols) continue;       // of a wavefront too many
                const i32x4 hv = *(const i32x4*)(smem + row * kOutRow + ch * 16);
                i32x4* dst = (i32x4*)(o + (int64_t)row * p.ldo * 2 + ch * 16);
                if constexpr (decltype(past_l2)::value) {
                    __builtin_nontemporal_store(hv, dst);
                    asm volatile("" ::: "memory");       // else the compiler makes one store of this one and the plain one
                } else {
                    *dst = hv;
                }
            }
        };
        if (p.stream > 1 || (p.stream && tc.mtiles == 1)) store_rows(Num<1>{});
        else store_rows(Num<0>{});
    } else {
        const int col = nt * kCols + cw * 16 * FC + r;
        const bool mine = !kOwn || group == nt * CW + cw;
#pragma unroll
        for (int i = 0; i < TPW; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int row = (tile0 + i) * 16 + g * 4 + v;
                if (row >= rows_here || !mine || (RG > 1 && i >= tiles_mine) || (KG > 1 && kg > 0)) continue;
                const int64_t o = (int64_t)(row0 + row) * p.ldo + col;
                if constexpr (Op::kScaled) {
#pragma unroll
                    for (int f = 0; f < FC; ++f) ((typename Op::Out*)p.out)[o + f * 16] = (typename Op::Out)((float)acc[i][f][v] * col_scale[f] * row_scales[row]);
                } else {
                    const float wgt = p.row_w ? p.row_w[row0 + row] : 1.0f;
#pragma unroll
                    for (int f = 0; f < FC; ++f) {
                        const float y = acc[i][f][v] * wgt;
                        ((float*)p.out)[o + f * 16] = y;
                        if (p.out16) p.out16[o + f * 16] = (uint16_t)f32_to_bf16_bits(y);
                    }
                }
            }
    }
    if (clock_probe) {
        const long long dc = clock64() - probe_c, dw = wall_clock64() - probe_w;
        if (dw > 0) p.status[2 + MODE] = (int32_t)(dc * 100 / dw);       // MHz
    }
    if (bad && lane == 0 && p.status) atomicOr(p.status, 1);
}

template <class Op, int MODE, int RT, int CW, int FC, int RG, int D, int KG = 1>
int launch_rows(GemmParams& p, int cols, int R, int n_exp, hipStream_t st) {
    p.NT = (cols / 16 + CW * FC - 1) / (CW * FC);
    hipLaunchKernelGGL((ffn_rows<Op, MODE, RT, CW, FC, RG, D, KG>), dim3(rows_grid(p.NT, R, 16 * RT, n_exp)), dim3(64 * CW * RG * KG), 0, st, p);
    MOE_HIP_TRY(hipGetLastError());
    return MOE_OK;
}

// Where the expert GEMMs take this kernel (rows_kernel_takes, moe_ffn_common.h): up to 80 rows per expert on average (of all experts: the launches of a streamed
// layer take what the resident layer's single launch takes).  us for the layer, moe_ffn_gemm.h's kernel / this one:
// Mixtral-8x7B shape (2 of 8 experts) 1 token 196 / 165, 4: 364 / 355, 16: 469 / 455, 64: 477 / 466, 150: 485 / 478, 256 (64
// rows each): 522 / 511, 288: 532 / 520, 400 (100 rows): 552 / 560; 64 experts of 2048 x 1024, 8 per token, 20 tokens 192 /
// 183, 400: 241 / 235, 600 (75 rows): 252 / 247, 777 (97 rows): 259 / 262; DBRX shape 120 tokens 1089 / 1036, 250: 1129 / 1096.
// What is left is the weights' way from HBM: with 4, 36 and 256 tokens of the Mixtral-8x7B shape 6.5, 6.7 and 5.8 TB/s in the
// gate/up launch, 6.2, 6.6 and 5.9 in the down launch, whatever the depth and the block.
// The average is all the host knows.  An expert with more rows than a block reads its weights once per row tile, 1.1 to 2.3 times
// over the fabric.  Skewed routing (40 % of the rows on one expert, or one expert with every token) is still 2 - 25 % faster this
// way; with every token on the same k experts two of the shapes lose, all other experts being empty: DBRX shape 80 tokens 395 /
// 439, 130: 452 / 534, 176: 470 / 563, 256: 521 / 539, 300: 674 / 649; Mixtral-8x22B shape 130 tokens 365 / 465, 200 and more: within 4 %
// (8x7B shape 130 tokens 284 / 265, 300: 382 / 320).
// Up to here 64-row blocks with half the columns; 45 .. 72 rows need two of them per expert for some experts, and the second
// one reads the weights again (176 tokens of the Mixtral-8x7B shape, 44 rows: 489 against 503 with 128-row blocks).
constexpr int kRows64Max = 44;

template <class Op>
int gate_up_rows(GemmParams& p, int F, int R, int rows_each, int n_exp, hipStream_t st) {
    if (rows_each <= kRows64Max) return launch_rows<Op, 0, 4, 4, 1, 1, 4>(p, F, R, n_exp, st);
    return launch_rows<Op, 0, 8, 8, 1, 1, 2>(p, F, R, n_exp, st);
}

template <class Op>
int down_rows(GemmParams& p, int H, int R, int rows_each, int n_exp, hipStream_t st) {
    if (rows_each <= kRows64Max) return launch_rows<Op, 1, 4, 4, 2, 1, 4>(p, H, R, n_exp, st);
    return launch_rows<Op, 1, 8, 8, 1, 1, 4>(p, H, R, n_exp, st);
}

// The dense linear map (moe_host.h: linear_takes_rows_kernel says when it comes here, linear_rows_block with which blocks).  A compute unit has some 110 lines under way; a line from HBM holds its place for about
// 0.55 us, one from the L2 for 0.13, so a compute unit brings 25 GB/s of the one or 110 GB/s of the other, and the launch wants every
// compute unit to take an equal share.  With one and two groups the wavefronts split the rows too (their weights meet in the L1); three
// groups with two row groups each lost 1 - 2 us with weights from HBM (4096 x 6144 100 tokens 22.8 / 24.0).  More groups with row groups: 20 - 40 % slower.
// us for the launch, the blocks before (32 columns, or 64, or 128 rows x 64 columns) / these, weights where the call before left them | from HBM: 4096 x 4096
// 36 tokens 16.7 / 15.7 | 18.1 / 17.1, 100: 20.1 / 16.9 | 21.8 / 18.5; 4096 x 6144 160: 27.6 / 22.2 | 29.3 / 24.5, 256: 28.2 / 24.0 | 38.3 / 30.1; 6144 x 9216 100: 38.7 / 31.9 | 52.3 /
// 37.7; 2048 x 3072 100: 12.3 / 10.3 | 12.9 / 10.7, 400: 17.0 / 14.7 | 17.0 / 14.9; 4096 x 512 4000: 46.2 / 27.2; 512 x 512 300: 6.6 / 5.0; equal where the blocks are what they
// were (4096 x 6144 100: 64 columns).  Up to 64 rows four groups are the most: more
// columns per block only leave compute units idle (6144 x 9216 40 tokens 29.1 / 27.4).
// Temporal loads, us without / with the non-temporal hint, weights where the call before left them (one matrix fits the 256 MiB
// last-level cache) | weights from HBM: 4096 x 6144 64 tokens 17 / 21 | 21 / 22; 6144 x 9216 64 tokens 30 / 35 | 38 / 37, 128: 40 /
// 59 | 58 / 60 (with the blocks before).
// Groups of wavefronts that split k change the order of the sums, which the O projection hands on to a rounding and the router: left out.  So are
// two k-steps behind one barrier: within 5 % either way, the barriers are not what the launch waits for.
// KG teams, of eight wavefronts two: sixteen wavefronts are the most, with 128 registers each.  With teams the blocks of 32 rows, and of 64 rows and one group, are
// launch_linear_i8's own, in other forms: by its rules no call comes here for them.
template <class Op, int KG>
int linear_rows(GemmParams& p, int N, int T, hipStream_t st) {
    static_assert(KG == 1 || KG == 4, "");
    const LinearBlock b = linear_rows_block(T, p.KT * kTileK, N);        // k as bf16 would have it in these bytes
    constexpr int K8 = KG < 2 ? KG : 2;
    if (b.rows == 128) return launch_rows<Op, 1, 8, 4, 1, 2, 4, K8>(p, N, T, 1, st);
    if constexpr (KG == 1) {
        if (b.rows == 32) return b.groups == 1 ? launch_rows<Op, 1, 2, 1, 1, 2, 8>(p, N, T, 1, st) : launch_rows<Op, 1, 2, 2, 1, 2, 8>(p, N, T, 1, st);
        if (b.groups == 1) return launch_rows<Op, 1, 4, 1, 1, 4, 8>(p, N, T, 1, st);
    }
    switch (b.groups) {
        case 2: return launch_rows<Op, 1, 4, 2, 1, 2, KG == 4 ? 4 : 6, KG>(p, N, T, 1, st);
        case 4: return launch_rows<Op, 1, 4, 4, 1, 1, 4, KG>(p, N, T, 1, st);
        case 5: return launch_rows<Op, 1, 4, 5, 1, 1, 4, K8>(p, N, T, 1, st);
        case 6: return launch_rows<Op, 1, 4, 6, 1, 1, 4, K8>(p, N, T, 1, st);
        default: return launch_rows<Op, 1, 4, 8, 1, 1, 4, K8>(p, N, T, 1, st);
    }
}

}  // namespace
}  // namespace moe
