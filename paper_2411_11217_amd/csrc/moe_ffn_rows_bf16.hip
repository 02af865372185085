// a3 and the dense linear map for launches with few rows per expert, bf16 operands: where a launch comes here, and with which blocks (the kernel
// is in moe_ffn_rows.h).
#include "moe_ffn_rows.h"

namespace moe {
// Where the expert GEMMs take this kernel: up to 80 rows per expert on average (of all experts: the launches of a streamed
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
constexpr int kRowsKernelMax = 80;
// Up to here 64-row blocks with half the columns; 45 .. 72 rows need two of them per expert for some experts, and the second
// one reads the weights again (176 tokens of the Mixtral-8x7B shape, 44 rows: 489 against 503 with 128-row blocks).
constexpr int kRows64Max = 44;

bool rows_kernel_takes(int rows_each) { return rows_each <= kRowsKernelMax; }

int launch_gate_up_rows_bf16(GemmParams& p, int F, int R, int rows_each, int n_exp, hipStream_t st) {
    if (rows_each <= kRows64Max) return launch_rows<Bf16, 0, 4, 4, 1, 1, 4>(p, F, R, n_exp, st);
    return launch_rows<Bf16, 0, 8, 8, 1, 1, 2>(p, F, R, n_exp, st);
}

int launch_down_rows_bf16(GemmParams& p, int H, int R, int rows_each, int n_exp, hipStream_t st) {
    if (rows_each <= kRows64Max) return launch_rows<Bf16, 1, 4, 4, 2, 1, 4>(p, H, R, n_exp, st);
    return launch_rows<Bf16, 1, 8, 8, 1, 1, 4>(p, H, R, n_exp, st);
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
int launch_linear_rows_bf16(GemmParams& p, int N, int T, hipStream_t st) {
    const LinearBlock b = linear_rows_block(T, p.KT * kTileK, N);
    if (b.rows == 128) return launch_rows<Bf16, 1, 8, 4, 1, 2, 4>(p, N, T, 1, st);
    if (b.rows == 32) return b.groups == 1 ? launch_rows<Bf16, 1, 2, 1, 1, 2, 8>(p, N, T, 1, st) : launch_rows<Bf16, 1, 2, 2, 1, 2, 8>(p, N, T, 1, st);
    switch (b.groups) {
        case 1: return launch_rows<Bf16, 1, 4, 1, 1, 4, 8>(p, N, T, 1, st);
        case 2: return launch_rows<Bf16, 1, 4, 2, 1, 2, 6>(p, N, T, 1, st);
        case 4: return launch_rows<Bf16, 1, 4, 4, 1, 1, 4>(p, N, T, 1, st);
        case 5: return launch_rows<Bf16, 1, 4, 5, 1, 1, 4>(p, N, T, 1, st);
        case 6: return launch_rows<Bf16, 1, 4, 6, 1, 1, 4>(p, N, T, 1, st);
        default: return launch_rows<Bf16, 1, 4, 8, 1, 1, 4>(p, N, T, 1, st);
    }
}

}  // namespace moe
