// a3 and the dense linear map in 8-bit integers: which kernel a launch takes.
//
//   gate/up:  g, u = (whole-number sums) * x_scale[row] * w_scale[column],  h = bf16(silu(g) * u)
//   between:  the rows of h in 8 bits with a scale each (moe_quant.hip)
//   down:     out = bf16((whole-number sums) * h_scale[row] * row_w[row] * w_scale[column])
// h is rounded to bf16 on its way to the 8 bits, as the bf16 layer's is: its scale is known only when all column tiles of its row are done, and as
// float32 the way there and back would cost twice the bytes.  The step of the 8 bits is max |h| / 127; bf16 is off by |h| / 256 at most, which is half of
// that step for the largest values and less for all others: with the half step of the 8 bits themselves h_q is off by up to a whole one.  out is rounded
// to bf16 to halve the bytes that the down launch writes and the combine reads; the product itself, an exact sum times two scales, would have float32.
//   What the roundings do, in numpy on normal values, 4096 x 14336: by way of bf16 1.1 % of the whole numbers are others (by one), h_q is off by 2.842e-2 of h's rms
// instead of 2.837e-2; out is off by 3.500e-2 of the same network on operands that are not quantised, 3.505e-2 with h's rounding and 3.510e-2 with both.  1024 x
// 2816: 1.2 %, 2.145e-2 instead of 2.139e-2; 2.813e-2, 2.815e-2 and 2.819e-2.
//
// Kernels, tiles and pages count bytes along k (moe_ffn_op.h), so a launch over k integers is the launch over k / 2 bf16 in its loads, its MFMAs and their
// times, and the rules measured for those hold with k / 2 in the place of k.
#include "moe_ffn_rows.h"
#include "moe_ffn_thin.h"

namespace moe {

typedef Int8<float> ToFloat;
typedef Int8<__bf16> ToBf16;
constexpr int kUnits = 256;                  // compute units
constexpr int kTileRows = 256;               // of the blocks of moe_ffn_gemm.h

// The kernel for few rows up to this many rows per expert on average.  us for the call, that kernel / the 256-row blocks: Mixtral-8x7B shape 37 rows 242 / 250, 75: 256 / 263, 100: 268 / 273, 125: 356 /
// 286; 2048 x 4096 64: 59.3 / 61.2, 100: 63.7 / 63.8, 125: 79 / 66; 1024 x 2816 80: 38.1 / 38.5, 100: 40.5 / 39.2; 64 experts of 2048 x 1024 80: 96 / 107, 100: 102 / 111, 125: 128 / 117; DBRX shape 80: 557 / 571,
// 100: 580 / 580; 40 % of the rows on one expert, 2048 x 4096 64: 67.5 / 74, 100: 73 / 75, Mixtral-8x7B shape 64: 282 / 296, 100: 322 / 327.
constexpr int kFewRows = 96;
// Weights with the non-temporal hint beyond this many bytes: half of the last-level cache.  A layer's weights are still there from the call before only in a program that has no other layer.  us,
// without / with the hint, 2048 x 4096 (201 MB), the same weights in every call | three layers in turn: 16 tokens 40 / 38 | 45 / 41, 100: 46 / 51 | 53 / 50, 400: 57 / 63 | 63 / 61; 1024 x 2816 (69 MB) 100
// tokens 28 / 30 | 28 / 31, six layers 32 / 31.  Mixtral-8x7B shape 64 tokens 255 / 231, 256: 288 / 252, 1000: 421 / 389.
constexpr int64_t kHintBytes = (int64_t)128 << 20;

// Blocks of the kernel for few rows: 64 rows up to kRows64Max per expert on average, else 128.  Features per block: 128, which read the rows half as often as 64, where these are blocks enough.  us for the
// call, 64 / 128: 2048 x 4096 160 tokens (256 blocks of 128) 53.6 / 52.4, 64 experts of 2048 x 1024 320 tokens 87.0 / 85.3, 1024 x 2816 64 tokens 31.4 / 30.3, 5 experts of 1280 x 768 (30) 26 tokens 18.1 / 20.3, 133: 23.8 / 24.8.
// Where 64 take over, below 64 or 128 blocks, was looked at on the last of these alone, whose 30 are far below either.
//   With more than kRows64Max rows 112 where a compute unit then has less to read: it has weights from HBM at 25 GB/s whatever the others do, so the one with the most blocks is what the launch waits for.  112 / 128:
// Mixtral-8x7B shape 256 tokens (1024 blocks, four to a compute unit / 896, three and a half) 245.6 / 249.2, DBRX shape 320 tokens (six / five and a quarter) 551 / 558, but 2048 x 4096 256 tokens (296 / 256) 67.4 / 56.0.
static int launch_gate_up_few(GemmParams& p, const moe_shape& s, int R, int rows_each, hipStream_t st) {
    const int64_t groups = s.F / 16;
    const bool tall = rows_each > kRows64Max;
    if (s.E * (groups / 8) < (tall ? 64 : 128)) return tall ? launch_rows<ToFloat, 0, 8, 4, 1, 1, 2>(p, s.F, R, s.E, st) : launch_rows<ToFloat, 0, 4, 4, 1, 1, 4>(p, s.F, R, s.E, st);
    if (!tall) return launch_rows<ToFloat, 0, 4, 8, 1, 1, 4>(p, s.F, R, s.E, st);
    auto longest = [&](int cw) { return (s.E * ((groups + cw - 1) / cw) + kUnits - 1) / kUnits * (2 * cw + 1); };      // half a group's time for the rows
    return longest(7) < longest(8) ? launch_rows<ToFloat, 0, 8, 7, 1, 1, 2>(p, s.F, R, s.E, st) : launch_rows<ToFloat, 0, 8, 8, 1, 1, 2>(p, s.F, R, s.E, st);
}

// Columns per block: 128, or 64 or 32 where they still make one round and 128 leave compute units without a block.  us for the call, 128 / 64 / 32: 2048 x 4096 64 tokens (128 blocks of 128) 47.9 / 44.8 / 44.6, 256: 56.3 / 52.7 /
// 57.6; 1024 x 2816 64 tokens (64) 31.3 / 28.7 / 28.1, 256: 36.6 / 34.9 / 34.4; 5 experts of 1280 x 768 66 tokens (50) 20.3 / 19.6 / 19.6, but 106 tokens (128 rows to a block, six k-steps) 24.2 / 24.9 / 25.2; Mixtral-8x7B shape 64 (256)
// 230 / 231 / 233, 256: 250 / 263 / 293.  The twelve k-steps lie between the six of that shape and the 22 of 1024 x 2816; nothing between them was measured.
static int launch_down_few(GemmParams& p, const moe_shape& s, int R, int rows_each, hipStream_t st) {
    const int64_t blocks = (int64_t)s.E * (s.H / 128);
    if (rows_each > kRows64Max) {
        if (2 * blocks <= kUnits && p.KT >= 12) return launch_rows<ToBf16, 1, 8, 4, 1, 1, 4>(p, s.H, R, s.E, st);
        return launch_rows<ToBf16, 1, 8, 8, 1, 1, 4>(p, s.H, R, s.E, st);
    }
    if (4 * blocks <= kUnits) return launch_rows<ToBf16, 1, 4, 2, 1, 1, 4>(p, s.H, R, s.E, st);
    if (2 * blocks <= kUnits) return launch_rows<ToBf16, 1, 4, 4, 1, 1, 4>(p, s.H, R, s.E, st);
    return launch_rows<ToBf16, 1, 4, 8, 1, 1, 4>(p, s.H, R, s.E, st);
}

int launch_expert_ffn_i8(const moe_shape& s, const FfnI8Args& a, hipStream_t st) {
    const int R = s.T * s.k, rows_each = R / s.E;
    const Geom g = geometry(s);
    FfnArgs f{};
    f.x_perm = a.x;
    f.offsets = a.offsets;
    f.page_table = a.page_table;
    f.pool = a.pool;
    f.pool_pages = a.pool_pages;
    f.h = a.h;
    f.out = (float*)a.out;
    f.status = a.status;
    f.e_end = s.E;
    f.gather_src = a.row_src;
    GemmParams p{};
    fill_common(p, s, g, f);
    fill_gate_up(p, s, g, f);
    p.a_scale = a.x_scale;
    p.w_scale = a.scales.w1;
    p.w_scale_up = a.scales.w3;
    // as launch_expert_ffn_bf16 (moe_ffn_bf16.hip)
    const bool streams = rows_each <= 256 && (int64_t)s.E * 3 * s.H * s.F > kHintBytes;
    p.stream = !streams ? 0 : s.F >= 6144 && s.E * g.dt >= kUnits ? 2 : 1;
    const bool few = rows_each <= kFewRows;
    const int64_t row_tiles_each = std::max<int64_t>(1, (rows_each - p.tall_rows + kTileRows - 1) / kTileRows);
    auto half_round = [&]() {
        const int64_t last = s.E * row_tiles_each * p.NT % kUnits;
        return last != 0 && last <= kUnits / 2;
    };
    int rc = !few ? (half_round() ? launch_gate_up_halves_i8(p, R, s.E, st) : launch_gate_up_i8(p, R, s.E, st))
             : thin_takes_gate_up(s) ? launch_thin<ToFloat, 0, 2>(p, s.F, R, s.E, st) : launch_gate_up_few(p, s, R, rows_each, st);
    if (rc != MOE_OK) return rc;
    rc = launch_quantize_i8(R, s.F, a.h, MOE_DTYPE_BF16, s.F, a.h_q, a.h_scale, p.stream != 0, const_cast<int32_t*>(a.offsets) + s.E, false, st);      // only read
    if (rc != MOE_OK) return rc;
    fill_down(p, s, g, f);
    p.A = (const char*)a.h_q;
    p.a_scale = a.h_scale;
    p.w_scale = a.scales.w2;
    p.row_w = a.row_w;
    if (few) return thin_takes_down(s, s.F / 2) ? launch_thin<ToBf16, 1, 1>(p, s.H, R, s.E, st) : launch_down_few(p, s, R, rows_each, st);
    const int opt = get_opt(OPT_DOWN_COLS);
    const int64_t narrow_tiles = s.E * row_tiles_each * g.dt;
    if (opt == 1 || (opt == 0 && narrow_tiles <= kUnits)) {
        p.NT = (int32_t)g.dt;
        return narrow_tiles <= kUnits / 2 ? launch_down_narrow_halves_i8(p, R, s.E, st) : launch_down_narrow_i8(p, R, s.E, st);
    }
    // Always with the last round in halves where the tiles that the routing makes leave it at most half full: even routings lose nothing by it, uneven ones, whose tiles the host does not know, gain.  us for
    // the call, whole / halves: Mixtral-8x7B shape 4096 tokens even 1172 / 1172, 40 % of the rows on one expert 1266 / 1240, 2500 of those 851 / 823; 2048 x 4096 4096 tokens even 212 / 212, uneven 274 / 259.
    return launch_down_i8(p, R, s.E, st);
}

int launch_linear_i8(const LinearI8Args& a, hipStream_t st) {
    GemmParams p{};
    p.A = (const char*)a.x;
    p.lda_bytes = a.K;
    p.dense_rows = a.T;
    p.table = a.page_table;
    p.pool = a.pool;
    p.page_bytes = a.page_bytes;
    p.tile_bytes = (int64_t)kTileN * kTileKI8;
    p.pool_pages = (int32_t)std::min<int64_t>(a.pool_pages, 0x7fffffff);
    p.tpp = (int32_t)(a.page_bytes / p.tile_bytes);
    p.ppe = (int32_t)a.pages;
    p.KT = a.K / kTileKI8;
    p.n_page_tiles = a.N / kTileN;
    p.e_end = 1;
    p.out = a.out;
    p.ldo = a.N;
    p.n_cols = a.N;
    p.status = a.status;
    p.a_scale = a.x_scale;
    p.w_scale = a.w_scale;
    p.xcd_remap = get_opt(OPT_XCD_REMAP);
    p.half_tiles = get_opt(OPT_HALF_TILES);
    p.tall_rows = get_opt(OPT_TALL_TILES) ? 32 : 0;
    p.tall_first = get_opt(OPT_TALL_FIRST);
    p.balance = get_opt(OPT_BALANCE);
    p.chunked = std::min(std::max(get_opt(OPT_CHUNKED), 0), 32);
    // as launch_linear_bf16 (moe_ffn_bf16.hip)
    if (linear_takes_rows_kernel(a.T, a.K / 2, a.N)) {
        // Teams that share k, since sums of whole numbers are exact in any order: a block's way through all of k is what a launch of one round waits for.  us, one team /
        // four (of eight wavefronts: two), weights where the call before left them | from HBM: 4096 x 6144 40 rows 13.5 / 11.9 | 16.4 / 13.3, 256: 19.2 / 18.5 | 21.4 / 19.9; 14336 x 4096 100: 40.8 / 30.3 |
        // 44.8 / 32.3; 2048 x 4096 40: 9.0 / 8.4 | 9.4 / 8.3, 256: 10.6 / 10.7 | 11.5 / 11.4; below 2048 the start of the teams costs what they save.
        //   Where blocks of 32 rows and 16 columns make one round: eight teams of two wavefronts, with a k of middle length, or where only 32 columns make one round, four teams of
        // four.  us, the blocks above / 32 x 16 / 32 x 32: 4096 x 1024 100 rows 9.9 / 7.3 / 8.7, 4096 x 128 1000: 11.0 / 8.0 / 8.8, 2000: 11.9 / 16.6 / 9.9, 14336 x 512 256: 26.9 / 17.7 / 22.6, 14336 x 4096 1: 30.6 / 17.2 / 18.0,
        // 2816 x 1024 100: 8.8 / 7.4 / 7.7, 2048 x 1024 100: 7.2 / 6.8 / 6.4, 1536 x 1024: 6.8 / 6.7 / 6.3, 1024 x 1024: 5.7 / 6.5 / 6.0.
        const int64_t row_tiles = ((int64_t)a.T + 31) / 32;
        if (p.KT >= 20 && row_tiles * (a.N / 16) <= kUnits) return launch_rows<ToFloat, 1, 2, 1, 1, 2, 4, 8>(p, a.N, a.T, 1, st);
        if (p.KT >= 12 && row_tiles * (a.N / 32) <= kUnits) return launch_rows<ToFloat, 1, 2, 2, 1, 2, 4, 4>(p, a.N, a.T, 1, st);
        // Or 48 columns, four teams of three: 4096 x 6144 64 rows 11.5 / 10.2 (from HBM 14.0 / 12.0), 6144 x 6144 36: 13.9 / 13.0 (16.8 / 14.8).
        if (p.KT >= 20 && row_tiles * ((a.N / 16 + 2) / 3) <= kUnits) return launch_rows<ToFloat, 1, 2, 3, 1, 1, 4, 4>(p, a.N, a.T, 1, st);
        return p.KT < 16 ? linear_rows<ToFloat, 1>(p, a.N, a.T, st) : linear_rows<ToFloat, 4>(p, a.N, a.T, st);
    }
    const int wide_tiles = (p.n_page_tiles + 1) / 2;
    if ((int64_t)(a.T / kTileRows + 1) * wide_tiles >= 2 * kUnits) {
        p.NT = wide_tiles;
        return launch_linear_wide_i8(p, a.T, st);
    }
    p.NT = p.n_page_tiles;
    const int64_t half_tiles = (int64_t)((a.T + 127) / 128) * p.NT;
    const bool low = p.half_tiles && a.T > 128 && half_tiles <= kUnits && (a.T > 160 || half_tiles <= 224 || p.KT <= 32);
    if (low) p.tall_rows = 0;
    return launch_linear_narrow_i8(p, low ? 128 : kTileRows, a.T, st);
}

}  // namespace moe
