// a3 and the dense linear map in 8-bit integers: which kernel a launch takes.
//
//   gate/up:  g, u = (whole-number sums) * x_scale[row] * w_scale[column],  h = bf16(silu(g) * u)
//   between:  the rows of h in 8 bits with a scale each (moe_quant.hip)
//   down:     out = bf16((whole-number sums) * h_scale[row] * row_w[row] * w_scale[column])
// h is rounded to bf16 on its way to the 8 bits, as the bf16 layer's is: its scale is known only when all column tiles of its row are done, and as
// float32 the way there and back would cost twice the bytes.  The step of the 8 bits is max |h| / 127; bf16 is off by |h| / 512 at most, a quarter of
// that step for the largest values and less for all others.
#include "moe_ffn_rows.h"

namespace moe {

typedef Int8<float> ToFloat;
typedef Int8<__bf16> ToBf16;

int launch_expert_ffn_i8(const moe_shape& s, const FfnI8Args& a, hipStream_t st) {
    const int R = s.T * s.k;
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
    int rc = launch_rows<ToFloat, 0, 8, 8, 1, 1, 2>(p, s.F, R, s.E, st);
    if (rc != MOE_OK) return rc;
    rc = launch_quantize_i8(R, s.F, a.h, MOE_DTYPE_BF16, s.F, a.h_q, a.h_scale, st);
    if (rc != MOE_OK) return rc;
    fill_down(p, s, g, f);
    p.A = (const char*)a.h_q;
    p.a_scale = a.h_scale;
    p.w_scale = a.scales.w2;
    p.row_w = a.row_w;
    return launch_rows<ToBf16, 1, 8, 8, 1, 1, 4>(p, s.H, R, s.E, st);
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
    return launch_rows<ToFloat, 1, 4, 4, 1, 1, 4>(p, a.N, a.T, 1, st);
}

}  // namespace moe
