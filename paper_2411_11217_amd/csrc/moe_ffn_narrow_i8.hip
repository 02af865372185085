// a3, 8-bit integers: the down launch with 128-wide column tiles, whole, or with 64-wide ones in its last, or only, round.
#include "moe_ffn_gemm.h"

namespace moe {

int launch_down_narrow_i8(const GemmParams& p, int R, int n_exp, hipStream_t st) { return launch_stages<Int8<__bf16>, 1, 1>(p, R, n_exp, st); }

int launch_down_narrow_halves_i8(const GemmParams& p, int R, int n_exp, hipStream_t st) { return launch_stages<Int8<__bf16>, 1, 1, BM, true>(p, R, n_exp, st); }

}  // namespace moe
