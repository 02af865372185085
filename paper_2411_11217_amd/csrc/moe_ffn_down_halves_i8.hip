// a3, 8-bit integers: the down launch whose last round of tiles is computed in halves.
#include "moe_ffn_gemm.h"

namespace moe {

int launch_down_halves_i8(const GemmParams& p, int R, int n_exp, hipStream_t st) { return launch_stages<Int8<__bf16>, 1, 2, BM, true>(p, R, n_exp, st); }

}  // namespace moe
