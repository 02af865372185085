// a3, 8-bit integers: the down launch of the 256-row blocks, its last round of tiles in halves where that is at most half full.
#include "moe_ffn_gemm.h"

namespace moe {

int launch_down_i8(const GemmParams& p, int R, int n_exp, hipStream_t st) { return launch_stages<Int8<__bf16>, 1, 2, BM, true>(p, R, n_exp, st); }

}  // namespace moe
