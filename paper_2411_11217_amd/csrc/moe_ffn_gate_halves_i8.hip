// a3, 8-bit integers: the gate/up launch whose last round of tiles is computed in halves (see tail_tile in moe_tile_order.h).
#include "moe_ffn_gemm.h"

namespace moe {

int launch_gate_up_halves_i8(const GemmParams& p, int R, int n_exp, hipStream_t st) { return launch_stages<Int8<float>, 0, 2, BM, true>(p, R, n_exp, st); }

}  // namespace moe
