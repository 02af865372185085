// a3, 8-bit integers: the gate/up launch of the 256-row blocks.  Every kernel of these blocks has a file of its own: each takes a minute or more to compile.
#include "moe_ffn_gemm.h"

namespace moe {

int launch_gate_up_i8(const GemmParams& p, int R, int n_exp, hipStream_t st) { return launch_stages<Int8<float>, 0, 2>(p, R, n_exp, st); }

}  // namespace moe
