// The dense linear map in 8-bit integers: launches of the 256-row blocks with 256 columns.
#include "moe_ffn_gemm.h"

namespace moe {

int launch_linear_wide_i8(const GemmParams& p, int T, hipStream_t st) { return launch_stages<Int8<float>, 1, 2>(p, T, 1, st); }

}  // namespace moe
