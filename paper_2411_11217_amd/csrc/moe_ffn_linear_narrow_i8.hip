// The dense linear map in 8-bit integers: launches of blocks with 128 columns and 256 or 128 rows.
#include "moe_ffn_gemm.h"

namespace moe {

int launch_linear_narrow_i8(const GemmParams& p, int rows, int T, hipStream_t st) {
    return rows == 128 ? launch_stages<Int8<float>, 1, 1, 128>(p, T, 1, st) : launch_stages<Int8<float>, 1, 1>(p, T, 1, st);
}

}  // namespace moe
