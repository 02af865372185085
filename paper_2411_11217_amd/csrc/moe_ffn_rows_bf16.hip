// a3 and the dense linear map for launches with few rows per expert, bf16 operands.
#include "moe_ffn_rows.h"

namespace moe {

int launch_gate_up_rows_bf16(GemmParams& p, int F, int R, int rows_each, int n_exp, hipStream_t st) { return gate_up_rows<Bf16>(p, F, R, rows_each, n_exp, st); }

int launch_down_rows_bf16(GemmParams& p, int H, int R, int rows_each, int n_exp, hipStream_t st) { return down_rows<Bf16>(p, H, R, rows_each, n_exp, st); }

int launch_linear_rows_bf16(GemmParams& p, int N, int T, hipStream_t st) { return linear_rows<Bf16, 1>(p, N, T, st); }

}  // namespace moe
