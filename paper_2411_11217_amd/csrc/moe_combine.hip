// a4. Un-permute and combine: y[t] = sum_slot w[t][slot] * out[row_of[t*k+slot]].
// Pure HBM traffic (read R*H floats, or bf16 behind 8-bit products, write T*H floats): one block per token,
// four elements at a time along the row, the k rows of a token summed in slot order so the
// result does not depend on scheduling.
#include <type_traits>

#include "moe_internal.h"

namespace moe {
namespace {

__device__ __forceinline__ float4 as_floats(const float4& v) { return v; }
__device__ __forceinline__ float4 as_floats(const uint2& v) {        // four bf16
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
}

template <class Four>
__global__ __launch_bounds__(256) void combine_kernel(const Four* __restrict__ out, const int32_t* __restrict__ row_of,
                                                      const float* __restrict__ topk_w, int k, int R, int row_vec,
                                                      float4* __restrict__ y, const int32_t* __restrict__ found, int32_t* __restrict__ status) {
    const int t = blockIdx.x;
    __shared__ int32_t rows[MOE_MAX_EXPERTS];
    __shared__ float wts[MOE_MAX_EXPERTS];
    if (threadIdx.x < k) {
        const int r = row_of[(size_t)t * k + threadIdx.x];
        rows[threadIdx.x] = min(max(r, 0), R - 1);          // never leaves the buffer
        wts[threadIdx.x] = topk_w ? topk_w[(size_t)t * k + threadIdx.x] : 1.0f;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < row_vec; c += 256) {
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < k; ++s) {
            const float4 v = as_floats(out[(size_t)rows[s] * row_vec + c]);
            const float ws = wts[s];
            acc.x = fmaf(ws, v.x, acc.x);
            acc.y = fmaf(ws, v.y, acc.y);
            acc.z = fmaf(ws, v.z, acc.z);
            acc.w = fmaf(ws, v.w, acc.w);
        }
        y[(size_t)t * row_vec + c] = acc;
    }
    if constexpr (std::is_same<Four, uint2>::value)
        if (t == 0 && threadIdx.x == 0 && found && found[0]) atomicOr(status, found[0]);
}

}  // namespace

int launch_combine(const moe_shape& s, const void* out, const int32_t* row_of, const float* topk_w, float* y,
                   hipStream_t st, const int32_t* found, int32_t* status) {
    if (s.dtype == MOE_DTYPE_I8)
        hipLaunchKernelGGL(combine_kernel<uint2>, dim3(s.T), dim3(256), 0, st, (const uint2*)out, row_of, topk_w, s.k, s.T * s.k, s.H / 4, (float4*)y, found, status);
    else
        hipLaunchKernelGGL(combine_kernel<float4>, dim3(s.T), dim3(256), 0, st, (const float4*)out, row_of, topk_w, s.k, s.T * s.k, s.H / 4, (float4*)y, nullptr, nullptr);
    MOE_HIP_TRY(hipGetLastError());
    return MOE_OK;
}

}  // namespace moe
