// Rows in 8-bit integers with a scale each: any rows (moe_quantize_i8), and the rows of the residual and RMS norm (moe_add_rmsnorm_i8).
//
//   scale = max |v| / 127,  q = rint(v * (127 / max |v|)),  q * scale stands for v, off by at most half a scale
//
// All of it in float32, each operation rounded by itself (no fused multiply-add), so that the whole numbers are the same
// wherever they are computed that way.  A scale is at least 2^-126: below that its inverse would not be a float, and a row of
// zeros has a scale like any other.  A row that holds an infinity or a NaN has the scale NaN and zeros, so that every product
// with it is NaN rather than a number that looks like one.
#include <algorithm>

#include "moe_internal.h"

using namespace moe;

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kInfinity = 0x7f800000u;
constexpr float kSmallest = 0x1p-126f;

// The largest of non-negative floats by their bits, over a row's threads: an infinity is above every number and a NaN above that.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, m, 64));
    return v;
}
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t magnitude(const f32x4& v) { return max(max(magnitude(v.x), magnitude(v.y)), max(magnitude(v.z), magnitude(v.w))); }

struct RowScale {
    float scale, inverse;
};
__device__ __forceinline__ RowScale scale_of(uint32_t most) {
    if (most >= kInfinity) return {__uint_as_float(0x7fc00000u), 0.f};
    const float m = __uint_as_float(most);
    return {fmaxf(m / 127.f, kSmallest), fminf(127.f / m, 1.f / kSmallest)};
}

// Four whole numbers in a word.  Adding 1.5 * 2^23 rounds to the nearest whole number, ties to even, and leaves it in the low bits.
__device__ __forceinline__ uint32_t quantized(const f32x4& v, const RowScale& s) {
#pragma clang fp contract(off)
    if (s.inverse == 0.f) return 0;              // 0 * infinity is not
    constexpr float magic = 12582912.f;
    const uint32_t a = __float_as_uint(v.x * s.inverse + magic), b = __float_as_uint(v.y * s.inverse + magic), c = __float_as_uint(v.z * s.inverse + magic),
                   d = __float_as_uint(v.w * s.inverse + magic);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400), __builtin_amdgcn_perm(b, a, 0x0c0c0400), 0x05040100);
}

__device__ __forceinline__ f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
__device__ __forceinline__ f32x4 load4(const uint16_t* p) {
    const u32x2 v = *reinterpret_cast<const u32x2*>(p);
    return f32x4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)};
}

constexpr int kThreads = 256;

// A block to a row.  PER vectors of four elements to a thread stay in registers; with PER = 0 the row is read twice.
template <class In, int PER>
__global__ __launch_bounds__(kThreads) void quantize_kernel(const In* __restrict__ x, int64_t row_elements, int T, int vectors, uint32_t* __restrict__ q,
                                                            float* __restrict__ scale) {
    __shared__ uint32_t part[kThreads / 64];
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
        const In* const row = x + t * row_elements;
        uint32_t* const out = q + t * vectors;
        f32x4 v[PER ? PER : 1];
        uint32_t most = 0;
        if constexpr (PER > 0) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int c = threadIdx.x + i * kThreads;
                v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (c < vectors) v[i] = load4(row + 4 * c);
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) most = max(most, magnitude(v[i]));
        } else {
            for (int c = threadIdx.x; c < vectors; c += kThreads) most = max(most, magnitude(load4(row + 4 * (int64_t)c)));
        }
        most = wave_max(most);
        __syncthreads();                         // the row before this one has read `part`
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
        __syncthreads();
        const RowScale s = scale_of(max(max(part[0], part[1]), max(part[2], part[3])));
        if constexpr (PER > 0) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int c = threadIdx.x + i * kThreads;
                if (c < vectors) out[c] = quantized(v[i], s);
            }
        } else {
            for (int c = threadIdx.x; c < vectors; c += kThreads) out[c] = quantized(load4(row + 4 * (int64_t)c), s);
        }
        if (threadIdx.x == 0) scale[t] = s.scale;
    }
}

constexpr int kMostBlocks = 1 << 20;             // rows beyond them are taken in turn

template <class In>
int launch_quantize(int T, int N, const In* x, int64_t row_elements, int8_t* q, float* scale, hipStream_t st) {
    const dim3 grid(std::min(T, kMostBlocks)), block(kThreads);
    const int vectors = N / 4, per = (vectors + kThreads - 1) / kThreads;
    if (per <= 4) hipLaunchKernelGGL((quantize_kernel<In, 4>), grid, block, 0, st, x, row_elements, T, vectors, (uint32_t*)q, scale);
    else if (per <= 16) hipLaunchKernelGGL((quantize_kernel<In, 16>), grid, block, 0, st, x, row_elements, T, vectors, (uint32_t*)q, scale);
    else hipLaunchKernelGGL((quantize_kernel<In, 0>), grid, block, 0, st, x, row_elements, T, vectors, (uint32_t*)q, scale);
    MOE_HIP_TRY(hipGetLastError());
    return MOE_OK;
}

// One block per row, as add_rmsnorm_kernel (moe_dense.hip): s = hidden + delta stays in registers, its squares are added up, then the
// magnitudes of y are compared.
constexpr int kMaxVec = 8;                       // vectors of four to a thread: H <= 8192

struct NormArgs {
    const float *hidden, *delta, *gamma;
    float* hidden_out;
    uint16_t* x_out;
    uint32_t* q;
    float* scale;
    float eps;
    int T, vectors;
};

template <int PER>
__global__ __launch_bounds__(kThreads) void add_rmsnorm_i8_kernel(const NormArgs a) {
    __shared__ float sums[kThreads / 64];
    __shared__ uint32_t part[kThreads / 64];
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const int64_t row = t * a.vectors;
        f32x4 v[PER];
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = threadIdx.x + i * kThreads;
            v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (c < a.vectors) {
                v[i] = load4(a.delta + 4 * (row + c));
                if (a.hidden) v[i] += load4(a.hidden + 4 * (row + c));
            }
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = threadIdx.x + i * kThreads;
            if (c < a.vectors && a.hidden_out) *reinterpret_cast<f32x4*>(a.hidden_out + 4 * (row + c)) = v[i];
            ss += (v[i].x * v[i].x + v[i].y * v[i].y) + (v[i].z * v[i].z + v[i].w * v[i].w);
        }
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) ss += __shfl_xor(ss, m, 64);
        if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = ss;
        __syncthreads();
        const float r = 1.f / sqrtf(((sums[0] + sums[1]) + (sums[2] + sums[3])) / (float)(a.vectors * 4) + a.eps);
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = threadIdx.x + i * kThreads;
            if (c < a.vectors) v[i] = v[i] * r * load4(a.gamma + 4 * c);
            most = max(most, magnitude(v[i]));
        }
        most = wave_max(most);
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
        __syncthreads();                         // also: everyone has read `sums`
        const RowScale s = scale_of(max(max(part[0], part[1]), max(part[2], part[3])));
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = threadIdx.x + i * kThreads;
            if (c >= a.vectors) continue;
            if (a.x_out) *reinterpret_cast<u32x2*>(a.x_out + 4 * (row + c)) = __builtin_bit_cast(u32x2, __builtin_convertvector(v[i], bf16x4));      // to nearest even
            a.q[row + c] = quantized(v[i], s);
        }
        if (threadIdx.x == 0) a.scale[t] = s.scale;
    }
}

}  // namespace

namespace moe {

int launch_quantize_i8(int T, int N, const void* x, int x_dtype, int64_t row_elements, int8_t* q, float* scale, hipStream_t st) {
    return x_dtype == MOE_DTYPE_F32 ? launch_quantize(T, N, (const float*)x, row_elements, q, scale, st) : launch_quantize(T, N, (const uint16_t*)x, row_elements, q, scale, st);
}

int launch_add_rmsnorm_i8(int T, int H, const float* hidden, const float* delta, const float* gamma, float eps, float* hidden_out, void* x_out, int8_t* q, float* scale,
                          hipStream_t st) {
    const NormArgs a{hidden, delta, gamma, hidden_out, (uint16_t*)x_out, (uint32_t*)q, scale, eps, T, H / 4};
    const dim3 grid(std::min(T, kMostBlocks)), block(kThreads);
    if (a.vectors <= 4 * kThreads) hipLaunchKernelGGL((add_rmsnorm_i8_kernel<4>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((add_rmsnorm_i8_kernel<kMaxVec>), grid, block, 0, st, a);
    MOE_HIP_TRY(hipGetLastError());
    return MOE_OK;
}

bool norm_takes(int32_t H, float eps) { return H > 0 && H % 4 == 0 && H <= 4 * kThreads * kMaxVec && eps >= 0.f; }

}  // namespace moe

extern "C" {

int moe_quantize_i8(int32_t T, int32_t N, const void* x, int32_t x_dtype, int64_t row_elements, int8_t* x_q, float* x_scale, void* stream) {
    if (x_dtype != MOE_DTYPE_F32 && x_dtype != MOE_DTYPE_BF16) return MOE_ERR_UNSUPPORTED_DTYPE;
    if (T < 0 || N <= 0 || N % 4 != 0 || row_elements < N || row_elements % 4 != 0 || row_elements > INT32_MAX) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    const int64_t esize = x_dtype == MOE_DTYPE_F32 ? 4 : 2, x_bytes = ((T - 1) * row_elements + N) * esize, q_bytes = (int64_t)T * N, s_bytes = (int64_t)T * 4;
    if (!x || !x_q || !x_scale || (uintptr_t)x % (4 * esize) != 0 || (uintptr_t)x_q % 4 != 0 || (uintptr_t)x_scale % 4 != 0) return MOE_ERR_INVALID_ARG;
    if (overlap(x, x_bytes, x_q, q_bytes) || overlap(x, x_bytes, x_scale, s_bytes) || overlap(x_q, q_bytes, x_scale, s_bytes)) return MOE_ERR_INVALID_ARG;
    return launch_quantize_i8(T, N, x, x_dtype, row_elements, x_q, x_scale, (hipStream_t)stream);
}

int moe_add_rmsnorm_i8(int32_t T, int32_t H, const float* hidden, const float* delta, const float* gamma, float eps, float* hidden_out, void* x_out, int8_t* x_q,
                       float* x_scale, void* stream) {
    if (T < 0 || !norm_takes(H, eps)) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if (!delta || !gamma || !x_q || !x_scale || (uintptr_t)x_q % 4 != 0 || (uintptr_t)x_scale % 4 != 0 || (uintptr_t)x_out % 8 != 0) return MOE_ERR_INVALID_ARG;
    if (!aligned16(hidden) || !aligned16(delta) || !aligned16(gamma) || !aligned16(hidden_out)) return MOE_ERR_INVALID_ARG;
    const int64_t n = (int64_t)T * H;
    const struct { const void* p; int64_t bytes; } in[] = {{hidden, n * 4}, {delta, n * 4}, {gamma, (int64_t)H * 4}},
        out[] = {{hidden_out, n * 4}, {x_out, n * 2}, {x_q, n}, {x_scale, (int64_t)T * 4}};
    for (int o = 0; o < 4; ++o) {
        if (!out[o].p) continue;
        for (const auto& i : in)       // the residual stream may be updated in place
            if (i.p && overlap(i.p, i.bytes, out[o].p, out[o].bytes) && !(o == 0 && out[o].p == i.p && i.p != gamma)) return MOE_ERR_INVALID_ARG;
        for (int q = o + 1; q < 4; ++q)
            if (out[q].p && overlap(out[o].p, out[o].bytes, out[q].p, out[q].bytes)) return MOE_ERR_INVALID_ARG;
    }
    return launch_add_rmsnorm_i8(T, H, hidden, delta, gamma, eps, hidden_out, x_out, x_q, x_scale, (hipStream_t)stream);
}

}  // extern "C"
