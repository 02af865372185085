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

// FAR: with the non-temporal hint.  What is read here is read for the last time, and with the hint it comes faster where it does not come from the caches: us in a graph
// over buffers that exceed the last-level cache, without / with, rows in 8 bits 14336 x 4096 bf16 (176 MB) 32.0 / 30.6 (5.76 TB/s), float32 9857 x 4096 36.4 / 33.8; norm
// 9857 x 6144 (787 MB) 140 / 132 (5.96 TB/s), 30000 x 1024 84 / 77, but 4000 x 4096 (246 MB) 42.3 / 43.9.  What is written is read next: written with the hint the same
// calls take 29.1 and 131, and who reads the 8-bit rows 25 and 30 more.  Except h between two launches that stream weights (`past`): lines that the caches have
// to write back cost these more (experts of the Mixtral-8x7B shape, 256 tokens 260 / 248).  hidden_out, which nobody wants for a layer, takes the hint too.
constexpr int64_t kQuantizeFar = (int64_t)16 << 20, kNormFar = (int64_t)256 << 20;      // more bytes than these
template <bool FAR, class V>
__device__ __forceinline__ V load_as(const void* p) {
    return FAR ? __builtin_nontemporal_load(reinterpret_cast<const V*>(p)) : *reinterpret_cast<const V*>(p);
}
template <bool FAR, class V>
__device__ __forceinline__ void store_as(void* p, V v) {
    if constexpr (FAR) __builtin_nontemporal_store(v, reinterpret_cast<V*>(p));
    else *reinterpret_cast<V*>(p) = v;
}
__device__ __forceinline__ f32x4 widened(uint32_t a, uint32_t b) {   // four bf16
    return f32x4{__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u), __uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u)};
}

// VEC elements of a row as they lie in memory, 8 or 16 bytes.
template <class In, int VEC>
struct Piece;
template <>
struct Piece<float, 4> {
    typedef f32x4 Raw;
    typedef uint32_t Out;
    __device__ static uint32_t most(const Raw& v) { return magnitude(v); }
    __device__ static Out quantized4(const Raw& v, const RowScale& s) { return quantized(v, s); }
};
template <>
struct Piece<uint16_t, 4> {
    typedef u32x2 Raw;
    typedef uint32_t Out;
    __device__ static uint32_t most(const Raw& v) { return magnitude(widened(v.x, v.y)); }
    __device__ static Out quantized4(const Raw& v, const RowScale& s) { return quantized(widened(v.x, v.y), s); }
};
template <>
struct Piece<uint16_t, 8> {
    typedef u32x4 Raw;
    typedef u32x2 Out;
    __device__ static uint32_t most(const Raw& v) { return max(magnitude(widened(v.x, v.y)), magnitude(widened(v.z, v.w))); }
    __device__ static Out quantized4(const Raw& v, const RowScale& s) { return Out{quantized(widened(v.x, v.y), s), quantized(widened(v.z, v.w), s)}; }
};

constexpr int kMostBlocks = 1 << 20;             // rows beyond theirs are taken in turn

// words: device, or null: rows from *words on are left as they were, or with `clear` four words that are set to zero.  WAVES wavefronts to a row; with one, four rows to a block.  PER pieces to a thread stay in registers as they came; with PER = 0 the row is
// read twice, without hints.
template <class In, int VEC, int WAVES, int PER, bool FAR, bool PAST>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void quantize_kernel(const In* __restrict__ x, int64_t row_elements, int T, int pieces, bool clear, int8_t* __restrict__ q,
                                                                                 float* __restrict__ scale, int32_t* __restrict__ words) {
    typedef Piece<In, VEC> P;
    __shared__ uint32_t part[WAVES];
    constexpr int kRows = WAVES == 1 ? 4 : 1, kThreads = 64 * WAVES;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int me = WAVES == 1 ? lane : threadIdx.x;
    int rows = T;
    if (words) {                                 // one argument for both: with another, every launch took 0.1 to 0.6 us more
        if (!clear) rows = min(T, *words);       // wanted at the first store only
        else if (blockIdx.x == 0 && threadIdx.x < 4) words[threadIdx.x] = 0;
    }
    for (int64_t t = (int64_t)blockIdx.x * kRows + (WAVES == 1 ? wave : 0); t < T; t += (int64_t)gridDim.x * kRows) {
        const In* const row = x + t * row_elements;
        int8_t* const out = q + t * pieces * VEC;
        typename P::Raw v[PER ? PER : 1];
        uint32_t most = 0;
        if constexpr (PER > 0) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int c = me + i * kThreads;
                v[i] = typename P::Raw{};
                if (c < pieces) v[i] = load_as<FAR, typename P::Raw>(row + VEC * c);
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) most = max(most, P::most(v[i]));
        } else {
            for (int c = me; c < pieces; c += kThreads) most = max(most, P::most(load_as<false, typename P::Raw>(row + (int64_t)VEC * c)));
        }
        most = wave_max(most);
        if constexpr (WAVES > 1) {
            __syncthreads();                     // the row before this one has read `part`
            if (lane == 0) part[wave] = most;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WAVES; ++w) most = max(most, part[w]);
        }
        const RowScale s = scale_of(most);
        if (t >= rows) continue;
        if constexpr (PER > 0) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int c = me + i * kThreads;
                if (c < pieces) store_as<PAST>(out + VEC * c, P::quantized4(v[i], s));
            }
        } else {
            for (int c = me; c < pieces; c += kThreads) store_as<false>(out + (int64_t)VEC * c, P::quantized4(load_as<false, typename P::Raw>(row + (int64_t)VEC * c), s));
        }
        if (me == 0) scale[t] = s.scale;
    }
}

template <class In, int VEC, int WAVES, int PER>
int launch_quantize(int T, int pieces, const In* x, int64_t row_elements, int8_t* q, float* scale, bool past, int32_t* words, bool clear, hipStream_t st) {
    const dim3 grid(std::min(WAVES == 1 ? T / 4 + (T % 4 != 0) : T, kMostBlocks)), block(WAVES == 1 ? 256 : 64 * WAVES);
    const bool far = (int64_t)T * pieces * VEC * ((int)sizeof(In) + 1) > kQuantizeFar;
    auto kernel = quantize_kernel<In, VEC, WAVES, PER, false, false>;
    if constexpr (PER > 0) {
        if (far) kernel = quantize_kernel<In, VEC, WAVES, PER, true, false>;
        if constexpr (VEC == 8)                  // h, whose rows are multiples of 256 bf16
            if (past) kernel = quantize_kernel<In, VEC, WAVES, PER, true, true>;
    }
    hipLaunchKernelGGL(kernel, grid, block, 0, st, x, row_elements, T, pieces, clear, q, scale, words);
    MOE_HIP_TRY(hipGetLastError());
    return MOE_OK;
}

// Wavefronts by the length of the row alone: a row's loads are then under way at once, and what is in flight fills the chip.  us, 256 threads to
// every row / these: 512 x 14336 9.1 / 5.9, 8192 x 14336 88 / 64, 60000 x 256 53 / 17, 1 x 28672 10.4 / 3.2.
template <class In, int VEC>
int launch_quantize(int T, int N, const In* x, int64_t row_elements, int8_t* q, float* scale, bool past, int32_t* words, bool clear, hipStream_t st) {
    const int pieces = N / VEC;
    if (pieces <= 64) return launch_quantize<In, VEC, 1, 1>(T, pieces, x, row_elements, q, scale, past, words, clear, st);
    if (pieces <= 128) return launch_quantize<In, VEC, 1, 2>(T, pieces, x, row_elements, q, scale, past, words, clear, st);
    if (pieces <= 512) return launch_quantize<In, VEC, 4, 2>(T, pieces, x, row_elements, q, scale, past, words, clear, st);
    if (pieces <= 1024) return launch_quantize<In, VEC, 8, 2>(T, pieces, x, row_elements, q, scale, past, words, clear, st);
    if (pieces <= 2048) return launch_quantize<In, VEC, 16, 2>(T, pieces, x, row_elements, q, scale, past, words, clear, st);
    if (pieces <= 4096) return launch_quantize<In, VEC, 16, 4>(T, pieces, x, row_elements, q, scale, past, words, clear, st);
    return launch_quantize<In, VEC, 16, 0>(T, pieces, x, row_elements, q, scale, past, words, clear, st);
}

// Residual and norm: one pass over the rows.  s = hidden + delta stays in registers, its squares are added up, then the magnitudes of y are
// compared; gamma comes while the sums are formed.  How many wavefronts a row has goes by H alone, so that a row's sum, and with it its bits, are the
// same in every call.
constexpr int kMostH = 8192;

struct NormArgs {
    const float *hidden, *delta, *gamma;
    float* hidden_out;
    uint16_t* x_out;
    int8_t* q;
    float* scale;
    float eps;
    int T, vectors;                              // of four elements
};

template <int WAVES, int PER, bool FAR>
__global__ __launch_bounds__(64 * WAVES) void add_rmsnorm_i8_kernel(const NormArgs a) {
    __shared__ float sums[WAVES];
    __shared__ uint32_t part[WAVES];
    constexpr int kThreads = 64 * WAVES;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const int64_t row = t * a.vectors;
        f32x4 v[PER], g[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = threadIdx.x + i * kThreads;
            v[i] = g[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (c < a.vectors) v[i] = load_as<FAR, f32x4>(a.delta + 4 * (row + c));
        }
        if (a.hidden)
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int c = threadIdx.x + i * kThreads;
                if (c < a.vectors) g[i] = load_as<FAR, f32x4>(a.hidden + 4 * (row + c));
            }
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = threadIdx.x + i * kThreads;
            if (a.hidden) v[i] += g[i];
            if (c < a.vectors) {
                g[i] = load_as<false, f32x4>(a.gamma + 4 * c);
                if (a.hidden_out) store_as<FAR>(a.hidden_out + 4 * (row + c), v[i]);
            }
            ss += (v[i].x * v[i].x + v[i].y * v[i].y) + (v[i].z * v[i].z + v[i].w * v[i].w);
        }
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) ss += __shfl_xor(ss, m, 64);
        if constexpr (WAVES > 1) {
            if (lane == 0) sums[wave] = ss;
            __syncthreads();
            ss = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) ss += sums[w];
        }
        const float r = 1.f / sqrtf(ss / (float)(a.vectors * 4) + a.eps);
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            v[i] = v[i] * r * g[i];
            if (threadIdx.x + i * kThreads < a.vectors) most = max(most, magnitude(v[i]));      // what is behind the row is 0 * r, which may be NaN
        }
        most = wave_max(most);
        if constexpr (WAVES > 1) {
            if (lane == 0) part[wave] = most;
            __syncthreads();                     // also: everyone has read `sums`
#pragma unroll
            for (int w = 0; w < WAVES; ++w) most = max(most, part[w]);
        }
        const RowScale s = scale_of(most);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = threadIdx.x + i * kThreads;
            if (c >= a.vectors) continue;
            if (a.x_out) store_as<false>(a.x_out + 4 * (row + c), __builtin_bit_cast(u32x2, __builtin_convertvector(v[i], bf16x4)));      // to nearest even
            store_as<false>(a.q + 4 * (row + c), quantized(v[i], s));
        }
        if (threadIdx.x == 0) a.scale[t] = s.scale;
    }
}

template <int WAVES, int PER>
int launch_norm(const NormArgs& a, hipStream_t st) {
    const dim3 grid(std::min(a.T, kMostBlocks)), block(64 * WAVES);
    if ((int64_t)a.T * a.vectors * 4 * 13 > kNormFar) hipLaunchKernelGGL((add_rmsnorm_i8_kernel<WAVES, PER, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((add_rmsnorm_i8_kernel<WAVES, PER, false>), grid, block, 0, st, a);
    MOE_HIP_TRY(hipGetLastError());
    return MOE_OK;
}

}  // namespace

namespace moe {

int launch_quantize_i8(int T, int N, const void* x, int x_dtype, int64_t row_elements, int8_t* q, float* scale, bool past, int32_t* words, bool clear, hipStream_t st) {
    if (x_dtype == MOE_DTYPE_F32) return launch_quantize<float, 4>(T, N, (const float*)x, row_elements, q, scale, past, words, clear, st);
    if (N % 8 == 0 && row_elements % 8 == 0 && aligned16(x) && (uintptr_t)q % 8 == 0) return launch_quantize<uint16_t, 8>(T, N, (const uint16_t*)x, row_elements, q, scale, past, words, clear, st);
    return launch_quantize<uint16_t, 4>(T, N, (const uint16_t*)x, row_elements, q, scale, past, words, clear, st);
}

int launch_add_rmsnorm_i8(int T, int H, const float* hidden, const float* delta, const float* gamma, float eps, float* hidden_out, void* x_out, int8_t* q, float* scale,
                          hipStream_t st) {
    const NormArgs a{hidden, delta, gamma, hidden_out, (uint16_t*)x_out, q, scale, eps, T, H / 4};
    if (H <= 256) return launch_norm<1, 1>(a, st);
    if (H <= 1024) return launch_norm<4, 1>(a, st);
    if (H <= 2048) return launch_norm<4, 2>(a, st);
    if (H <= 4096) return launch_norm<8, 2>(a, st);
    if (H <= 6144) return launch_norm<8, 3>(a, st);
    return launch_norm<8, 4>(a, st);
}

bool norm_takes(int32_t H, float eps) { return H > 0 && H % 4 == 0 && H <= kMostH && eps >= 0.f; }

}  // namespace moe

extern "C" {

int moe_quantize_i8(int32_t T, int32_t N, const void* x, int32_t x_dtype, int64_t row_elements, int8_t* x_q, float* x_scale, void* stream) {
    if (x_dtype != MOE_DTYPE_F32 && x_dtype != MOE_DTYPE_BF16) return MOE_ERR_UNSUPPORTED_DTYPE;
    if (T < 0 || N <= 0 || N % 4 != 0 || row_elements < N || row_elements % 4 != 0 || row_elements > INT32_MAX) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    const int64_t esize = x_dtype == MOE_DTYPE_F32 ? 4 : 2, x_bytes = ((T - 1) * row_elements + N) * esize, q_bytes = (int64_t)T * N, s_bytes = (int64_t)T * 4;
    if (!x || !x_q || !x_scale || (uintptr_t)x % (4 * esize) != 0 || (uintptr_t)x_q % 4 != 0 || (uintptr_t)x_scale % 4 != 0) return MOE_ERR_INVALID_ARG;
    if (overlap(x, x_bytes, x_q, q_bytes) || overlap(x, x_bytes, x_scale, s_bytes) || overlap(x_q, q_bytes, x_scale, s_bytes)) return MOE_ERR_INVALID_ARG;
    return launch_quantize_i8(T, N, x, x_dtype, row_elements, x_q, x_scale, false, nullptr, false, (hipStream_t)stream);
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
