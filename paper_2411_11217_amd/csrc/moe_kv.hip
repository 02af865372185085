// What a step does to a paged key-value cache before its attention: block tables and slot maps (moe_kv_assign), norm and
// rotation of queries and keys with the write of keys and values into the cache (moe_qk_norm_rope).
#include <algorithm>

#include "moe_internal.h"

using namespace moe;

namespace {

// ---- block tables and slot maps ---------------------------------------------------
// Two prefix sums over the requests (rows, new pages), then every row, page and request finds its place by itself.  One
// launch: every block forms both sums from the counts (at most 4096 requests, 32 KB) and serves the rows it strides over;
// a launch for the sums alone would cost more than all of it.
constexpr int kAssignThreads = 256;
constexpr uint32_t kManyRows = 1u << 30;         // sums stop here: nothing that large is ever served

struct AssignArgs {
    const int32_t *cached, *fresh, *free_pages, *free_head;
    int32_t *block_table, *seq_len, *row_start, *positions, *slots, *request, *free_head_out, *status;
    int B, T, P, max_pages, n_free;
    int64_t pool_pages;
};

struct Wants {                                   // what a request asks for
    int cached, held, need;                      // tokens and pages it has, new pages
    bool bad, fits;                              // a negative count; not bad, and rows and pages have room
};
__device__ __forceinline__ uint32_t rows_of(int fresh, int T) { return (uint32_t)min(max(fresh, 0), T + 1); }
__device__ __forceinline__ Wants wants(const AssignArgs& a, int b, uint32_t row) {
    Wants w;
    const int c = a.cached[b], f = a.fresh[b];
    w.bad = c < 0 || f < 0;
    w.cached = max(c, 0);
    w.held = (int)(((int64_t)w.cached + a.P - 1) / a.P);
    const int64_t pages = ((int64_t)w.cached + max(f, 0) + a.P - 1) / a.P;
    w.fits = !w.bad && (uint64_t)row + (uint32_t)f <= (uint32_t)a.T && pages <= a.max_pages;
    w.need = w.fits ? (int)pages - w.held : 0;
    return w;
}
__device__ __forceinline__ uint32_t add_rows(uint32_t x, uint32_t y) { return min(x + y, kManyRows); }

// The sum over the threads before this one, and over all of them.  part: one word per wavefront.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* part, uint32_t& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t incl = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t u = __shfl_up(incl, d, 64);
        if (lane >= d) incl = add_rows(incl, u);
    }
    uint32_t before = __shfl_up(incl, 1, 64);
    if (lane == 0) before = 0;
    __syncthreads();
    if (lane == 63) part[wave] = incl;
    __syncthreads();
    uint32_t run = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kAssignThreads / 64; ++w) {
        if (w < wave) run = add_rows(run, part[w]);
        total = add_rows(total, part[w]);
    }
    return add_rows(run, before);
}

// The last of n ascending sums that is at most v; the first is 0.
__device__ __forceinline__ int last_at_most(const uint32_t* sums, int n, uint32_t v) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] <= v) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(kAssignThreads) void assign_kernel(const AssignArgs a) {
    extern __shared__ uint32_t sums[];           // [B] rows before a request, [B] new pages before it
    __shared__ uint32_t part[kAssignThreads / 64];
    __shared__ uint32_t s_used;
    uint32_t* row0 = sums;
    uint32_t* page0 = sums + a.B;
    const int per = (a.B + kAssignThreads - 1) / kAssignThreads;
    const int b0 = min((int)threadIdx.x * per, a.B), b1 = min(b0 + per, a.B);
    const int head = a.free_head[0];
    const bool head_ok = head >= 0 && head <= a.n_free;
    const uint32_t left = head_ok ? (uint32_t)(a.n_free - head) : 0;
    if (threadIdx.x == 0) s_used = 0;

    uint32_t rows = 0, total_rows, total_pages;
    for (int b = b0; b < b1; ++b) rows = add_rows(rows, rows_of(a.fresh[b], a.T));
    uint32_t row = block_scan(rows, part, total_rows);
    uint32_t pages = 0;
    for (int b = b0; b < b1; ++b) {
        row0[b] = row;
        pages = add_rows(pages, (uint32_t)wants(a, b, row).need);
        row = add_rows(row, rows_of(a.fresh[b], a.T));
    }
    uint32_t page = block_scan(pages, part, total_pages);
    uint32_t used = 0;
    int flags = head_ok ? 0 : 1;
    for (int b = b0; b < b1; ++b) {
        const Wants w = wants(a, b, row0[b]);
        page0[b] = page;
        page = add_rows(page, (uint32_t)w.need);
        const bool served = w.fits && (w.need == 0 || page <= left);
        if (served && w.need) used = page;
        if (!served) flags |= w.bad ? 1 : (uint64_t)row0[b] + (uint32_t)a.fresh[b] > (uint32_t)a.T ? 4 : 2;
    }
    if (used) atomicMax(&s_used, used);
    __syncthreads();

    const uint32_t T = (uint32_t)a.T;
    const uint32_t live = min(total_rows, T);
    const uint32_t n = max(max(T, (uint32_t)a.B + 1), min(total_pages, left));
    for (uint32_t i = blockIdx.x * kAssignThreads + threadIdx.x; i < n; i += gridDim.x * kAssignThreads) {
        if (i < T) {
            int pos = 0, slot = -1, req = -1;
            if (i < live) {
                req = last_at_most(row0, a.B, i);
                const Wants w = wants(a, req, row0[req]);
                pos = (int)min((int64_t)w.cached + (i - row0[req]), (int64_t)INT32_MAX);
                if (w.fits && (w.need == 0 || page0[req] + (uint32_t)w.need <= left)) {
                    const int p = pos / a.P;
                    const int got = p < w.held ? a.block_table[(size_t)req * a.max_pages + p] : a.free_pages[head + (int)page0[req] + p - w.held];
                    if (got >= 0 && got < a.pool_pages) slot = got * a.P + (pos - p * a.P);
                    else flags |= 1;
                }
            }
            a.positions[i] = pos;
            a.slots[i] = slot;
            a.request[i] = req;
        }
        if (i < (uint32_t)a.B) {
            const Wants w = wants(a, i, row0[i]);
            const bool served = w.fits && (w.need == 0 || page0[i] + (uint32_t)w.need <= left);
            a.seq_len[i] = served ? w.cached + a.fresh[i] : w.cached;
            a.row_start[i] = (int)min(row0[i], T);
        } else if (i == (uint32_t)a.B) {
            a.row_start[i] = (int)live;
            a.free_head_out[0] = head + (int)s_used;
        }
        if (i < min(total_pages, left)) {
            const int b = last_at_most(page0, a.B, i);
            const Wants w = wants(a, b, row0[b]);
            if (page0[b] + (uint32_t)w.need <= left) a.block_table[(size_t)b * a.max_pages + w.held + (int)(i - page0[b])] = a.free_pages[head + (int)i];
        }
    }
    if (a.status && flags) atomicOr(a.status, flags);
}

// ---- norm and rotation of queries and keys, the write into the cache --------------------------
// One pass over the rows of the projection: every element is read once and written once, and the kernel is bound by HBM.
// A head is held by LPH lanes (a power of two, head_dim / 8 rounded up), eight elements each as two vectors of four: in the
// part that is rotated by halves the vectors are elements 4 l .. and rot / 2 + 4 l .., the two sides of four pairs, so that a
// rotation needs no other lane; elsewhere they are neighbours.  rot_dim is a multiple of 8, so no lane has both kinds.
// The angle is formed in 64 bits as a number of turns, whose whole part falls away exactly: at position 10^6 a float
// product would be off by 0.03 radians.
constexpr int kRopeWaves = 4;

struct RopeArgs {
    const void* qkv;
    const float *q_gamma, *k_gamma;
    const double* inv_freq;
    const int32_t *positions, *slots;
    void *q, *k_cache, *v_cache;
    int32_t* status;
    int64_t row_elements, pool_tokens;
    float eps;
    int T, n_q, n_kv, D, P, rot, lph;
};

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const uint16_t* p) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    return float4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)};
}
__device__ __forceinline__ void store4(float* p, const float4& v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(uint16_t* p, const float4& v) {
    uint2 o;
    o.x = f32_to_bf16_bits(v.x) | (f32_to_bf16_bits(v.y) << 16);
    o.y = f32_to_bf16_bits(v.z) | (f32_to_bf16_bits(v.w) << 16);
    *reinterpret_cast<uint2*>(p) = o;
}

template <class In, class Out, bool PAIRS>
__global__ __launch_bounds__(kRopeWaves * 64) void qk_norm_rope_kernel(const RopeArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = blockIdx.x;
    const int l = lane & (a.lph - 1), group = lane / a.lph, per_wave = 64 / a.lph;
    const int D = a.D, half = a.rot / 2;
    const bool holds = l * 8 < D;
    const bool turns = l * 8 < a.rot;
    const int o0 = turns && !PAIRS ? 4 * l : 8 * l, o1 = turns && !PAIRS ? half + 4 * l : 8 * l + 4;
    float c[4], s[4];
    const int pos = a.positions[t];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        c[i] = 1.f;
        s[i] = 0.f;
        if (turns) {
            const double n = (double)pos * (a.inv_freq[4 * l + i] * 0.15915494309189533577);
            sincospif(2.0f * (float)(n - rint(n)), &s[i], &c[i]);
        }
    }
    const int64_t slot = a.slots[t];
    const bool keeps = slot >= 0 && slot < a.pool_tokens;
    if (slot != -1 && !keeps && a.status && threadIdx.x == 0) atomicOr(a.status, 1);
    const int64_t page = keeps ? slot / a.P : 0;
    const int place = keeps ? (int)(slot - page * a.P) : 0;

    const int heads = a.n_q + 2 * a.n_kv;
    for (int h0 = wave * per_wave; h0 < heads; h0 += kRopeWaves * per_wave) {      // the same number of rounds for all lanes of a wavefront
        const int h = h0 + group;
        const bool live = holds && h < heads;
        float4 x{0.f, 0.f, 0.f, 0.f}, y{0.f, 0.f, 0.f, 0.f};
        if (live) {
            const In* src = (const In*)a.qkv + (int64_t)t * a.row_elements + (int64_t)h * D;
            x = load4(src + o0);
            y = load4(src + o1);
        }
        const bool is_v = h >= a.n_q + a.n_kv;
        const float* gamma = h < a.n_q ? a.q_gamma : a.k_gamma;
        float sum = x.x * x.x + x.y * x.y + x.z * x.z + x.w * x.w + y.x * y.x + y.y * y.y + y.z * y.z + y.w * y.w;
        for (int m = 1; m < a.lph; m <<= 1) sum += __shfl_xor(sum, m, 64);
        if (!live) continue;
        if (!is_v) {
            if (gamma) {
                const float r = 1.0f / sqrtf(sum / (float)D + a.eps);
                const float4 g0 = load4(gamma + o0), g1 = load4(gamma + o1);
                x = float4{x.x * r * g0.x, x.y * r * g0.y, x.z * r * g0.z, x.w * r * g0.w};
                y = float4{y.x * r * g1.x, y.y * r * g1.y, y.z * r * g1.z, y.w * r * g1.w};
            }
            if (turns) {
                if (PAIRS) {
                    const float4 u = x, v = y;
                    x = float4{u.x * c[0] - u.y * s[0], u.y * c[0] + u.x * s[0], u.z * c[1] - u.w * s[1], u.w * c[1] + u.z * s[1]};
                    y = float4{v.x * c[2] - v.y * s[2], v.y * c[2] + v.x * s[2], v.z * c[3] - v.w * s[3], v.w * c[3] + v.z * s[3]};
                } else {
                    const float4 u = x, v = y;
                    x = float4{u.x * c[0] - v.x * s[0], u.y * c[1] - v.y * s[1], u.z * c[2] - v.z * s[2], u.w * c[3] - v.w * s[3]};
                    y = float4{v.x * c[0] + u.x * s[0], v.y * c[1] + u.y * s[1], v.z * c[2] + u.z * s[2], v.w * c[3] + u.w * s[3]};
                }
            }
        }
        Out* dst;
        if (h < a.n_q) {
            dst = (Out*)a.q + ((int64_t)t * a.n_q + h) * D;
        } else {
            if (!keeps) continue;
            const int kv = is_v ? h - a.n_q - a.n_kv : h - a.n_q;
            dst = (Out*)(is_v ? a.v_cache : a.k_cache) + ((page * a.n_kv + kv) * a.P + place) * D;
        }
        store4(dst + o0, x);
        store4(dst + o1, y);
    }
}

template <class In, class Out>
int launch_rope(const RopeArgs& a, bool pairs, hipStream_t st) {
    if (pairs) hipLaunchKernelGGL((qk_norm_rope_kernel<In, Out, true>), dim3(a.T), dim3(kRopeWaves * 64), 0, st, a);
    else hipLaunchKernelGGL((qk_norm_rope_kernel<In, Out, false>), dim3(a.T), dim3(kRopeWaves * 64), 0, st, a);
    MOE_HIP_TRY(hipGetLastError());
    return MOE_OK;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace

extern "C" {

int moe_kv_assign(const moe_kv_shape* s, int32_t B, int32_t T, const int32_t* cached, const int32_t* fresh,
                  const int32_t* free_pages, int32_t n_free, const int32_t* free_head, int32_t* block_table,
                  int32_t* seq_len, int32_t* row_start, int32_t* positions, int32_t* slots, int32_t* request,
                  int32_t* free_head_out, int32_t* status, void* stream) {
    int rc = validate_kv(s);
    if (rc != MOE_OK) return rc;
    if (B < 0 || B > MOE_MAX_REQUESTS || T < 0 || T >= (int32_t)kManyRows || n_free < 0) return MOE_ERR_INVALID_ARG;
    if (B == 0 && T == 0) return MOE_OK;
    if (!free_head || !free_head_out || !row_start || (n_free > 0 && !free_pages)) return MOE_ERR_INVALID_ARG;
    if (B > 0 && (!cached || !fresh || !block_table || !seq_len)) return MOE_ERR_INVALID_ARG;
    if (T > 0 && (!positions || !slots || !request)) return MOE_ERR_INVALID_ARG;
    const struct { const void* p; int64_t bytes; } in[] = {{cached, (int64_t)B * 4}, {fresh, (int64_t)B * 4}, {free_pages, (int64_t)n_free * 4}, {free_head, 4}},
        out[] = {{seq_len, (int64_t)B * 4}, {row_start, (int64_t)B * 4 + 4}, {positions, (int64_t)T * 4}, {slots, (int64_t)T * 4}, {request, (int64_t)T * 4},
                 {free_head_out, 4}, {block_table, (int64_t)B * s->max_pages * 4}};
    for (const auto& i : in)
        for (const auto& o : out)
            if (i.p && o.p && i.bytes && o.bytes && overlap(i.p, i.bytes, o.p, o.bytes)) return MOE_ERR_INVALID_ARG;
    const AssignArgs a{cached, fresh, free_pages, free_head, block_table, seq_len, row_start, positions, slots, request, free_head_out, status,
                       B, T, s->page_tokens, s->max_pages, n_free, s->pool_pages};
    const int blocks = std::min((std::max(T, B + 1) + kAssignThreads - 1) / kAssignThreads, 1024);
    hipLaunchKernelGGL(assign_kernel, dim3(blocks), dim3(kAssignThreads), (size_t)B * 8, (hipStream_t)stream, a);
    MOE_HIP_TRY(hipGetLastError());
    return MOE_OK;
}

int moe_qk_norm_rope(const moe_kv_shape* s, int32_t T, const void* qkv, int32_t qkv_dtype, int64_t row_elements,
                     const float* q_gamma, const float* k_gamma, float eps, const double* inv_freq, int32_t rot_dim,
                     int32_t pairs, const int32_t* positions, const int32_t* slots, void* q, void* k_cache, void* v_cache,
                     int32_t* status, void* stream) {
    int rc = validate_kv(s);
    if (rc != MOE_OK) return rc;
    if (qkv_dtype != MOE_DTYPE_F32 && qkv_dtype != MOE_DTYPE_BF16) return MOE_ERR_UNSUPPORTED_DTYPE;
    const int64_t esize = qkv_dtype == MOE_DTYPE_F32 ? 4 : 2, out_size = s->dtype == MOE_DTYPE_F32 ? 4 : 2;
    const int64_t width = (int64_t)(s->n_q + 2 * s->n_kv) * s->head_dim;
    if (T < 0 || row_elements < width || row_elements > INT32_MAX || row_elements * esize % 16 != 0) return MOE_ERR_INVALID_ARG;
    if (rot_dim < 0 || rot_dim > s->head_dim || rot_dim % 8 != 0 || !(eps >= 0.f)) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if (!qkv || !positions || !slots || !q || !k_cache || !v_cache || (rot_dim > 0 && !inv_freq)) return MOE_ERR_INVALID_ARG;
    if (!aligned16(qkv) || !aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(q_gamma) || !aligned16(k_gamma))
        return MOE_ERR_INVALID_ARG;
    const int64_t cache_bytes = s->pool_pages * s->page_tokens * s->n_kv * s->head_dim * out_size, in_bytes = T * row_elements * esize;
    const int64_t q_bytes = (int64_t)T * s->n_q * s->head_dim * out_size;
    if (overlap(qkv, in_bytes, q, q_bytes) || overlap(qkv, in_bytes, k_cache, cache_bytes) || overlap(qkv, in_bytes, v_cache, cache_bytes) ||
        overlap(k_cache, cache_bytes, v_cache, cache_bytes) || overlap(q, q_bytes, k_cache, cache_bytes) || overlap(q, q_bytes, v_cache, cache_bytes))
        return MOE_ERR_INVALID_ARG;
    int lph = 4;
    while (lph * 8 < s->head_dim) lph *= 2;
    const RopeArgs a{qkv, q_gamma, k_gamma, inv_freq, positions, slots, q, k_cache, v_cache, status, row_elements, s->pool_pages * s->page_tokens, eps,
                     T, s->n_q, s->n_kv, s->head_dim, s->page_tokens, rot_dim, lph};
    hipStream_t st = (hipStream_t)stream;
    if (qkv_dtype == MOE_DTYPE_F32)
        return s->dtype == MOE_DTYPE_F32 ? launch_rope<float, float>(a, pairs != 0, st) : launch_rope<float, uint16_t>(a, pairs != 0, st);
    return s->dtype == MOE_DTYPE_F32 ? launch_rope<uint16_t, float>(a, pairs != 0, st) : launch_rope<uint16_t, uint16_t>(a, pairs != 0, st);
}

}  // extern "C"
