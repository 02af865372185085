// Attention of single tokens over a paged key-value cache (moe_attn_decode).
#include <algorithm>

#include "moe_internal.h"

using namespace moe;

namespace {

struct AttnArgs {
    const void *q, *k, *v;
    const int32_t *seq_len, *table_row, *block_table;
    void* out;
    float* lse;
    int32_t* status;
    int R, n_q, n_kv, D, P, max_pages, table_rows, window;
    int64_t pool_pages;
    float scale;
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t* p, float v) { *p = (uint16_t)f32_to_bf16_bits(v); }

// One wavefront per row and query head, 64 tokens at a time: a lane has the score of its token, then the sums of the
// elements lane, lane + 64, ..
template <class Elem>
__global__ __launch_bounds__(64) void attn_kernel(const AttnArgs a) {
    const int lane = threadIdx.x, r = blockIdx.x, h = blockIdx.y;
    const int kv = h / (a.n_q / a.n_kv), D = a.D;
    const int row = a.table_row ? a.table_row[r] : r;
    int len = max(a.seq_len[r], 0), flags = 0;
    if (len > a.max_pages * a.P) {
        len = a.max_pages * a.P;
        flags = 1;
    }
    if (row < 0 || row >= a.table_rows) {
        len = 0;
        if (row != -1) flags = 1;
    }
    const int first = a.window ? max(0, len - a.window) : 0;
    const Elem* q = (const Elem*)a.q + ((int64_t)r * a.n_q + h) * D;
    float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int t0 = first; t0 < len; t0 += 64) {
        const int t = min(t0 + lane, len - 1), p = t / a.P;
        int64_t page = a.block_table[(int64_t)row * a.max_pages + p];
        if (page < 0 || page >= a.pool_pages) {
            page = 0;
            flags |= 1;
        }
        const int64_t at = ((page * a.n_kv + kv) * a.P + (t - p * a.P)) * D;
        const Elem* k = (const Elem*)a.k + at;
        float s = 0.f;
        for (int d = 0; d < D; ++d) s = fmaf(to_float(q[d]), to_float(k[d]), s);
        s = t0 + lane < len ? s * a.scale : -INFINITY;
        float top = s;
        for (int x = 32; x >= 1; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
        const float m_new = fmaxf(m, top), ref = m_new == -INFINITY ? 0.f : m_new;
        const float w = expf(s - ref), fade = expf(m - ref);
        m = m_new;
        l = l * fade + w;
        for (float& v : acc) v *= fade;
        for (int j = 0; j < min(64, len - t0); ++j) {
            const Elem* v = (const Elem*)a.v + __shfl(at, j, 64);
            const float wj = __shfl(w, j, 64);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i * 64 + lane < D) acc[i] = fmaf(wj, to_float(v[i * 64 + lane]), acc[i]);
        }
    }
    for (int x = 32; x >= 1; x >>= 1) l += __shfl_xor(l, x, 64);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    Elem* out = (Elem*)a.out + ((int64_t)r * a.n_q + h) * D;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i * 64 + lane < D) put(out + i * 64 + lane, acc[i] * inv);
    if (a.lse && lane == 0) a.lse[(int64_t)r * a.n_q + h] = l == 0.f ? -INFINITY : m + logf(l);
    if (flags && a.status) atomicOr(a.status, flags);
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

int check_rows(const moe_kv_shape* s, int32_t R) {
    int rc = validate_kv(s);
    if (rc != MOE_OK) return rc;
    const int64_t tiles = ((int64_t)s->max_pages * s->page_tokens + 15) / 16;
    return R < 0 || R * tiles > INT32_MAX ? MOE_ERR_INVALID_ARG : MOE_OK;
}

}  // namespace

extern "C" {

int moe_attn_workspace_bytes(const moe_kv_shape* s, int32_t R, size_t* bytes) {
    int rc = check_rows(s, R);
    if (rc != MOE_OK) return rc;
    if (!bytes) return MOE_ERR_INVALID_ARG;
    *bytes = MOE_ATTN_COUNTER_BYTES;
    return MOE_OK;
}

int moe_attn_decode(const moe_kv_shape* s, int32_t R, const void* q, const int32_t* seq_len, const int32_t* table_row,
                    const int32_t* block_table, int32_t table_rows, const void* k_cache, const void* v_cache, int32_t window,
                    float scale, void* out, float* lse, void* workspace, size_t workspace_bytes, int32_t* status,
                    void* stream) {
    size_t need = 0;
    int rc = moe_attn_workspace_bytes(s, R, &need);
    if (rc != MOE_OK) return rc;
    if (window < 0 || table_rows < 0 || !(scale == scale)) return MOE_ERR_INVALID_ARG;
    if (R == 0) return MOE_OK;
    if (!q || !seq_len || !block_table || !k_cache || !v_cache || !out || !workspace || table_rows < 1 || (!table_row && table_rows < R))
        return MOE_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out) || ((uintptr_t)workspace & 255) != 0) return MOE_ERR_INVALID_ARG;
    if (workspace_bytes < need) return MOE_ERR_WORKSPACE_TOO_SMALL;
    const int64_t esize = s->dtype == MOE_DTYPE_BF16 ? 2 : 4, row_bytes = (int64_t)R * s->n_q * s->head_dim * esize;
    const int64_t cache_bytes = s->pool_pages * s->page_tokens * s->n_kv * s->head_dim * esize;
    if (overlap(out, row_bytes, q, row_bytes) || overlap(out, row_bytes, k_cache, cache_bytes) || overlap(out, row_bytes, v_cache, cache_bytes) ||
        (lse && (overlap(lse, (int64_t)R * s->n_q * 4, out, row_bytes) || overlap(lse, (int64_t)R * s->n_q * 4, q, row_bytes))))
        return MOE_ERR_INVALID_ARG;
    const AttnArgs a{q, k_cache, v_cache, seq_len, table_row, block_table, out, lse, status, R, s->n_q, s->n_kv, s->head_dim, s->page_tokens,
                     s->max_pages, table_rows, window, s->pool_pages, scale};
    if (s->dtype == MOE_DTYPE_BF16) hipLaunchKernelGGL(attn_kernel<uint16_t>, dim3(R, s->n_q), dim3(64), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(attn_kernel<float>, dim3(R, s->n_q), dim3(64), 0, (hipStream_t)stream, a);
    MOE_HIP_TRY(hipGetLastError());
    return MOE_OK;
}

}  // extern "C"
