// Entry points of the layer in 8-bit integers and of its dense neighbours: argument checks, and the tasks as sequences of launches.
#include <algorithm>

#include "moe_internal.h"

using namespace moe;

namespace {

bool has_scales(const moe_expert_scales* s) { return s && s->w1 && s->w3 && s->w2; }

int check_linear(const moe_linear_shape* s) {
    const int rc = validate_linear(s);
    if (rc != MOE_OK) return rc;
    return s->dtype == MOE_DTYPE_I8 ? MOE_OK : MOE_ERR_UNSUPPORTED_DTYPE;
}

int check_layer(const moe_shape* s) {
    const int rc = validate_shape(s);
    if (rc != MOE_OK) return rc;
    if (s->dtype != MOE_DTYPE_I8) return MOE_ERR_UNSUPPORTED_DTYPE;
    return (int64_t)s->T * s->H < ((int64_t)1 << 32) ? MOE_OK : MOE_ERR_INVALID_ARG;        // rows are found by 32-bit offsets
}

int enqueue_linear(const moe_linear_shape& s, const int8_t* x_q, const float* x_scale, const int32_t* table, const void* pool, int64_t pool_pages, const float* w_scale,
                   float* out, int32_t* status, hipStream_t st) {
    const LinearI8Args a{x_q, x_scale, s.T, s.K, s.N, table, (const char*)pool, pool_pages, s.page_bytes, linear_pages(s), w_scale, out, status};
    return launch_linear_i8(a, st);
}

moe_shape routed(const moe_shape& s) {          // the shape for router and permutation, whose activations are bf16
    moe_shape r = s;
    r.dtype = MOE_DTYPE_BF16;
    return r;
}

// Byte offsets into the workspace of the layer, 256-byte aligned.
struct Layout {
    size_t status, ids, w, counts, offsets, row_src, row_of, row_w, scan, h, h_q, h_scale, out, total;
};
Layout layout(const moe_shape& s) {
    const size_t R = (size_t)s.T * s.k;
    Layout L;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t o = off;
        off = (off + std::max<size_t>(bytes, 4) + 255) / 256 * 256;
        return o;
    };
    L.status = take(16);
    L.ids = take(R * 4);
    L.w = take(R * 4);
    L.counts = take((size_t)s.E * 4);
    L.offsets = take((size_t)(s.E + 1) * 4);
    L.row_src = take(R * 4);
    L.row_of = take(R * 4);
    L.row_w = take(R * 4);
    L.scan = take(permute_workspace_bytes(routed(s)));
    L.h = take(R * s.F * 2);
    L.h_q = take(R * s.F);
    L.h_scale = take(R * 4);
    L.out = take(R * s.H * 2);
    L.total = off;
    return L;
}

int enqueue_layer(const moe_shape& s, const void* x, const int8_t* x_q, const float* x_scale, const void* Wr, const float* bias, const int32_t* page_table,
                  const void* pool, int64_t pool_pages, const moe_expert_scales& scales, float* y, char* ws, hipStream_t st, const int32_t* found = nullptr) {
    const Layout L = layout(s);
    const moe_shape r = routed(s);
    int32_t *status = (int32_t*)(ws + L.status), *ids = (int32_t*)(ws + L.ids), *offsets = (int32_t*)(ws + L.offsets), *row_src = (int32_t*)(ws + L.row_src),
            *row_of = (int32_t*)(ws + L.row_of);
    float *w = (float*)(ws + L.w), *row_w = (float*)(ws + L.row_w);
    // the status words are cleared by the router or the permutation
    const PlaceOut place{(int32_t*)(ws + L.counts), offsets, row_src, row_of, row_w, status};
    const bool places = route_places(r);
    int rc = launch_route(r, x, Wr, bias, ids, w, nullptr, st, places ? &place : nullptr);
    if (rc != MOE_OK) return rc;
    if (!places) {
        rc = launch_permute(r, ids, w, nullptr, place.counts, offsets, row_src, row_of, row_w, nullptr, ws + L.scan, status, st);
        if (rc != MOE_OK) return rc;
    }
    const FfnI8Args a{x_q, x_scale, row_src, offsets, page_table, (const char*)pool, pool_pages, scales, row_w, ws + L.h, (int8_t*)(ws + L.h_q), (float*)(ws + L.h_scale),
                      ws + L.out, status};
    rc = launch_expert_ffn_i8(s, a, st);
    if (rc != MOE_OK) return rc;
    return launch_combine(s, ws + L.out, row_of, nullptr, y, st, found, status);
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// [the layer's workspace][attn in 8 bits][its scales][O projection, float [T][H]][x_moe in 8 bits][its scales][the O projection's status words]
struct PostLayout {
    size_t a_q, a_scale, o, x_q, x_scale, found, total;
};
PostLayout post_layout(const moe_shape& s, int32_t K) {
    PostLayout L;
    const size_t T = (size_t)s.T;
    L.a_q = up256(layout(s).total);
    L.a_scale = L.a_q + up256(T * K);
    L.o = L.a_scale + up256(T * 4);
    L.x_q = L.o + up256(T * s.H * 4);
    L.x_scale = L.x_q + up256(T * s.H);
    L.found = L.x_scale + up256(T * 4);
    L.total = L.found + 256;
    return L;
}

}  // namespace

extern "C" {

int moe_linear_i8(const moe_linear_shape* s, const int8_t* x_q, const float* x_scale, const int32_t* page_table, const void* page_pool, int64_t pool_pages,
                  const float* w_scale, float* out, int32_t* status, void* stream) {
    const int rc = check_linear(s);
    if (rc != MOE_OK) return rc;
    if (s->T == 0) return MOE_OK;
    if (!x_q || !x_scale || !page_table || !page_pool || !w_scale || !out || pool_pages <= 0 || !aligned16(x_q) || !aligned16(page_pool)) return MOE_ERR_INVALID_ARG;
    const int64_t T = s->T;
    if (overlap(x_q, T * s->K, out, T * s->N * 4) || overlap(x_scale, T * 4, out, T * s->N * 4)) return MOE_ERR_INVALID_ARG;
    return enqueue_linear(*s, x_q, x_scale, page_table, page_pool, pool_pages, w_scale, out, status, (hipStream_t)stream);
}

int moe_expert_ffn_i8(const moe_shape* s, const int8_t* x_q, const float* x_scale, const int32_t* row_src, const int32_t* offsets, const int32_t* page_table,
                      const void* page_pool, int64_t pool_pages, const moe_expert_scales* scales, const float* row_w, void* h, int8_t* h_q, float* h_scale, void* out,
                      int32_t* status, void* stream) {
    const int rc = check_layer(s);
    if (rc != MOE_OK) return rc;
    if (s->T == 0) return MOE_OK;
    if (!x_q || !x_scale || !offsets || !page_table || !page_pool || !has_scales(scales) || !h || !h_q || !h_scale || !out || pool_pages <= 0) return MOE_ERR_INVALID_ARG;
    if (!aligned16(x_q) || !aligned16(page_pool) || !aligned16(h) || !aligned16(h_q) || !aligned16(out)) return MOE_ERR_INVALID_ARG;
    const int64_t R = (int64_t)s->T * s->k, x_rows = row_src ? s->T : R;
    const struct { const void* p; int64_t bytes; } buf[] = {{h, R * s->F * 2}, {h_q, R * s->F}, {h_scale, R * 4}, {out, R * s->H * 2}, {x_q, x_rows * s->H}, {x_scale, x_rows * 4}};
    for (int i = 0; i < 4; ++i)                 // what is written, against everything
        for (int j = i + 1; j < 6; ++j)
            if (overlap(buf[i].p, buf[i].bytes, buf[j].p, buf[j].bytes)) return MOE_ERR_INVALID_ARG;
    const FfnI8Args a{x_q, x_scale, row_src, offsets, page_table, (const char*)page_pool, pool_pages, *scales, row_w, h, h_q, h_scale, out, status};
    return launch_expert_ffn_i8(*s, a, (hipStream_t)stream);
}

int moe_layer_i8_workspace_bytes(const moe_shape* s, size_t* bytes) {
    const int rc = check_layer(s);
    if (rc != MOE_OK) return rc;
    if (!bytes) return MOE_ERR_INVALID_ARG;
    *bytes = layout(*s).total;
    return MOE_OK;
}

int moe_layer_i8(const moe_shape* s, const void* x, const int8_t* x_q, const float* x_scale, const void* Wr, const float* bias, const int32_t* page_table,
                 const void* page_pool, int64_t pool_pages, const moe_expert_scales* scales, float* y, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_layer(s);
    if (rc != MOE_OK) return rc;
    if (s->T == 0) return MOE_OK;
    if (!x || !x_q || !x_scale || !Wr || !page_table || !page_pool || !has_scales(scales) || !y || !workspace || pool_pages <= 0) return MOE_ERR_INVALID_ARG;
    if (!aligned16(x_q) || !aligned16(page_pool) || ((uintptr_t)workspace & 255) != 0) return MOE_ERR_INVALID_ARG;
    if (workspace_bytes < layout(*s).total) return MOE_ERR_WORKSPACE_TOO_SMALL;
    return enqueue_layer(*s, x, x_q, x_scale, Wr, bias, page_table, page_pool, pool_pages, *scales, y, (char*)workspace, (hipStream_t)stream);
}

int moe_pre_attention_i8(const moe_linear_shape* qkv_proj, const float* hidden, const float* delta, const float* norm_gamma, float eps, const int32_t* qkv_table,
                         const void* page_pool, int64_t pool_pages, const float* qkv_scale, float* hidden_out, int8_t* x_q, float* x_scale, float* qkv, int32_t* status,
                         void* stream) {
    int rc = check_linear(qkv_proj);
    if (rc != MOE_OK) return rc;
    if (!norm_takes(qkv_proj->K, eps)) return MOE_ERR_INVALID_ARG;
    if (qkv_proj->T == 0) return MOE_OK;
    if (!qkv_table || !page_pool || !qkv_scale || !hidden_out || !qkv || pool_pages <= 0 || !aligned16(x_q) || !aligned16(page_pool)) return MOE_ERR_INVALID_ARG;
    const int64_t T = qkv_proj->T, K = qkv_proj->K, out_bytes = T * qkv_proj->N * 4;
    if (x_q && x_scale && (overlap(x_q, T * K, qkv, out_bytes) || overlap(x_scale, T * 4, qkv, out_bytes) || overlap(hidden_out, T * K * 4, qkv, out_bytes))) return MOE_ERR_INVALID_ARG;
    rc = moe_add_rmsnorm_i8(qkv_proj->T, qkv_proj->K, hidden, delta, norm_gamma, eps, hidden_out, nullptr, x_q, x_scale, stream);
    if (rc != MOE_OK) return rc;
    return enqueue_linear(*qkv_proj, x_q, x_scale, qkv_table, page_pool, pool_pages, qkv_scale, qkv, status, (hipStream_t)stream);
}

int moe_post_attention_i8_workspace_bytes(const moe_shape* s, const moe_linear_shape* o_proj, size_t* bytes) {
    int rc = check_layer(s);
    if (rc != MOE_OK) return rc;
    rc = check_linear(o_proj);
    if (rc != MOE_OK) return rc;
    if (!bytes || o_proj->T != s->T) return MOE_ERR_INVALID_ARG;
    *bytes = post_layout(*s, o_proj->K).total;
    return MOE_OK;
}

int moe_post_attention_i8(const moe_shape* s, const moe_linear_shape* o_proj, const void* attn, const float* hidden, const int32_t* o_table, const float* o_scale,
                          const float* norm_gamma, float eps, const void* Wr, const float* bias, const int32_t* page_table, const void* page_pool, int64_t pool_pages,
                          const moe_expert_scales* scales, float* hidden_mid, void* x_moe, float* y, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_layer(s);
    if (rc != MOE_OK) return rc;
    rc = check_linear(o_proj);
    if (rc != MOE_OK) return rc;
    if (o_proj->T != s->T || o_proj->N != s->H || o_proj->page_bytes != s->page_bytes || !norm_takes(s->H, eps)) return MOE_ERR_INVALID_ARG;
    if (s->T == 0) return MOE_OK;
    if (!attn || !hidden || !o_table || !o_scale || !norm_gamma || !Wr || !page_table || !page_pool || !has_scales(scales) || !hidden_mid || !x_moe || !y || !workspace ||
        pool_pages <= 0)
        return MOE_ERR_INVALID_ARG;
    if ((uintptr_t)attn % 8 != 0 || !aligned16(hidden) || !aligned16(norm_gamma) || !aligned16(hidden_mid) || !aligned16(x_moe) || !aligned16(page_pool) ||
        ((uintptr_t)workspace & 255) != 0)
        return MOE_ERR_INVALID_ARG;
    const PostLayout L = post_layout(*s, o_proj->K);
    if (workspace_bytes < L.total) return MOE_ERR_WORKSPACE_TOO_SMALL;
    hipStream_t st = (hipStream_t)stream;
    char* ws = (char*)workspace;
    int8_t *a_q = (int8_t*)(ws + L.a_q), *x_q = (int8_t*)(ws + L.x_q);
    float *a_scale = (float*)(ws + L.a_scale), *x_scale = (float*)(ws + L.x_scale), *o = (float*)(ws + L.o);
    // The router clears the layer's status words behind the O projection, which therefore has its own: cleared with attn's rows, joined to the others by the combine.
    int32_t* const found = (int32_t*)(ws + L.found);
    rc = launch_quantize_i8(s->T, o_proj->K, attn, MOE_DTYPE_BF16, o_proj->K, a_q, a_scale, false, found, true, st);
    if (rc != MOE_OK) return rc;
    rc = enqueue_linear(*o_proj, a_q, a_scale, o_table, page_pool, pool_pages, o_scale, o, found, st);
    if (rc != MOE_OK) return rc;
    rc = launch_add_rmsnorm_i8(s->T, s->H, hidden, o, norm_gamma, eps, hidden_mid, x_moe, x_q, x_scale, st);
    if (rc != MOE_OK) return rc;
    return enqueue_layer(*s, x_moe, x_q, x_scale, Wr, bias, page_table, page_pool, pool_pages, *scales, y, ws, st, found);
}

}  // extern "C"
