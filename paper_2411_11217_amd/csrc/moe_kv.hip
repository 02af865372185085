// What a step does to a paged key-value cache before its attention: block tables and slot maps (moe_kv_assign), norm and
// rotation of queries and keys with the write of keys and values into the cache (moe_qk_norm_rope).
#include <algorithm>

#include "moe_internal.h"

using namespace moe;

namespace {

// ---- block tables and slot maps ---------------------------------------------------
// Two prefix sums over the requests (rows, new pages), then every row, page and request finds its place by itself, with a
// search in the sums.  One launch: every block forms both sums from the counts (at most 4096 requests, 32 KB that come from
// the L2) and serves the rows it strides over; a launch for the sums alone would cost more.  A call writes 12 bytes per row; it is bound by
// the latency of its chain (counts, two sums, page, slot; 1024 threads, since the sums' part of it grows with the requests per thread) up to some 100000
// rows.  us in a graph: 36 requests of one token 3.8, 128 prompts of 18600 tokens 6.1, 4000 requests with 529000 rows 16.
constexpr uint32_t kManyRows = 1u << 30;         // sums stop here: nothing that large is ever served
constexpr uint32_t kServed = 1u << 31;           // beside a sum of pages

struct AssignArgs {
    const int32_t *cached, *fresh, *free_pages, *free_head;
    int32_t *block_table, *seq_len, *row_start, *positions, *slots, *request, *free_head_out, *status;
    uint64_t page_magic;
    int page_shift;
    int B, T, P, max_pages, n_free, vectors;     // vectors: positions, slots and request are 16-byte aligned
    uint32_t pool_pages;
};

// Pages of n tokens.
__device__ __forceinline__ int pages_of(const AssignArgs& a, int n) { return n > 0 ? divide(n - 1, a.page_magic, a.page_shift) + 1 : 0; }
__device__ __forceinline__ uint32_t rows_of(int fresh, int T) { return (uint32_t)min(max(fresh, 0), T + 1); }
__device__ __forceinline__ uint32_t add_rows(uint32_t x, uint32_t y) { return min(x + y, kManyRows); }

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t add_moved(uint32_t v) { return add_rows(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false)); }

// The sum over the threads before this one, and over all of them.  part: one word per wavefront.
template <int THREADS>
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* part, uint32_t& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t incl = add_moved<0x111, 0xf>(v);    // one lane up in rows of 16, then two, four, eight, from row to row, from half to half
    incl = add_moved<0x112, 0xf>(incl);
    incl = add_moved<0x114, 0xf>(incl);
    incl = add_moved<0x118, 0xf>(incl);
    incl = add_moved<0x142, 0xa>(incl);
    incl = add_moved<0x143, 0xc>(incl);
    if (lane == 63) part[wave] = incl;
    uint32_t run = __shfl_up(incl, 1, 64);       // saturated sums cannot be taken apart again
    if (lane == 0) run = 0;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) run = add_rows(run, part[w]);
        total = add_rows(total, part[w]);
    }
    return run;
}

// The last of n ascending sums that is at most v; the first is 0.
__device__ __forceinline__ int last_at_most(const uint32_t* sums, int n, uint32_t v) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((sums[mid] & ~kServed) <= v) lo = mid;
        else hi = mid;
    }
    return lo;
}

// PER requests to a thread: B <= THREADS * PER.  ROWS rows to a thread, one search for them.
template <int THREADS, int PER, int ROWS>
__global__ __launch_bounds__(THREADS) void assign_kernel(const AssignArgs a) {
    extern __shared__ uint32_t sums[];           // [B] rows before a request, [B] new pages before it and whether it is served
    __shared__ uint32_t row_part[THREADS / 64], page_part[THREADS / 64], s_used;
    uint32_t* const row0 = sums;
    uint32_t* const page0 = sums + a.B;
    const int b0 = threadIdx.x * PER;
    const uint32_t T = (uint32_t)a.T;
    if (threadIdx.x == 0) s_used = 0;
    const int head = a.free_head[0];
    int cached[PER], fresh[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        cached[j] = b0 + j < a.B ? a.cached[b0 + j] : 0;
        fresh[j] = b0 + j < a.B ? a.fresh[b0 + j] : 0;
    }
    const bool head_ok = head >= 0 && head <= a.n_free;
    const uint32_t left = head_ok ? (uint32_t)(a.n_free - head) : 0;
    int flags = head_ok ? 0 : 1;

    uint32_t rows = 0, pages = 0, total_rows, total_pages, row[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) rows = add_rows(rows, rows_of(fresh[j], a.T));
    rows = block_scan<THREADS>(rows, row_part, total_rows);
    int need[PER];
    bool fits[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        row[j] = rows;
        if (b0 + j < a.B) row0[b0 + j] = rows;
        rows = add_rows(rows, rows_of(fresh[j], a.T));
        const bool bad = cached[j] < 0 || fresh[j] < 0, room = rows <= T;
        // cached + fresh <= max_pages * P < 2^31 where the pages fit
        const bool held = !bad && (uint32_t)cached[j] + (uint32_t)fresh[j] <= (uint32_t)(a.max_pages * a.P);
        fits[j] = held && room;
        need[j] = fits[j] ? pages_of(a, cached[j] + fresh[j]) - pages_of(a, cached[j]) : 0;
        pages = add_rows(pages, (uint32_t)need[j]);
        if (!fits[j]) flags |= bad ? 1 : !room ? 4 : 2;
    }
    pages = block_scan<THREADS>(pages, page_part, total_pages);
    uint32_t used = 0;
    bool served[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const uint32_t before = pages;
        pages = add_rows(pages, (uint32_t)need[j]);
        served[j] = fits[j] && (need[j] == 0 || pages <= left);
        if (served[j] && need[j]) used = pages;
        if (fits[j] && !served[j]) flags |= 2;
        if (b0 + j < a.B) page0[b0 + j] = before | (served[j] ? kServed : 0);
    }
    if (used) atomicMax(&s_used, used);
    if (blockIdx.x == 0) {
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (b0 + j < a.B) {
                a.seq_len[b0 + j] = served[j] ? cached[j] + fresh[j] : max(cached[j], 0);
                a.row_start[b0 + j] = (int)min(row[j], T);
            }
        if (flags && a.status) atomicOr(a.status, flags);
    }
    flags = 0;
    __syncthreads();
    const uint32_t live = min(total_rows, T), n_pages = s_used;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.row_start[a.B] = (int)live;
        a.free_head_out[0] = head + (int)n_pages;
    }

    const uint32_t step = gridDim.x * THREADS, me = blockIdx.x * THREADS + threadIdx.x;
    for (uint32_t i = me; i < n_pages; i += step) {          // all of them are served requests'
        const int b = last_at_most(page0, a.B, i);
        a.block_table[(size_t)b * a.max_pages + pages_of(a, a.cached[b]) + (int)(i - (page0[b] & ~kServed))] = a.free_pages[head + (int)i];
    }
    for (uint32_t i = me * ROWS; i < T; i += step * ROWS) {
        int pos[ROWS], slot[ROWS], req[ROWS];
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            pos[j] = 0;
            slot[j] = req[j] = -1;
        }
        if (i < live) {
            int b = last_at_most(row0, a.B, i), of = -1, last_page = -1, page = -1;
            int had = 0, held = 0;
#pragma unroll
            for (int j = 0; j < ROWS; ++j) {
                if (i + j >= live) continue;
                while (b + 1 < a.B && row0[b + 1] <= i + j) ++b;
                if (b != of) {
                    of = b;
                    had = max(a.cached[b], 0);
                    held = pages_of(a, had);
                    last_page = -1;
                }
                req[j] = b;
                pos[j] = (int)min((int64_t)had + (i + j - row0[b]), (int64_t)INT32_MAX);
                const uint32_t before = page0[b];
                if (before & kServed) {
                    const int p = divide(pos[j], a.page_magic, a.page_shift);
                    if (p != last_page) {
                        last_page = p;
                        page = p < held ? a.block_table[(size_t)b * a.max_pages + p] : a.free_pages[head + (int)(before & ~kServed) + p - held];
                    }
                    if ((uint32_t)page < a.pool_pages) slot[j] = page * a.P + (pos[j] - p * a.P);
                    else flags |= 1;
                }
            }
        }
        if (ROWS == 4 && a.vectors && i + 4 <= T) {
            *reinterpret_cast<int4*>(a.positions + i) = int4{pos[0], pos[1 % ROWS], pos[2 % ROWS], pos[3 % ROWS]};
            *reinterpret_cast<int4*>(a.slots + i) = int4{slot[0], slot[1 % ROWS], slot[2 % ROWS], slot[3 % ROWS]};
            *reinterpret_cast<int4*>(a.request + i) = int4{req[0], req[1 % ROWS], req[2 % ROWS], req[3 % ROWS]};
        } else {
#pragma unroll
            for (int j = 0; j < ROWS; ++j)
                if (i + j < T) {
                    a.positions[i + j] = pos[j];
                    a.slots[i + j] = slot[j];
                    a.request[i + j] = req[j];
                }
        }
    }
    if (a.status && flags) atomicOr(a.status, flags);
}

template <int THREADS, int PER, int ROWS>
int launch_assign(const AssignArgs& a, hipStream_t st) {
    // a block for as many rows as its threads take at once; beyond 2^17 threads (512 blocks of 256, 128 of 1024: half of the compute
    // units) they stride
    const int blocks = (int)std::min<int64_t>(std::max<int64_t>(((int64_t)a.T + ROWS * THREADS - 1) / (ROWS * THREADS), 1), 2 * 256 * 256 / THREADS);
    hipLaunchKernelGGL((assign_kernel<THREADS, PER, ROWS>), dim3(blocks), dim3(THREADS), (size_t)a.B * 8, st, a);
    MOE_HIP_TRY(hipGetLastError());
    return MOE_OK;
}

// Four rows to a thread save searches and stores where there are many; the rows of single tokens are as many requests, and then
// each is a chain of loads of its own.  us in a graph, one row / four: 36 single tokens 3.7 / 5.7, 4000 9.7 / 11.9, 60000 rows of 250 prompts 6.1 / 7.6, 73000 of
// 500 8.5 / 9.9, 150000 of 256 7.4 / 7.5, 200000 of 2000 11.5 / 11.3, 529000 of 4000 19.2 / 16.8.
constexpr int kSingleRows = 1 << 17;
template <int THREADS, int PER>
int launch_assign(const AssignArgs& a, hipStream_t st) {
    return a.T <= kSingleRows ? launch_assign<THREADS, PER, 1>(a, st) : launch_assign<THREADS, PER, 4>(a, st);
}

// ---- norm and rotation of queries and keys, the write into the cache --------------------------
// One pass over the rows of the projection: every element is read once and written once, and the kernel is bound by HBM.
// A head is held by LPH lanes (a power of two, head_dim / 8 rounded up), eight elements each as two vectors of four: in the
// part that is rotated by halves the vectors are elements 4 l .. and rot / 2 + 4 l .., the two sides of four pairs, so that a
// rotation needs no other lane; elsewhere they are neighbours.  rot_dim is a multiple of 8, so no lane has both kinds.
// The angle is formed in 64 bits as a number of turns, whose whole part falls away exactly: at position 10^6 a float
// product would be off by 0.03 radians.  Every wavefront forms the four angles of its lanes once for all of its heads.  9857 rows of 48 + 2 * 8 heads
// of 128, 484 MB: 83 us, where a kernel that only copies such rows, with the same hints, takes 80.5; float32 to float32,
// 646 MB, 115 and 108.5.  256 rows of 32 + 2 * 8 heads 4.4 us, of which 2.9 are the launch.
constexpr int kFewRows = 512;

struct RopeArgs {
    const void* qkv;
    const float *q_gamma, *k_gamma;
    const double* inv_freq;
    const int32_t *positions, *slots;
    void *q, *k_cache, *v_cache;
    int32_t* status;
    int64_t row_elements, pool_tokens;
    uint64_t page_magic;
    int page_shift;
    float eps, per_element;
    int T, n_q, n_kv, D, P, rot, lph;
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

template <bool FAR, class V>
__device__ __forceinline__ V load_as(const void* p) {
    return FAR ? __builtin_nontemporal_load(reinterpret_cast<const V*>(p)) : *reinterpret_cast<const V*>(p);
}
template <bool FAR, class V>
__device__ __forceinline__ void store_as(void* p, V v) {
    if constexpr (FAR) __builtin_nontemporal_store(v, reinterpret_cast<V*>(p));
    else *reinterpret_cast<V*>(p) = v;
}
template <bool FAR>
__device__ __forceinline__ f32x4 load4(const float* p) { return load_as<FAR, f32x4>(p); }
template <bool FAR>
__device__ __forceinline__ f32x4 load4(const uint16_t* p) {
    const u32x2 v = load_as<FAR, u32x2>(p);
    return f32x4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)};
}
template <bool FAR>
__device__ __forceinline__ void store4(float* p, f32x4 v) { store_as<FAR, f32x4>(p, v); }
template <bool FAR>
__device__ __forceinline__ void store4(uint16_t* p, f32x4 v) {
    store_as<FAR, u32x2>(p, __builtin_bit_cast(u32x2, __builtin_convertvector(v, bf16x4)));       // to nearest even
}

// Sine and cosine of `turns` turns.  What is left of a quarter turn, up to 45 degrees either way, is small enough for the first terms of the
// Taylor series: those left out are below 2 10^-9 (sine) and 3 10^-8 (cosine).
__device__ __forceinline__ void sine_cosine(double turns, float& sine, float& cosine) {
    const double quarters = (turns - rint(turns)) * 4.0, whole = rint(quarters);
    const float x = (float)(quarters - whole) * 1.57079632679489661923f, x2 = x * x;
    const float s = fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), x);
    const float c = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 40320, -1.f / 720), 1.f / 24), -0.5f), 1.f);
    const int q = (int)whole;
    const float a = q & 1 ? c : s, b = q & 1 ? s : c;
    sine = __uint_as_float(__float_as_uint(a) ^ ((uint32_t)(q & 2) << 30));
    cosine = __uint_as_float(__float_as_uint(b) ^ ((uint32_t)((q + 1) & 2) << 30));
}

// A block has one row and WAVES wavefronts: with up to 512 rows (two blocks per compute unit) eight, for the latency, with more
// four, and then neither side is kept in the caches (FAR).  us in a graph, 32 + 2 * 8 heads of 128, float32 in, bf16 out: 256 rows with
// eight / four 4.5 / 5.4, 1000 rows 11.2 / 10.7, 9857 rows 80 / 75; with the hint 700 rows 8.8 / 7.3, 5000 rows 43 / 37, 9857 rows 76 / 68.
template <class In, class Out, bool PAIRS, int WAVES, bool FAR>
__global__ __launch_bounds__(WAVES * 64) void qk_norm_rope_kernel(const RopeArgs a) {
    constexpr int AT_ONCE = 2;                               // groups of heads whose loads are under way together
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = blockIdx.x;
    const int l = lane & (a.lph - 1), group = lane / a.lph, per_wave = 64 / a.lph;
    const int D = a.D, half = a.rot / 2;
    const bool holds = l * 8 < D;
    const bool turns = l * 8 < a.rot;
    const int o0 = turns && !PAIRS ? 4 * l : 8 * l, o1 = turns && !PAIRS ? half + 4 * l : 8 * l + 4;
    const int heads = a.n_q + 2 * a.n_kv;
    const In* const row = (const In*)a.qkv + (int64_t)t * a.row_elements;
    const int64_t slot = a.slots[t];
    const int pos = a.positions[t];
    f32x4 c{1.f, 1.f, 1.f, 1.f}, s{0.f, 0.f, 0.f, 0.f};
    bool angles = false;
    const bool keeps = slot >= 0 && slot < a.pool_tokens;
    if (slot != -1 && !keeps && a.status && wave == 0 && lane == 0) atomicOr(a.status, 1);
    const int64_t page = keeps ? divide((int)slot, a.page_magic, a.page_shift) : 0;
    const int place = keeps ? (int)(slot - page * a.P) : 0;

    for (int h0 = wave * per_wave; h0 < heads; h0 += AT_ONCE * WAVES * per_wave) {      // the same number of rounds for all lanes of a wavefront
        f32x4 x[AT_ONCE], y[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int h = h0 + j * WAVES * per_wave + group;
            x[j] = y[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (holds && h < heads) {
                x[j] = load4<FAR>(row + (int64_t)h * D + o0);
                y[j] = load4<FAR>(row + (int64_t)h * D + o1);
            }
        }
        if (!angles) {                                       // once, while the first loads are under way
            angles = true;
            if (turns)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float sine, cosine;
                    sine_cosine((double)pos * (a.inv_freq[4 * l + i] * 0.15915494309189533577), sine, cosine);
                    s[i] = sine;
                    c[i] = cosine;
                }
        }
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int hw = h0 + j * WAVES * per_wave;        // the wavefront's first
            if (hw >= heads) break;
            const int h = hw + group;
            const bool is_v = h >= a.n_q + a.n_kv;
            const float* gamma = h < a.n_q ? a.q_gamma : a.k_gamma;
            f32x4 u = x[j], v = y[j];
            if (a.q_gamma || a.k_gamma) {                    // a sum over the lanes of the head
                const f32x4 uu = u * u, vv = v * v;
                float sum = ((uu.x + uu.y) + (uu.z + uu.w)) + ((vv.x + vv.y) + (vv.z + vv.w));
                for (int m = 1; m < a.lph; m <<= 1) sum += __shfl_xor(sum, m, 64);
                if (gamma && !is_v && holds) {
                    const float r = rsqrtf(fmaf(sum, a.per_element, a.eps));
                    u = u * r * load4<false>(gamma + o0);
                    v = v * r * load4<false>(gamma + o1);
                }
            }
            if (!is_v && turns) {                            // 1 and 0 for sine and cosine would not leave the neighbour of an infinite value alone
                const f32x4 f = u, g = v;
                if (PAIRS) {
                    u = f32x4{f.x * c.x - f.y * s.x, f.y * c.x + f.x * s.x, f.z * c.y - f.w * s.y, f.w * c.y + f.z * s.y};
                    v = f32x4{g.x * c.z - g.y * s.z, g.y * c.z + g.x * s.z, g.z * c.w - g.w * s.w, g.w * c.w + g.z * s.w};
                } else {
                    u = f * c - g * s;
                    v = g * c + f * s;
                }
            }
            if (!holds || h >= heads) continue;
            Out* dst;
            if (h < a.n_q) {
                dst = (Out*)a.q + ((int64_t)t * a.n_q + h) * D;
            } else {
                if (!keeps) continue;
                const int kv = is_v ? h - a.n_q - a.n_kv : h - a.n_q;
                dst = (Out*)(is_v ? a.v_cache : a.k_cache) + ((page * a.n_kv + kv) * a.P + place) * D;
            }
            store4<FAR>(dst + o0, u);
            store4<FAR>(dst + o1, v);
        }
    }
}

template <class In, class Out, int WAVES>
int launch_rope(const RopeArgs& a, bool pairs, hipStream_t st) {
    constexpr bool far = WAVES == 4;
    if (pairs) hipLaunchKernelGGL((qk_norm_rope_kernel<In, Out, true, WAVES, far>), dim3(a.T), dim3(WAVES * 64), 0, st, a);
    else hipLaunchKernelGGL((qk_norm_rope_kernel<In, Out, false, WAVES, far>), dim3(a.T), dim3(WAVES * 64), 0, st, a);
    MOE_HIP_TRY(hipGetLastError());
    return MOE_OK;
}

template <class In, class Out>
int launch_rope(const RopeArgs& all, bool pairs, hipStream_t st) {
    constexpr int kRows = 1 << 23;                           // of a launch: a grid has less than 2^32 threads
    for (int t0 = 0; t0 < all.T; t0 += std::min(kRows, all.T - t0)) {
        RopeArgs a = all;
        a.T = std::min(kRows, all.T - t0);
        a.qkv = (const In*)all.qkv + t0 * all.row_elements;
        a.positions += t0;
        a.slots += t0;
        a.q = (Out*)all.q + (int64_t)t0 * all.n_q * all.D;
        const int rc = a.T <= kFewRows ? launch_rope<In, Out, 8>(a, pairs, st) : launch_rope<In, Out, 4>(a, pairs, st);
        if (rc != MOE_OK) return rc;
    }
    return MOE_OK;
}

}  // namespace

extern "C" {

int moe_kv_assign(const moe_kv_shape* s, int32_t B, int32_t T, const int32_t* cached, const int32_t* fresh,
                  const int32_t* free_pages, int32_t n_free, const int32_t* free_head, int32_t* block_table,
                  int32_t* seq_len, int32_t* row_start, int32_t* positions, int32_t* slots, int32_t* request,
                  int32_t* free_head_out, int32_t* status, void* stream) {
    int rc = validate_kv(s);
    if (rc != MOE_OK) return rc;
    if (B < 0 || B > MOE_MAX_REQUESTS || T < 0 || T >= (int32_t)kManyRows || n_free < 0) return MOE_ERR_INVALID_ARG;
    if (B == 0 && T == 0 && (!free_head || !free_head_out || !row_start)) return MOE_OK;         // nothing to hand on
    if (!free_head || !free_head_out || !row_start || (n_free > 0 && !free_pages)) return MOE_ERR_INVALID_ARG;
    if (B > 0 && (!cached || !fresh || !block_table || !seq_len)) return MOE_ERR_INVALID_ARG;
    if (T > 0 && (!positions || !slots || !request)) return MOE_ERR_INVALID_ARG;
    const struct { const void* p; int64_t bytes; } in[] = {{cached, (int64_t)B * 4}, {fresh, (int64_t)B * 4}, {free_pages, (int64_t)n_free * 4}, {free_head, 4}},
        out[] = {{seq_len, (int64_t)B * 4}, {row_start, (int64_t)B * 4 + 4}, {positions, (int64_t)T * 4}, {slots, (int64_t)T * 4}, {request, (int64_t)T * 4},
                 {free_head_out, 4}, {block_table, (int64_t)B * s->max_pages * 4}};
    for (const auto& i : in)
        for (const auto& o : out)
            if (i.p && o.p && i.bytes && o.bytes && overlap(i.p, i.bytes, o.p, o.bytes)) return MOE_ERR_INVALID_ARG;
    AssignArgs a{};
    a.cached = cached;
    a.fresh = fresh;
    a.free_pages = free_pages;
    a.free_head = free_head;
    a.block_table = block_table;
    a.seq_len = seq_len;
    a.row_start = row_start;
    a.positions = positions;
    a.slots = slots;
    a.request = request;
    a.free_head_out = free_head_out;
    a.status = status;
    a.page_magic = division_magic(s->page_tokens, a.page_shift);
    a.B = B;
    a.T = T;
    a.P = s->page_tokens;
    a.max_pages = s->max_pages;
    a.n_free = n_free;
    a.vectors = aligned16(positions) && aligned16(slots) && aligned16(request);
    a.pool_pages = (uint32_t)s->pool_pages;
    return B <= 256 ? launch_assign<256, 1>(a, (hipStream_t)stream) : launch_assign<1024, 4>(a, (hipStream_t)stream);
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
    RopeArgs a{};
    a.qkv = qkv;
    a.q_gamma = q_gamma;
    a.k_gamma = k_gamma;
    a.inv_freq = inv_freq;
    a.positions = positions;
    a.slots = slots;
    a.q = q;
    a.k_cache = k_cache;
    a.v_cache = v_cache;
    a.status = status;
    a.row_elements = row_elements;
    a.pool_tokens = s->pool_pages * s->page_tokens;
    a.page_magic = division_magic(s->page_tokens, a.page_shift);
    a.eps = eps;
    a.per_element = 1.f / (float)s->head_dim;
    a.T = T;
    a.n_q = s->n_q;
    a.n_kv = s->n_kv;
    a.D = s->head_dim;
    a.P = s->page_tokens;
    a.rot = rot_dim;
    a.lph = lph;
    hipStream_t st = (hipStream_t)stream;
    if (qkv_dtype == MOE_DTYPE_F32)
        return s->dtype == MOE_DTYPE_F32 ? launch_rope<float, float>(a, pairs != 0, st) : launch_rope<float, uint16_t>(a, pairs != 0, st);
    return s->dtype == MOE_DTYPE_F32 ? launch_rope<uint16_t, float>(a, pairs != 0, st) : launch_rope<uint16_t, uint16_t>(a, pairs != 0, st);
}

}  // extern "C"
