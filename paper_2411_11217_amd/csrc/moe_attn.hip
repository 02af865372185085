// Attention of single tokens over a paged key-value cache (moe_attn_decode).
//
//   out = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale q.k_t - m),  m = max_t scale q.k_t
//
// Every key and value is read once and meets n_q / n_kv query heads: 2 (n_q / n_kv) operations per element, so the kernel
// is bound by the bytes of the cache (HBM), and the small calls by latency.  What follows from that:
//
// Split.  A key/value head's rows are cut into tiles of kTile tokens, numbered row by row, and dealt in equal runs to the
// blocks of that head and inside a block to its wavefronts: every wavefront has the same number of tiles (one more or less), whatever the
// lengths are, and streams over them without a barrier, with a running maximum and sum.  A row that one wavefront has to
// itself is written at once; a row of several wavefronts of a block is joined through LDS, one of several blocks through
// the workspace by the block that comes last (a counter per row that is split; the partial results are added in the order of the
// tiles, so which block that is changes no bit).
//   Where a run starts is found by every block itself, from the lengths on the device: a prefix sum over all rows.
//
// Registers instead of LDS.  Keys are the A operand of an MFMA (16 tokens), the up to 16 query heads of the key/value head the
// B operand: lane (r, g) = (lane % 16, lane / 16) loads 16 bytes of token r's row, and gets back the scores of tokens
// 4 g .. 4 g + 3 against head r.  For the second product the lane needs values of exactly these tokens, as A operand one
// element d per MFMA: it loads d-chunk r of each of its four tokens, whole rows per instruction, and the transposition
// into pairs of tokens stays inside the lane (v_perm).  So the weights never leave the lane that computed them, maxima
// cross the four lane groups and nothing else does, and LDS is not used in the loop.
//   bf16: 32 tokens are the 32 steps of one 16x16x32 MFMA.  The weights are split into two bf16 parts, 16 bits of each weight: half
// a bf16 step on the weights would show in the outputs.  f32: 16x16x4 MFMAs, 16 tokens, nothing is rounded.
#include <algorithm>

#include "moe_internal.h"

using namespace moe;

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4, kThreads = kWaves * 64;
constexpr int kMaxRuns = 512;                    // blocks of one head at most: their weights in a join fit 32 KB of LDS

struct AttnArgs {
    const char *q, *k, *v;
    const int32_t *seq_len, *table_row, *block_table;
    char* out;
    float* lse;
    int32_t* counters;
    float* parts;
    int32_t* status;
    uint64_t page_magic;                         // t / P == t * page_magic >> page_shift for 0 <= t < 2^31
    int page_shift;
    int R, n_q, n_kv, group, head_tiles, P, max_pages, table_rows, window, runs;
    uint32_t pool_pages;
    float scale_log2;
};

// Tokens of a tile, and the elements of a vector of 16 bytes.
template <class Elem> struct Kind;
template <> struct Kind<uint16_t> { static constexpr int kTile = 32, kPerDword = 2; };
template <> struct Kind<float> { static constexpr int kTile = 16, kPerDword = 1; };

// ---- rows and their tiles -----------------------------------------------------------
struct Row {
    int len, first, table;                       // tokens first <= t < len are seen; row of the block table
};
__device__ __forceinline__ Row row_of(const AttnArgs& a, int r, int& flags) {
    Row w;
    w.len = max(a.seq_len[r], 0);
    w.table = a.table_row ? a.table_row[r] : r;
    const int most = a.max_pages * a.P;
    if (w.len > most) {
        w.len = most;
        flags |= 1;
    }
    if ((uint32_t)w.table >= (uint32_t)a.table_rows) {
        if (w.table != -1) flags |= 1;
        w.len = 0;
        w.table = 0;
    }
    w.first = a.window ? max(0, w.len - a.window) : 0;
    return w;
}
// A row without tokens has one tile, in which nothing is seen: its zeros are written like any other result.
template <int TILE>
__device__ __forceinline__ int tiles_of(const Row& w) {
    return max(1, (w.len + TILE - 1) / TILE - w.first / TILE);
}

__device__ __forceinline__ int wave_sum_before(int v, int lane, int& total) {
    int incl = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(incl, d, 64);
        if (lane >= d) incl += u;
    }
    total = __builtin_amdgcn_readlane(incl, 63);
    return incl - v;
}

// ---- the two products -------------------------------------------------------------------
__device__ __forceinline__ f32x4 scores(uint16_t, u32x4 k, u32x4 q, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 scores(float, u32x4 k, u32x4 q, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[i]), __uint_as_float(q[i]), c, 0, 0, 0);
    return c;
}

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302); }

__device__ __forceinline__ float max_of_groups(float v) {
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float sum_of_groups(float v) {
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

__device__ __forceinline__ uint32_t pack(uint16_t, float a, float b) { return f32_to_bf16_bits(a) | (f32_to_bf16_bits(b) << 16); }
__device__ __forceinline__ uint32_t pack(float, float a, float) { return __float_as_uint(a); }

// Dwords of a row are dealt to the 16 lanes r as vectors of four (chunk c: dword (c * 16 + r) * 4 ..), and what does not fill
// such a round as shorter ones.  Byte of lane r's dword i.
template <int ND>
__device__ __forceinline__ int dword_at(int r, int i) {
    constexpr int full = ND / 4, rest = ND % 4;
    return i < full * 4 ? (i / 4) * 256 + r * 16 + (i % 4) * 4 : full * 256 + r * (rest * 4) + (i - full * 4) * 4;
}
template <int N> struct Dwords { uint32_t v[N]; };
template <int ND>
__device__ __forceinline__ void load_row(const char* p, int r, uint32_t (&v)[ND]) {
    constexpr int full = ND / 4, rest = ND % 4;
#pragma unroll
    for (int c = 0; c < full; ++c) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(p + c * 256 + r * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[c * 4 + i] = x[i];
    }
    if constexpr (rest > 0) {
        const Dwords<rest> x = *reinterpret_cast<const Dwords<rest>*>(p + full * 256 + r * (rest * 4));
#pragma unroll
        for (int i = 0; i < rest; ++i) v[full * 4 + i] = x.v[i];
    }
}
template <int ND>
__device__ __forceinline__ void store_row(char* p, int r, const uint32_t (&v)[ND]) {
    constexpr int full = ND / 4, rest = ND % 4;
#pragma unroll
    for (int c = 0; c < full; ++c) *reinterpret_cast<u32x4*>(p + c * 256 + r * 16) = u32x4{v[c * 4], v[c * 4 + 1], v[c * 4 + 2], v[c * 4 + 3]};
    if constexpr (rest > 0) {
        Dwords<rest> x;
#pragma unroll
        for (int i = 0; i < rest; ++i) x.v[i] = v[full * 4 + i];
        *reinterpret_cast<Dwords<rest>*>(p + full * 256 + r * (rest * 4)) = x;
    }
}

// A partial result in LDS or in the workspace: f32x4 [E][4 H] (element e of lane (r, g) at e * 4 H + g * H + r, H heads), then
// maxima [H] and sums [H].
constexpr int part_floats(int D, int H) { return H * (D + 2) + (-(H * (D + 2)) & 3); }

// Partial results in the workspace are written by one XCD and read by another in the same launch.  Each XCD has an L2 of its own, and
// a fence that makes plain stores visible writes back, one that makes plain loads current throws away, all of it: with fences
// 256 requests took 707 us, 61 with a window 438.  These go past the L2 instead, as atomic accesses of device
// scope, eight bytes each; what orders them is the wait for the stores before the counter goes up.
__device__ __forceinline__ void put_far(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float get_far(const float* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
struct Halves { uint64_t lo, hi; };
__device__ __forceinline__ void put_far(f32x4* p, f32x4 v) {
    const Halves h = __builtin_bit_cast(Halves, v);
    __hip_atomic_store((uint64_t*)p, h.lo, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store((uint64_t*)p + 1, h.hi, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x4 get_far(const f32x4* p) {
    Halves h;
    h.lo = __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    h.hi = __hip_atomic_load((const uint64_t*)p + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return __builtin_bit_cast(f32x4, h);
}
__device__ __forceinline__ void far_stores_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

struct Split {                                   // a row that a wavefront shares with others
    int row, start, tiles;                       // row -1: none; tiles from `start` on
    int ends;                                    // this part has the row's last tile
};

template <class Elem, int D>
__global__ __launch_bounds__(kThreads) void attn_kernel(const AttnArgs a) {
    constexpr int TILE = Kind<Elem>::kTile, SUB = TILE / 16, EPD = Kind<Elem>::kPerDword;
    constexpr int ROW_BYTES = D * (int)sizeof(Elem), KS = ROW_BYTES / 64, ND = ROW_BYTES / 64, E = D / 16;
    extern __shared__ __align__(16) float s_parts[];         // [wavefront][2] partial results; in the last join its weights
    __shared__ int s_before[kThreads];
    __shared__ int s_sum[kWaves];
    __shared__ Split s_split[kWaves * 2];
    __shared__ Split s_shared[2];                            // rows shared with the blocks before and behind
    __shared__ int s_last[2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int r = lane & 15, g = lane >> 4;
    const int heads_x = a.n_kv * a.head_tiles;
    const int run = blockIdx.x / heads_x, hx = blockIdx.x - run * heads_x;
    const int kv = hx % a.n_kv, tile0 = hx / a.n_kv * 16;    // key/value head, first of its query heads
    const int H = min(a.group - tile0, 16);
    const int head0 = kv * a.group + tile0;
    int flags = 0;

    // ---- which tiles
    const int per = (a.R + kThreads - 1) / kThreads;
    int mine = 0;
    for (int i = threadIdx.x * per; i < min((int)(threadIdx.x + 1) * per, a.R); ++i) mine += tiles_of<TILE>(row_of(a, i, flags));
    if (run != 0 || hx != 0) flags = 0;                      // one block reports
    int wave_total, before = wave_sum_before(mine, lane, wave_total);
    if (lane == 0) s_sum[wave] = wave_total;
    if (lane < 2) s_split[wave * 2 + lane].row = -1;
    if (threadIdx.x < 2) s_shared[threadIdx.x].row = -1;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += s_sum[w];
        total += s_sum[w];
    }
    s_before[threadIdx.x] = before;
    __syncthreads();
    const int share = max((total + a.runs - 1) / a.runs, kWaves);
    const int b0 = min(run * share, total), b1 = min(b0 + share, total);
    if (flags && a.status) atomicOr(a.status, flags);
    if (b0 == b1) return;
    flags = 0;
    const int per_wave = (b1 - b0 + kWaves - 1) / kWaves;
    const int x0 = min(b0 + wave * per_wave, b1), x1 = min(x0 + per_wave, b1);

    if (x0 < x1) {
        // the rows around tile x0: lane i has row base + i
        int below = 0;
#pragma unroll
        for (int j = 0; j < kWaves; ++j) below += __popcll(__ballot(s_before[j * 64 + lane] <= x0));
        int base = (below - 1) * per, start = s_before[below - 1], at;
        Row rows;
        int n_rows;
        auto load_rows = [&]() __attribute__((always_inline)) {
            const int i = base + lane;
            int none = 0;
            rows = row_of(a, min(i, a.R - 1), none);
            n_rows = i < a.R ? tiles_of<TILE>(rows) : 0;
        };
        for (;;) {
            load_rows();
            int sum;
            const int ahead = wave_sum_before(n_rows, lane, sum);
            if (start + sum > x0) {
                at = __ffsll((long long)__ballot(start + ahead + n_rows > x0)) - 1;
                start += __builtin_amdgcn_readlane(ahead, at);
                break;
            }
            start += sum;
            base += 64;
        }
        struct Now {                                         // a row and a tile in it, the same for the whole wavefront
            int row, start, tiles, len, first, table, t0;    // t0: first token of the tile
        };
        auto row_now = [&](int x) __attribute__((always_inline)) {
            Now w;
            w.row = base + at;
            w.start = start;
            w.tiles = __builtin_amdgcn_readlane(n_rows, at);
            w.len = __builtin_amdgcn_readlane(rows.len, at);
            w.first = __builtin_amdgcn_readlane(rows.first, at);
            w.table = __builtin_amdgcn_readlane(rows.table, at);
            w.t0 = (w.first / TILE + x - start) * TILE;
            return w;
        };
        auto next_of = [&](const Now& w, int x) __attribute__((always_inline)) {      // tile x, the one behind w's
            if (x < w.start + w.tiles) {
                Now n = w;
                n.t0 += TILE;
                return n;
            }
            start = w.start + w.tiles;
            if (++at == 64) {
                base += 64;
                at = 0;
                load_rows();
            }
            return row_now(x);
        };
        // Row of the cache (in units of D elements) of token t0 + lane % TILE; tokens that are not seen take the nearest that is.
        auto place = [&](const Now& w) __attribute__((always_inline)) {
            const int t = max(min(w.t0 + (lane & (TILE - 1)), w.len - 1), w.first);
            const int p = (int)(((uint64_t)(uint32_t)t * a.page_magic) >> a.page_shift);
            uint32_t page = (uint32_t)a.block_table[(int64_t)w.table * a.max_pages + p];
            if (page >= a.pool_pages) {
                if (w.len > 0) flags |= 1;
                page = 0;
            }
            return (page * (uint32_t)a.n_kv + (uint32_t)kv) * (uint32_t)a.P + (uint32_t)(t - p * a.P);
        };
        u32x4 kf[SUB][KS], qf[KS];
        uint32_t vf[SUB][4][ND];
        auto load_k = [&](uint32_t where) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                const char* p = a.k + (uint64_t)(uint32_t)__shfl((int)where, u * 16 + r, 64) * ROW_BYTES + g * 16;
#pragma unroll
                for (int s = 0; s < KS; ++s) kf[u][s] = *reinterpret_cast<const u32x4*>(p + s * 64);
            }
        };
        auto load_v = [&](uint32_t where) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) load_row<ND>(a.v + (uint64_t)(uint32_t)__shfl((int)where, u * 16 + g * 4 + i, 64) * ROW_BYTES, r, vf[u][i]);
        };
        auto load_q = [&](int row) __attribute__((always_inline)) {
            const char* p = a.q + ((int64_t)row * a.n_q + head0 + min(r, H - 1)) * ROW_BYTES + g * 16;
#pragma unroll
            for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const u32x4*>(p + s * 64);
        };

        f32x4 acc[E];
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};

        Now now = row_now(x0);
        int from = x0;                                       // the first tile of the current row that is this wavefront's
        {
            const uint32_t where = place(now);
            load_q(now.row);
            load_k(where);
            load_v(where);
        }
        Now nxt = now;
        uint32_t where_nxt = 0;
        if (x0 + 1 < x1) {
            nxt = next_of(now, x0 + 1);
            where_nxt = place(nxt);
        }
        auto tile = [&](int x, auto more_c) __attribute__((always_inline)) {
            constexpr bool more = decltype(more_c)::value;
            f32x4 sc[SUB];
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                sc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < KS; ++s) sc[u] = scores(Elem{}, kf[u][s], qf[s], sc[u]);
            }
            if (more) {
                if (nxt.row != now.row) load_q(nxt.row);
                load_k(where_nxt);
            }
            const bool whole = now.t0 >= now.first && now.t0 + TILE <= now.len;
            float top = -INFINITY;
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = now.t0 + u * 16 + g * 4 + i;
                    const float v = sc[u][i] * a.scale_log2;
                    sc[u][i] = whole || (t >= now.first && t < now.len) ? v : -INFINITY;
                    top = fmaxf(top, sc[u][i]);
                }
            const float m_new = fmaxf(m, max_of_groups(top));
            const float ref = m_new == -INFINITY ? 0.f : m_new;
            if (__any(m_new > m)) {
                const float fade = __builtin_amdgcn_exp2f(m - ref);
                l *= fade;
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] *= fade;
                m = m_new;
            }
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sc[u][i] = __builtin_amdgcn_exp2f(sc[u][i] - ref);
                    l += sc[u][i];
                }
            if (!whole) {                                    // weight 0 times whatever the repeated token holds is not always 0
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int t = now.t0 + u * 16 + g * 4 + i;
                        const bool seen = t >= now.first && t < now.len;
#pragma unroll
                        for (int d = 0; d < ND; ++d) vf[u][i][d] = seen ? vf[u][i][d] : 0;
                    }
            }
            if constexpr (SUB == 2) {
                u32x4 hi, lo;
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        const uint32_t p0 = __float_as_uint(sc[u][i]), p1 = __float_as_uint(sc[u][i + 1]);
                        hi[u * 2 + i / 2] = high_halves(p0, p1);
                        const float r0 = sc[u][i] - __uint_as_float(p0 & 0xffff0000u), r1 = sc[u][i + 1] - __uint_as_float(p1 & 0xffff0000u);
                        lo[u * 2 + i / 2] = high_halves(__float_as_uint(r0), __float_as_uint(r1));
                    }
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    const u32x4 even = {low_halves(vf[0][0][d], vf[0][1][d]), low_halves(vf[0][2][d], vf[0][3][d]),
                                        low_halves(vf[1][0][d], vf[1][1][d]), low_halves(vf[1][2][d], vf[1][3][d])};
                    const u32x4 odd = {high_halves(vf[0][0][d], vf[0][1][d]), high_halves(vf[0][2][d], vf[0][3][d]),
                                       high_halves(vf[1][0][d], vf[1][1][d]), high_halves(vf[1][2][d], vf[1][3][d])};
                    acc[d * 2] = scores(uint16_t{}, even, hi, acc[d * 2]);
                    acc[d * 2 + 1] = scores(uint16_t{}, odd, hi, acc[d * 2 + 1]);
                    acc[d * 2] = scores(uint16_t{}, even, lo, acc[d * 2]);
                    acc[d * 2 + 1] = scores(uint16_t{}, odd, lo, acc[d * 2 + 1]);
                }
            } else {
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[0][i][d]), sc[0][i], acc[d], 0, 0, 0);
            }
            if (more) load_v(where_nxt);
            const bool ends = x + 1 == now.start + now.tiles;
            if (ends || !more) {
                l = sum_of_groups(l);
                const bool begins = from == now.start;
                if (begins && ends) {
                    const float inv = l == 0.f ? 0.f : 1.f / l;
                    if (r < H) {
                        char* out = a.out + ((int64_t)now.row * a.n_q + head0 + r) * ROW_BYTES;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t v[ND];
#pragma unroll
                            for (int d = 0; d < ND; ++d) v[d] = pack(Elem{}, acc[d * EPD][i] * inv, acc[d * EPD + EPD - 1][i] * inv);
                            store_row<ND>(out, g * 4 + i, v);
                        }
                        if (a.lse && g == 0) a.lse[(int64_t)now.row * a.n_q + head0 + r] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
                    }
                } else {
                    const int slot = wave * 2 + (begins ? 1 : 0);
                    float* part = s_parts + slot * part_floats(D, H);
                    if (r < H) {
#pragma unroll
                        for (int e = 0; e < E; ++e) reinterpret_cast<f32x4*>(part)[e * 4 * H + g * H + r] = acc[e];
                        if (g == 0) {
                            part[H * D + r] = m;
                            part[H * D + H + r] = l;
                        }
                    }
                    if (lane == 0) s_split[slot] = Split{now.row, now.start, now.tiles, ends ? 1 : 0};
                }
                m = -INFINITY;
                l = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};
                from = x + 1;
            }
            if (more) {
                now = nxt;
                if (x + 2 < x1) {
                    nxt = next_of(now, x + 2);
                    where_nxt = place(nxt);
                }
            }
        };
        for (int x = x0; x + 1 < x1; ++x) tile(x, std::true_type{});
        tile(x1 - 1, std::false_type{});
    }
    if (flags && a.status) atomicOr(a.status, flags);
    __syncthreads();

    // ---- rows that several wavefronts of the block share
    const int items = ND * 4 * H;                            // (dword d, lane c = g * H + r) of a result
    auto write_item = [&](int item, int row, const f32x4 (&v)[EPD]) __attribute__((always_inline)) {
        const int d = item / (4 * H), c = item - d * 4 * H, gg = c / H, rr = c - gg * H;
        char* out = a.out + ((int64_t)row * a.n_q + head0 + rr) * ROW_BYTES;
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t*>(out + dword_at<ND>(gg * 4 + i, d)) = pack(Elem{}, v[0][i], v[EPD - 1][i]);
    };
    const size_t part_size = part_floats(D, H);
    const size_t part_room = part_floats(D, min(a.group, 16));
    float* const my_parts = a.parts + ((size_t)hx * a.runs + run) * 2 * part_room;
    for (int i0 = 0; i0 < kWaves * 2;) {
        if (s_split[i0].row < 0) {
            ++i0;
            continue;
        }
        const Split first = s_split[i0];
        int i1 = i0 + 1, ends = first.ends;                  // parts i0 .. i1 - 1 are this row's, but for the empty ones
        for (; i1 < kWaves * 2 && (s_split[i1].row < 0 || s_split[i1].row == first.row); ++i1)
            if (s_split[i1].row >= 0) ends = s_split[i1].ends;
        const bool begins = i0 & 1;
        float* const global = my_parts + (begins ? part_room : 0);
        for (int item = threadIdx.x; item < items; item += kThreads) {
            const int d = item / (4 * H), c = item - d * 4 * H, rr = c % H;
            float top = -INFINITY, sum = 0.f;
            for (int k = i0; k < i1; ++k)
                if (s_split[k].row >= 0) top = fmaxf(top, s_parts[k * part_size + H * D + rr]);
            const float ref = top == -INFINITY ? 0.f : top;
            f32x4 v[EPD];
#pragma unroll
            for (int j = 0; j < EPD; ++j) v[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            for (int k = i0; k < i1; ++k) {
                if (s_split[k].row < 0) continue;
                const float* part = s_parts + k * part_size;
                const float w = __builtin_amdgcn_exp2f(part[H * D + rr] - ref);
                sum += w * part[H * D + H + rr];
#pragma unroll
                for (int j = 0; j < EPD; ++j) v[j] += w * reinterpret_cast<const f32x4*>(part)[(d * EPD + j) * 4 * H + c];
            }
            if (begins && ends) {
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
                for (int j = 0; j < EPD; ++j) v[j] *= inv;
                write_item(item, first.row, v);
                if (a.lse && item < H) a.lse[(int64_t)first.row * a.n_q + head0 + rr] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
            } else {
#pragma unroll
                for (int j = 0; j < EPD; ++j) put_far(reinterpret_cast<f32x4*>(global) + (d * EPD + j) * 4 * H + c, v[j]);
                if (item < H) {
                    put_far(global + H * D + rr, top);
                    put_far(global + H * D + H + rr, sum);
                }
            }
        }
        if (!(begins && ends) && threadIdx.x == 0) s_shared[begins ? 1 : 0] = first;
        i0 = i1;
    }

    // ---- rows that several blocks share: the one that comes last joins them
    far_stores_done();
    __syncthreads();
    if (s_shared[0].row < 0 && s_shared[1].row < 0) return;
    int32_t* const counters = a.counters + (size_t)hx * a.runs;
    if (threadIdx.x < 2) {
        const Split w = s_shared[threadIdx.x];
        int last = 0;
        if (w.row >= 0) {
            const int run0 = w.start / share, run1 = (w.start + w.tiles - 1) / share;
            last = atomicAdd(counters + run0, 1) == run1 - run0;
        }
        s_last[threadIdx.x] = last;
    }
    __syncthreads();
    for (int which = 0; which < 2; ++which) {
        if (!s_last[which]) continue;
        const Split w = s_shared[which];
        const int run0 = w.start / share, n = (w.start + w.tiles - 1) / share - run0 + 1;
        const float* const chain = a.parts + ((size_t)hx * a.runs + run0) * 2 * part_room;     // part k: the second slot of run0, the first of the others
        auto part_of = [&](int k) __attribute__((always_inline)) { return chain + (k ? (size_t)k * 2 : 1) * part_room; };
        float* const weight = s_parts;                       // [n][H]
        for (int h = wave; h < H; h += kWaves) {
            float top = -INFINITY, sum = 0.f;
            for (int k = lane; k < n; k += 64) top = fmaxf(top, get_far(part_of(k) + H * D + h));
#pragma unroll
            for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
            const float ref = top == -INFINITY ? 0.f : top;
            for (int k = lane; k < n; k += 64) sum += __builtin_amdgcn_exp2f(get_far(part_of(k) + H * D + h) - ref) * get_far(part_of(k) + H * D + H + h);
#pragma unroll
            for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, 64);
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            for (int k = lane; k < n; k += 64) weight[k * H + h] = __builtin_amdgcn_exp2f(get_far(part_of(k) + H * D + h) - ref) * inv;
            if (a.lse && lane == 0) a.lse[(int64_t)w.row * a.n_q + head0 + h] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
        }
        __syncthreads();
        for (int item = threadIdx.x; item < items; item += kThreads) {
            const int d = item / (4 * H), c = item - d * 4 * H, rr = c % H;
            f32x4 v[EPD];
#pragma unroll
            for (int j = 0; j < EPD; ++j) v[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int k = 0; k < n; ++k)
#pragma unroll
                for (int j = 0; j < EPD; ++j) v[j] += weight[k * H + rr] * get_far(reinterpret_cast<const f32x4*>(part_of(k)) + (d * EPD + j) * 4 * H + c);
            write_item(item, w.row, v);
        }
        if (threadIdx.x == 0) counters[run0] = 0;            // for the next call: nobody else of this one looks at it again
        __syncthreads();
    }
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// The launch: `runs` blocks for each key/value head and 16 of its query heads.
struct Plan {
    int head_tiles, runs;
    size_t parts_bytes, lds_bytes;
};
Plan plan_of(const moe_kv_shape& s, int32_t R) {
    Plan p;
    const int group = s.n_q / s.n_kv, H = std::min(group, 16), tile = s.dtype == MOE_DTYPE_BF16 ? Kind<uint16_t>::kTile : Kind<float>::kTile;
    p.head_tiles = (group + 15) / 16;
    const int64_t heads_x = (int64_t)s.n_kv * p.head_tiles;
    const int64_t tiles = R * (((int64_t)s.max_pages * s.page_tokens + tile - 1) / tile);
    constexpr int kBlocks = 1024;                // four for each of the 256 compute units
    p.runs = (int)std::max<int64_t>(1, std::min<int64_t>({kBlocks / heads_x, (tiles + kWaves - 1) / kWaves, kMaxRuns}));
    const size_t part = (size_t)part_floats(s.head_dim, H) * 4;
    p.parts_bytes = (size_t)heads_x * p.runs * 2 * part;
    p.lds_bytes = std::max((size_t)kWaves * 2 * part, (size_t)p.runs * H * 4);
    return p;
}

int check_rows(const moe_kv_shape* s, int32_t R) {
    int rc = validate_kv(s);
    if (rc != MOE_OK) return rc;
    const int64_t tiles = ((int64_t)s->max_pages * s->page_tokens + 15) / 16;
    return R < 0 || R * tiles > INT32_MAX ? MOE_ERR_INVALID_ARG : MOE_OK;
}

template <class Elem, int D>
int launch(const AttnArgs& a, const Plan& p, hipStream_t st) {
    if (p.lds_bytes > 64 * 1024)
        MOE_HIP_TRY(hipFuncSetAttribute((const void*)attn_kernel<Elem, D>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)p.lds_bytes));
    hipLaunchKernelGGL((attn_kernel<Elem, D>), dim3((uint32_t)p.runs * a.n_kv * p.head_tiles), dim3(kThreads), p.lds_bytes, st, a);
    MOE_HIP_TRY(hipGetLastError());
    return MOE_OK;
}

template <class Elem>
int launch(const AttnArgs& a, const Plan& p, int D, hipStream_t st) {
    switch (D) {
        case 32: return launch<Elem, 32>(a, p, st);
        case 64: return launch<Elem, 64>(a, p, st);
        case 96: return launch<Elem, 96>(a, p, st);
        case 128: return launch<Elem, 128>(a, p, st);
        case 160: return launch<Elem, 160>(a, p, st);
        case 192: return launch<Elem, 192>(a, p, st);
        case 224: return launch<Elem, 224>(a, p, st);
        default: return launch<Elem, 256>(a, p, st);
    }
}

}  // namespace

extern "C" {

int moe_attn_workspace_bytes(const moe_kv_shape* s, int32_t R, size_t* bytes) {
    int rc = check_rows(s, R);
    if (rc != MOE_OK) return rc;
    if (!bytes) return MOE_ERR_INVALID_ARG;
    *bytes = MOE_ATTN_COUNTER_BYTES + plan_of(*s, R).parts_bytes;
    return MOE_OK;
}

int moe_attn_decode(const moe_kv_shape* s, int32_t R, const void* q, const int32_t* seq_len, const int32_t* table_row,
                    const int32_t* block_table, int32_t table_rows, const void* k_cache, const void* v_cache, int32_t window,
                    float scale, void* out, float* lse, void* workspace, size_t workspace_bytes, int32_t* status,
                    void* stream) {
    int rc = check_rows(s, R);
    if (rc != MOE_OK) return rc;
    if (window < 0 || table_rows < 0 || !(scale == scale)) return MOE_ERR_INVALID_ARG;
    if (R == 0) return MOE_OK;
    if (!q || !seq_len || !block_table || !k_cache || !v_cache || !out || !workspace || table_rows < 1 || (!table_row && table_rows < R))
        return MOE_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out) || ((uintptr_t)workspace & 255) != 0) return MOE_ERR_INVALID_ARG;
    const Plan p = plan_of(*s, R);
    if (workspace_bytes < MOE_ATTN_COUNTER_BYTES + p.parts_bytes) return MOE_ERR_WORKSPACE_TOO_SMALL;
    const int64_t esize = s->dtype == MOE_DTYPE_BF16 ? 2 : 4, row_bytes = (int64_t)R * s->n_q * s->head_dim * esize;
    const int64_t cache_bytes = s->pool_pages * s->page_tokens * s->n_kv * s->head_dim * esize;
    if (overlap(out, row_bytes, q, row_bytes) || overlap(out, row_bytes, k_cache, cache_bytes) || overlap(out, row_bytes, v_cache, cache_bytes) ||
        (lse && (overlap(lse, (int64_t)R * s->n_q * 4, out, row_bytes) || overlap(lse, (int64_t)R * s->n_q * 4, q, row_bytes))))
        return MOE_ERR_INVALID_ARG;
    AttnArgs a{};
    a.q = (const char*)q;
    a.k = (const char*)k_cache;
    a.v = (const char*)v_cache;
    a.seq_len = seq_len;
    a.table_row = table_row;
    a.block_table = block_table;
    a.out = (char*)out;
    a.lse = lse;
    a.counters = (int32_t*)workspace;
    a.parts = (float*)((char*)workspace + MOE_ATTN_COUNTER_BYTES);
    a.status = status;
    int bits = 0;
    while (((int64_t)1 << bits) < s->page_tokens) ++bits;
    a.page_shift = 31 + bits;
    a.page_magic = ((uint64_t)1 << a.page_shift) / (uint64_t)s->page_tokens + 1;       // 33 bits at most; the error times 2^31 stays below 2^page_shift
    a.R = R;
    a.n_q = s->n_q;
    a.n_kv = s->n_kv;
    a.group = s->n_q / s->n_kv;
    a.head_tiles = p.head_tiles;
    a.P = s->page_tokens;
    a.max_pages = s->max_pages;
    a.table_rows = table_rows;
    a.window = window;
    a.runs = p.runs;
    a.pool_pages = (uint32_t)s->pool_pages;
    a.scale_log2 = scale * 1.4426950408889634074f;
    return s->dtype == MOE_DTYPE_BF16 ? launch<uint16_t>(a, p, s->head_dim, (hipStream_t)stream) : launch<float>(a, p, s->head_dim, (hipStream_t)stream);
}

}  // extern "C"
