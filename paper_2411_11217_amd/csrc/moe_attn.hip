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
// Products.  Keys are the A operand of an MFMA (16 tokens), the up to 16 query heads of the key/value head the B operand: lane (r, g) =
// (lane % 16, lane / 16) has 16 bytes of token r's row, and gets back the scores of tokens 4 g .. 4 g + 3 against head r.
// For the second product the lane needs values of exactly these tokens, as A operand one element d per MFMA: it loads
// d-chunk r of each of its four tokens, whole rows per instruction, and the transposition into pairs of tokens stays
// inside the lane (v_perm).  So the weights never leave the lane that computed them, and only maxima cross the four lane groups.
//   bf16: 32 tokens are the 32 steps of one 16x16x32 MFMA.  The weights are split into three bf16 parts of 8 bits, all 24 of a float32 weight, so
// nothing is rounded.  A part of 0 would make 0 * infinity of an infinite value, so no part of a weight that is not 0 is 0: the
// first is the largest number of 8 bits below the weight, the second that below what is left, the third the rest (1 to 256
// units of the weight's last place).  f32: 16x16x4 MFMAs, 16 tokens, nothing is rounded either.
//   The matrix cores are busy a third of the time (131001 tokens, 48 heads), so the columns that fewer than 16 heads leave empty cost nothing.
//
// us in a graph, and what of the bytes that is (a load-only kernel reads 6.2 TB/s here, 7.1 with the non-temporal hint; an empty launch takes 2):
// three float32 requests of up to 130 tokens 4.9; 36 requests of 60 to 700 tokens, 32 / 8 heads of 128, 15.7 (2.4 TB/s); 830 rows of six
// prompts 27; one request of 131001 tokens, 48 / 8 heads, 95 (5.6 TB/s); a window of 1000 tokens over 61
// requests, 20 / 20 heads of 96, 78 (5.1 TB/s); 256 requests of 500 to 5000 tokens, 32 / 8 heads, 322 to 334 (6.4 to 6.1 TB/s); in
// float32 128 such requests 322 (6.3 TB/s), one of 131001 tokens, 48 / 8 heads, 183 (5.9 TB/s).
#include <algorithm>
#include <type_traits>

#include "moe_internal.h"
#include "moe_attn_split.h"

using namespace moe;

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4, kThreads = kWaves * 64;

struct AttnArgs {
    const char *q, *k, *v;
    const int32_t *seq_len, *table_row, *block_table;
    char* out;
    float* lse;
    int32_t* counters;
    float* parts;
    int32_t* status;
    uint64_t page_magic;
    int page_shift;
    int R, n_q, n_kv, group, head_tiles, pack, P, max_pages, table_rows, window, runs;
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
    return max(1, (int)(((uint32_t)w.len + TILE - 1) / TILE) - w.first / TILE);
}

// Rows of prompts.  `pack` rows in a row (16 / heads, from a multiple of `pack` on) that see tokens of one request, up to 8 heads each,
// share the 16 columns of the MFMA: their tiles are read once instead of once per row.  A tile that all of them see whole takes one
// pass.  In any other the scores are masked column by column, and the second product is made once for each row, with the tokens that
// this row does not see taken out and the other columns left as they were: a later token's infinity would not be stopped by a
// weight of 0.  Where that costs more than it saves (shared_tiles) the rows stay by themselves.
struct Group {
    int lo, hi, sum;                             // tokens that some row sees; tiles of the rows one by one
    int clear_lo, clear_hi;                      // tokens that all rows see
    bool one;                                    // a full group, one request, tokens everywhere, none that no row sees in between
    // The next row's tokens: they have to touch those of the rows before it, so that no page is followed that no row sees.
    __device__ __forceinline__ void add(int first, int len, int tiles) {
        one = one && first <= hi && len >= lo;
        lo = min(lo, first);
        hi = max(hi, len);
        clear_lo = max(clear_lo, first);
        clear_hi = min(clear_hi, len);
        sum += tiles;
    }
};
template <int TILE>
__device__ __forceinline__ int joint_tiles(const Group& g, int pack) {      // 0: they do not share
    const int n = (int)(((uint32_t)g.hi + TILE - 1) / TILE) - g.lo / TILE;
    const int whole = max(0, g.clear_hi / TILE - (int)(((uint32_t)g.clear_lo + TILE - 1) / TILE));
    return g.one ? shared_tiles(n, whole, pack, g.sum) : 0;
}

// Sum over the lanes before this one, and over all of them, by data-parallel moves.
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_moved(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int wave_sum_before(int v, int& total) {
    int incl = add_moved<0x111, 0xf>(v);         // one lane up in rows of 16, then two, four, eight
    incl = add_moved<0x112, 0xf>(incl);
    incl = add_moved<0x114, 0xf>(incl);
    incl = add_moved<0x118, 0xf>(incl);
    incl = add_moved<0x142, 0xa>(incl);          // the last lane of rows 0 and 2 to rows 1 and 3
    incl = add_moved<0x143, 0xc>(incl);          // of the lower half to the upper
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

// Over the four lanes r, r + 16, r + 32, r + 48, in all of them.
struct Two { float a, b; };
__device__ __forceinline__ Two rows_swapped(float v) {
    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return {__uint_as_float(x[0]), __uint_as_float(x[1])};
}
__device__ __forceinline__ Two halves_swapped(float v) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return {__uint_as_float(x[0]), __uint_as_float(x[1])};
}
__device__ __forceinline__ float max_of_groups(float v) {
    const Two x = rows_swapped(v);
    const Two y = halves_swapped(fmaxf(x.a, x.b));
    return fmaxf(y.a, y.b);
}
__device__ __forceinline__ float sum_of_groups(float v) {
    const Two x = rows_swapped(v);
    const Two y = halves_swapped(x.a + x.b);
    return y.a + y.b;
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack(uint16_t, float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2)); }      // to nearest even
__device__ __forceinline__ uint32_t pack(float, float a, float) { return __float_as_uint(a); }

// Dwords of a row are dealt to the 16 lanes r as vectors of four (chunk c: dword (c * 16 + r) * 4 ..), and what does not fill
// such a round as shorter ones.  Byte of lane r's dword i.
template <int ND>
__device__ __forceinline__ int dword_at(int r, int i) {
    constexpr int full = ND / 4, rest = ND % 4;
    return i < full * 4 ? (i / 4) * 256 + r * 16 + (i % 4) * 4 : full * 256 + r * (rest * 4) + (i - full * 4) * 4;
}
template <int N> struct Dwords { uint32_t v[N]; };
// ONCE: nobody reads this data again, so it need not stay in a cache.
template <bool ONCE>
__device__ __forceinline__ u32x4 load16(const char* p) {
    return ONCE ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)) : *reinterpret_cast<const u32x4*>(p);
}
template <int ND, bool ONCE>
__device__ __forceinline__ void load_row(const char* p, int r, uint32_t (&v)[ND]) {
    constexpr int full = ND / 4, rest = ND % 4;
#pragma unroll
    for (int c = 0; c < full; ++c) {
        const u32x4 x = load16<ONCE>(p + c * 256 + r * 16);
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
// LDS of a wavefront: a partial result (a row that it does not begin), and one (a row that it does not end, its last) in the
// memory of the tile of keys, rows 16 bytes further apart than they are long (an odd number of chunks of 16 bytes: 16 lanes
// that read 16 rows take 16 different banks).
constexpr int key_floats(int D, int esize) { return 64 / esize * (D * esize + 16) / 4; }      // 64 / esize tokens
constexpr int wave_floats(int D, int H, int esize) {
    const int keys = key_floats(D, esize), part = part_floats(D, H);
    return part + (keys > part ? keys : part) + 64 / esize;      // and the places of a tile's tokens in the cache
}

// Partial results in the workspace are written by one XCD and read by another in the same launch.  Each XCD has an L2 of its own, and
// a fence that makes plain stores visible writes back, one that makes plain loads current throws away, all of it: with fences
// 256 requests took 707 us, 61 with a window 438.  So the stores go past the L2, as atomic ones of device scope, eight bytes
// each, and what orders them is the wait for them before the counter goes up.  They are read by plain loads: a launch
// starts without stale lines, and in this one nobody reads the (whole) lines of a part before it is complete.
__device__ __forceinline__ void put_far(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
struct Halves { uint64_t lo, hi; };
__device__ __forceinline__ void put_far(f32x4* p, f32x4 v) {
    const Halves h = __builtin_bit_cast(Halves, v);
    __hip_atomic_store((uint64_t*)p, h.lo, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store((uint64_t*)p + 1, h.hi, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void far_stores_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// In the workspace: [head tile][run][2] parts of whole lines: values, as in LDS but divided by their sum, and [H] weights, the
// logarithms of the sums.
constexpr int far_floats(int D, int H) { return (H * (D + 1) + 63) / 64 * 64; }

// LDS of the last join: a quad and two numbers for each thread, or each quad where these are more.
constexpr int join_floats(int D, int H) { return 6 * (kThreads > D * H / 4 ? kThreads : D * H / 4); }

struct Split {                                   // a row that a wavefront shares with others
    int row, start, tiles;                       // row -1: none; tiles from `start` on
    int cols;                                    // its columns that are results
    int ends;                                    // this part has the row's last tile
};

template <class Elem, int D, bool ONCE, bool PACKED>
__global__ __launch_bounds__(kThreads, D <= 128 ? 2 : 1) void attn_kernel(const AttnArgs a) {
    constexpr int TILE = Kind<Elem>::kTile, SUB = TILE / 16, EPD = Kind<Elem>::kPerDword;
    constexpr int ROW_BYTES = D * (int)sizeof(Elem), KS = ROW_BYTES / 64, ND = ROW_BYTES / 64, E = D / 16;
    constexpr int PITCH = ROW_BYTES + 16, CHUNKS = ROW_BYTES / 16, KN = TILE * CHUNKS / 64;      // of a tile in LDS; chunks of a row, loads of a tile
    // us for 64 requests of 500 to 5000 tokens, 8 key/value heads, bf16, rows one by one / 16 bytes at a time: heads of 64 60 / 55, 96: 82 / 76,
    // 160: 119 / 126 (which takes the registers of a second block).
    constexpr bool BY_ROWS = ROW_BYTES >= 256;
    extern __shared__ __align__(16) float s_parts[];         // of each wavefront wave_floats; in the last join join_floats
    __shared__ int s_before[kThreads];
    __shared__ int s_sum[kWaves];
    __shared__ Split s_split[kWaves * 2];
    __shared__ Split s_shared[2];                            // rows shared with the blocks before and behind
    __shared__ int s_last[2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);      // what is the same for a wavefront stays in scalar registers
    const int r = lane & 15, g = lane >> 4;
    const int heads_x = a.n_kv * a.head_tiles;
    const int run = blockIdx.x / heads_x, hx = blockIdx.x - run * heads_x;
    const int kv = hx % a.n_kv, tile0 = hx / a.n_kv * 16;    // key/value head, first of its query heads
    const int H = PACKED ? a.pack * a.group : min(a.group - tile0, 16);      // columns: query heads, of `pack` rows
    const int col_row = PACKED ? min(r, H - 1) / a.group : 0, col_head = min(r, H - 1) - col_row * a.group;      // of a group that shares them
    const int window_rows = PACKED ? 64 / a.pack * a.pack : 64;
    const int head0 = kv * a.group + tile0;
    int flags = 0;
    const int part_size = part_floats(D, H), wave_size = wave_floats(D, H, (int)sizeof(Elem));
    auto slot_of = [&](int slot) __attribute__((always_inline)) { return s_parts + (slot >> 1) * wave_size + (slot & 1) * part_size; };

    if (lane < 2) s_split[wave * 2 + lane].row = -1;
    if (threadIdx.x < 2) s_shared[threadIdx.x].row = -1;

    // ---- which tiles
    int base = 0, start = 0, at = 0;                         // lane i has row base + i; row base + at is the current one, its first tile is `start`
    Row rows, own;                                           // rows: of a group that shares its columns, what some row sees; own: the lane's row
    int clear_lo, clear_hi;                                  // what all of them see
    int joint;
    int n_rows, ahead, in_rows;                              // tiles of the lane's row (of the group: its first lane's), of the rows before it, of all
    auto load_rows = [&](int& report) __attribute__((always_inline)) {
        const int i = base + lane;
        const bool live = lane < window_rows && i < a.R;
        own = rows = row_of(a, min(i, a.R - 1), report);
        n_rows = live ? tiles_of<TILE>(rows) : 0;
        if constexpr (PACKED) {
            const int lead = lane - lane % a.pack;
            const uint64_t fit = __ballot(live && own.len > 0 && own.table == __shfl(own.table, lead, 64)), all = ((1ull << a.pack) - 1) << lead;
            const int first = __shfl(own.first, lead, 64), len = __shfl(own.len, lead, 64);
            Group grp{first, len, __shfl(n_rows, lead, 64), first, len, live && (fit & all) == all};
            for (int j = 1; j < a.pack; ++j) grp.add(__shfl(own.first, lead + j, 64), __shfl(own.len, lead + j, 64), __shfl(n_rows, lead + j, 64));
            const int shared = joint_tiles<TILE>(grp, a.pack);
            joint = shared > 0;
            if (joint) {
                n_rows = lane == lead ? shared : 0;
                rows.first = grp.lo;
                rows.len = grp.hi;
            }
            clear_lo = joint ? grp.clear_lo : own.first;
            clear_hi = joint ? grp.clear_hi : own.len;
        }
        ahead = wave_sum_before(n_rows, in_rows);
    };
    auto tiles_from = [&](int i) __attribute__((always_inline)) {      // of row i, or of the `pack` rows from i on
        if constexpr (!PACKED) {
            return tiles_of<TILE>(row_of(a, i, flags));
        } else {
            const Row lead = row_of(a, i, flags);
            Group grp{lead.first, lead.len, tiles_of<TILE>(lead), lead.first, lead.len, i + a.pack <= a.R && lead.len > 0};
            for (int j = 1; j < a.pack && i + j < a.R; ++j) {
                const Row w = row_of(a, i + j, flags);
                grp.one = grp.one && w.len > 0 && w.table == lead.table;
                grp.add(w.first, w.len, tiles_of<TILE>(w));
            }
            const int shared = joint_tiles<TILE>(grp, a.pack);
            return shared > 0 ? shared : grp.sum;
        }
    };
    int ignored = 0, total, per = 0;
    if (a.R <= window_rows) {                                // every wavefront has them all
        load_rows(flags);
        total = in_rows;
    } else {
        per = (a.R + kThreads - 1) / kThreads;
        if (PACKED) per = (per + a.pack - 1) / a.pack * a.pack;
        int mine = 0;
        for (int i = threadIdx.x * per; i < min((int)(threadIdx.x + 1) * per, a.R); i += PACKED ? a.pack : 1) mine += tiles_from(i);
        int sum, before = wave_sum_before(mine, sum);
        if (lane == 0) s_sum[wave] = sum;
        __syncthreads();
        total = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) before += s_sum[w];
            total += s_sum[w];
        }
        total = __builtin_amdgcn_readfirstlane(total);
        s_before[threadIdx.x] = before;
        __syncthreads();
    }
    if (run == 0 && hx == 0 && flags && a.status) atomicOr(a.status, flags);      // one block reports
    flags = 0;
    // The row of tile x, 0 <= x < total.
    auto find = [&](int x) __attribute__((always_inline)) {
        int before = 0;
        if (per) {
            int below = 0;
#pragma unroll
            for (int j = 0; j < kWaves; ++j) below += __popcll(__ballot(s_before[j * 64 + lane] <= x));
            base = (below - 1) * per;
            before = __builtin_amdgcn_readfirstlane(s_before[below - 1]);
            for (;; before += in_rows, base += window_rows) {
                load_rows(ignored);
                if (before + in_rows > x || base + window_rows >= a.R) break;
            }
        }
        at = max(__ffsll((long long)__ballot(before + ahead + n_rows > x)) - 1, 0);
        start = before + __builtin_amdgcn_readlane(ahead, at);
    };
    const Runs dealt = deal_tiles(total, a.runs);
    auto bound = [&](int w) __attribute__((always_inline)) {
        const int x = w * dealt.share;
        if (w == 0 || x >= total) return min(x, total);
        find(x);
        return run_end(dealt, x, start, __builtin_amdgcn_readlane(n_rows, at));
    };
    if (run * dealt.share >= total) return;
    const int b0 = bound(run), b1 = bound(run + 1);
    if (b0 == b1) return;
    const int per_wave = (b1 - b0 + kWaves - 1) / kWaves;
    const int x0 = min(b0 + wave * per_wave, b1), x1 = min(x0 + per_wave, b1);

    if (x0 < x1) {
        find(x0);
        struct Now {                                         // a row and a tile in it, the same for the whole wavefront
            int row, start, tiles, len, first, table, t0;    // t0: first token of the tile
            int clear_lo, clear_hi, cols;                    // the rest is PACKED's; of the columns cols are results
            int col_first, col_len;                          // what the lane's column sees
        };
        auto row_now = [&](int x) __attribute__((always_inline)) {
            Now w;
            w.row = min(base + at, a.R - 1);                 // lengths that change during the call (which is not allowed) reach no row that is not there
            w.start = start;
            w.tiles = __builtin_amdgcn_readlane(n_rows, at);
            w.len = __builtin_amdgcn_readlane(rows.len, at);
            w.first = __builtin_amdgcn_readlane(rows.first, at);
            w.table = __builtin_amdgcn_readlane(rows.table, at);
            w.t0 = (w.first / TILE + x - start) * TILE;
            w.clear_lo = w.first;
            w.clear_hi = w.len;
            w.cols = H;
            if constexpr (PACKED) {
                const bool all = __builtin_amdgcn_readlane(joint, at) != 0;
                w.clear_lo = __builtin_amdgcn_readlane(clear_lo, at);
                w.clear_hi = __builtin_amdgcn_readlane(clear_hi, at);
                w.cols = all ? H : a.group;
                w.col_first = __shfl(own.first, at + (all ? col_row : 0), 64);
                w.col_len = __shfl(own.len, at + (all ? col_row : 0), 64);
            }
            return w;
        };
        auto next_of = [&](const Now& w, int x) __attribute__((always_inline)) {      // tile x, the one behind w's
            if (x < w.start + w.tiles) {
                Now n = w;
                n.t0 += TILE;
                return n;
            }
            start = w.start + w.tiles;
            do {                                             // the next row, or group, that has tiles
                if (++at == window_rows) {
                    base += window_rows;
                    at = 0;
                    load_rows(ignored);
                }
            } while (PACKED && base < a.R && __builtin_amdgcn_readlane(n_rows, at) == 0);
            return row_now(x);
        };
        uint32_t* const places = reinterpret_cast<uint32_t*>(s_parts + (wave + 1) * wave_size) - TILE;
        // Rows of the cache (in units of D elements) of the tile's tokens; those that are not seen take the nearest that is.  The lanes
        // read the ones they load from LDS, four at a time (one cross-lane move for each took as long as the rest of the tile).
        auto place = [&](const Now& w) __attribute__((always_inline)) {
            const int t = max(min(w.t0 + (lane & (TILE - 1)), w.len - 1), w.first);
            const int p = divide(t, a.page_magic, a.page_shift);
            uint32_t page = (uint32_t)a.block_table[(int64_t)w.table * a.max_pages + p];
            if (page >= a.pool_pages) {
                if (w.len > 0) flags |= 1;
                page = 0;
            }
            places[lane & (TILE - 1)] = (page * (uint32_t)a.n_kv + (uint32_t)kv) * (uint32_t)a.P + (uint32_t)(t - p * a.P);
        };
        char* const keys = reinterpret_cast<char*>(slot_of(wave * 2 + 1));
        using Held = std::conditional_t<BY_ROWS, uint32_t[TILE / 4][ND], u32x4[KN]>;
        Held kr;
        [[maybe_unused]] Held vr;                            // if not BY_ROWS, until the keys have left the LDS
        u32x4 qf[KS];
        uint32_t vf[SUB][4][ND];                             // of token u * 16 + 4 g + i, the dwords of lane r
        // Keys come as whole cache lines and get to the lanes of the MFMA through the wavefront's own LDS: 16 rows x 64 bytes per load,
        // as the MFMA has them, are half lines, and 256 requests took 4 % longer, a window 12 %.  Where a row has less than 256 bytes, a
        // load takes 64 chunks of 16 bytes in a row, across its rows, of the values too (not BY_ROWS).
        auto load_tile = [&](const char* from, Held& v) __attribute__((always_inline)) {
            if constexpr (BY_ROWS) {
#pragma unroll
                for (int k = 0; k < TILE / 4; ++k) load_row<ND, ONCE>(from + (uint64_t)places[g * (TILE / 4) + k] * ROW_BYTES, r, v[k]);
            } else {
#pragma unroll
                for (int k = 0; k < KN; ++k) {
                    const int i = k * 64 + lane, t = i / CHUNKS;
                    v[k] = load16<ONCE>(from + (uint64_t)places[t] * ROW_BYTES + (i - t * CHUNKS) * 16);
                }
            }
        };
        auto stage_tile = [&](const Held& v) __attribute__((always_inline)) {
            if constexpr (BY_ROWS) {
#pragma unroll
                for (int k = 0; k < TILE / 4; ++k) store_row<ND>(keys + (g * (TILE / 4) + k) * PITCH, r, v[k]);
            } else {
#pragma unroll
                for (int k = 0; k < KN; ++k) {
                    const int i = k * 64 + lane, t = i / CHUNKS;
                    *reinterpret_cast<u32x4*>(keys + t * PITCH + (i - t * CHUNKS) * 16) = v[k];
                }
            }
        };
        auto load_v = [&]() __attribute__((always_inline)) {
            if constexpr (BY_ROWS) {
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) load_row<ND, ONCE>(a.v + (uint64_t)places[u * 16 + g * 4 + i] * ROW_BYTES, r, vf[u][i]);
            } else {
                load_tile(a.v, vr);
            }
        };
        auto load_q = [&](const Now& w) __attribute__((always_inline)) {
            const bool all = PACKED && w.cols > a.group;
            const int row = w.row + (all ? col_row : 0), head = PACKED ? (all ? col_head : min(r, a.group - 1)) : min(r, H - 1);
            const char* p = a.q + ((int64_t)row * a.n_q + head0 + head) * ROW_BYTES + g * 16;
#pragma unroll
            for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const u32x4*>(p + s * 64);
        };

        f32x4 acc[E];
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};

        Now now = row_now(x0);
        int from = x0;                                       // the first tile of the current row that is this wavefront's
        place(now);
        load_q(now);
        load_tile(a.k, kr);
        load_v();
        Now nxt = now;
        if (x0 + 1 < x1) {
            nxt = next_of(now, x0 + 1);
            place(nxt);
        }
        auto tile = [&](int x, auto more_c) __attribute__((always_inline)) {
            constexpr bool more = decltype(more_c)::value;
            stage_tile(kr);
            if (more) load_tile(a.k, kr);
            f32x4 sc[SUB];
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                sc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    sc[u] = scores(Elem{}, *reinterpret_cast<const u32x4*>(keys + (u * 16 + r) * PITCH + s * 64 + g * 16), qf[s], sc[u]);
            }
            if (more && nxt.row != now.row) load_q(nxt);
            const bool whole = now.t0 >= now.clear_lo && now.clear_hi - now.t0 >= TILE;
            const int see_from = PACKED ? now.col_first : now.first, see_to = PACKED ? now.col_len : now.len;
            float top = -INFINITY;
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) sc[u][i] *= a.scale_log2;
            if (!whole) {
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int t = now.t0 + u * 16 + g * 4 + i;
                        if (t < see_from || t >= see_to) sc[u][i] = -INFINITY;
                    }
            }
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[u][i]);
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
            if constexpr (!BY_ROWS) {
                stage_tile(vr);
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) load_row<ND, false>(keys + (u * 16 + g * 4 + i) * PITCH, r, vf[u][i]);
            }
            // Adds the tile's weighted values, of the tokens from `from_t` to `to_t` if not of all, to the columns that are `mine`: weight 0 times
            // whatever a repeated or later token holds is not always 0.
            auto add_values = [&](bool all, int from_t, int to_t, auto some_c, bool mine) __attribute__((always_inline)) {
                constexpr bool some = decltype(some_c)::value;
                uint32_t seen[SUB][4];                       // all bits or none
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int t = now.t0 + u * 16 + g * 4 + i;
                        seen[u][i] = t >= from_t && t < to_t ? ~0u : 0u;
                    }
                if constexpr (SUB == 2) {
                    u32x4 part[3];
                    uint32_t both[4];                        // of two tokens, as their values are paired
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int i = 0; i < 4; i += 2) {
                            float p0 = sc[u][i], p1 = sc[u][i + 1];
#pragma unroll
                            for (int n = 0; n < 3; ++n) {
                                // the largest part below what is left, for the last one what is left: none of a weight's parts is 0, unless the weight is
                                const uint32_t b0 = __builtin_elementwise_sub_sat(__float_as_uint(p0), n < 2 ? 1u : 0u), b1 = __builtin_elementwise_sub_sat(__float_as_uint(p1), n < 2 ? 1u : 0u);
                                part[n][u * 2 + i / 2] = high_halves(b0, b1);
                                p0 -= __uint_as_float(b0 & 0xffff0000u);
                                p1 -= __uint_as_float(b1 & 0xffff0000u);
                            }
                            both[u * 2 + i / 2] = low_halves(seen[u][i], seen[u][i + 1]);
                        }
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        u32x4 even = {low_halves(vf[0][0][d], vf[0][1][d]), low_halves(vf[0][2][d], vf[0][3][d]),
                                      low_halves(vf[1][0][d], vf[1][1][d]), low_halves(vf[1][2][d], vf[1][3][d])};
                        u32x4 odd = {high_halves(vf[0][0][d], vf[0][1][d]), high_halves(vf[0][2][d], vf[0][3][d]),
                                     high_halves(vf[1][0][d], vf[1][1][d]), high_halves(vf[1][2][d], vf[1][3][d])};
                        if (!all)
#pragma unroll
                            for (int n = 0; n < 4; ++n) {
                                even[n] &= both[n];
                                odd[n] &= both[n];
                            }
                        f32x4 x = acc[d * 2], y = acc[d * 2 + 1];
#pragma unroll
                        for (int n = 0; n < 3; ++n) {
                            x = scores(uint16_t{}, even, part[n], x);
                            y = scores(uint16_t{}, odd, part[n], y);
                        }
                        acc[d * 2] = !some || mine ? x : acc[d * 2];
                        acc[d * 2 + 1] = !some || mine ? y : acc[d * 2 + 1];
                    }
                } else {
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        f32x4 x = acc[d];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            x = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(all ? vf[0][i][d] : vf[0][i][d] & seen[0][i]), sc[0][i], x, 0, 0, 0);
                        acc[d] = !some || mine ? x : acc[d];
                    }
                }
            };
            if (PACKED && !whole && now.cols > a.group) {
                for (int j = 0; j < a.pack; ++j)
                    add_values(false, __builtin_amdgcn_readlane(now.col_first, j * a.group), __builtin_amdgcn_readlane(now.col_len, j * a.group), std::true_type{}, col_row == j);
            } else {
                add_values(whole, now.first, now.len, std::false_type{}, true);
            }
            if (more) load_v();
            const bool ends = x + 1 == now.start + now.tiles;
            if (ends || !more) {
                l = sum_of_groups(l);
                const bool begins = from == now.start;
                if (begins && ends) {
                    const float inv = l == 0.f ? 0.f : 1.f / l;
                    if (r < now.cols) {
                        const bool all = PACKED && now.cols > a.group;
                        const int64_t at_row = (int64_t)(now.row + (all ? col_row : 0)) * a.n_q + head0 + (all ? col_head : r);
                        char* out = a.out + at_row * ROW_BYTES;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t v[ND];
#pragma unroll
                            for (int d = 0; d < ND; ++d) v[d] = pack(Elem{}, acc[d * EPD][i] * inv, acc[d * EPD + EPD - 1][i] * inv);
                            store_row<ND>(out, g * 4 + i, v);
                        }
                        if (a.lse && g == 0) a.lse[at_row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
                    }
                } else {
                    const int slot = wave * 2 + (begins ? 1 : 0);
                    float* part = slot_of(slot);
                    int col = r;
                    asm("" : "+v"(col));                     // the addresses are formed here: kept through the loop they would be the registers it lacks
                    if (col < H) {
#pragma unroll
                        for (int e = 0; e < E; ++e) reinterpret_cast<f32x4*>(part)[e * 4 * H + g * H + col] = acc[e];
                        if (g == 0) {
                            part[H * D + col] = m;
                            part[H * D + H + col] = l;
                        }
                    }
                    if (lane == 0) s_split[slot] = Split{now.row, now.start, now.tiles, now.cols, ends ? 1 : 0};
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
                    place(nxt);
                }
            }
        };
        for (int x = x0; x + 1 < x1; ++x) tile(x, std::true_type{});
        tile(x1 - 1, std::false_type{});
    }
    if (flags && a.status) atomicOr(a.status, flags);
    __syncthreads();

    // ---- rows that several wavefronts of the block share.  Lane (r, g) of a wavefront has the values that it had in the loop, every
    // kWaves-th dword of them; the parts of a row are read together (one loop over items, parts after parts, took 3 us of a
    // call of 36 requests).
    auto place_of = [&](int row, int col) __attribute__((always_inline)) {      // of a column's result, among all heads of all rows
        const int further = PACKED ? col / a.group : 0;
        return (int64_t)(row + further) * a.n_q + head0 + col - further * a.group;
    };
    auto write_dword = [&](int row, int col, int group, int d, const f32x4 (&v)[EPD]) __attribute__((always_inline)) {
        char* out = a.out + place_of(row, col) * ROW_BYTES;
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t*>(out + dword_at<ND>(group * 4 + i, d)) = pack(Elem{}, v[0][i], v[EPD - 1][i]);
    };
    const size_t part_room = far_floats(D, PACKED ? H : min(a.group, 16));
    float* const my_parts = a.parts + ((size_t)hx * a.runs + run) * 2 * part_room;
    constexpr int PARTS = kWaves * 2;
    int part_row[PARTS];
#pragma unroll
    for (int k = 0; k < PARTS; ++k) part_row[k] = __builtin_amdgcn_readfirstlane(s_split[k].row);
#pragma unroll
    for (int i0 = 0; i0 < PARTS; ++i0) {
        if (part_row[i0] < 0) continue;
        bool before = false;                                 // the row's first part is not this one
#pragma unroll
        for (int k = 0; k < i0; ++k) before = before || part_row[k] == part_row[i0];
        if (before) continue;
        const int row = part_row[i0], cols = s_split[i0].cols;
        const bool begins = i0 & 1;
        bool ends = false;
        float top = -INFINITY, m_part[PARTS], l_part[PARTS];
#pragma unroll
        for (int k = i0; k < PARTS; ++k) {
            m_part[k] = -INFINITY;
            l_part[k] = 0.f;
            if (part_row[k] != row) continue;
            m_part[k] = slot_of(k)[H * D + min(r, H - 1)];
            l_part[k] = slot_of(k)[H * D + H + min(r, H - 1)];
            ends = s_split[k].ends;                          // the last one says
        }
        ends = __builtin_amdgcn_readfirstlane(ends);
#pragma unroll
        for (int k = i0; k < PARTS; ++k) top = fmaxf(top, m_part[k]);
        const float ref = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int k = i0; k < PARTS; ++k) {
            m_part[k] = __builtin_amdgcn_exp2f(m_part[k] - ref);
            sum += m_part[k] * l_part[k];
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const float log2_sum = sum == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(sum);
        float* const global = my_parts + (begins ? part_room : 0);
        for (int d = wave; d < ND; d += kWaves) {
            f32x4 v[EPD];
#pragma unroll
            for (int j = 0; j < EPD; ++j) v[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = i0; k < PARTS; ++k) {
                if (part_row[k] != row) continue;
#pragma unroll
                for (int j = 0; j < EPD; ++j) v[j] += m_part[k] * reinterpret_cast<const f32x4*>(slot_of(k))[(d * EPD + j) * 4 * H + g * H + min(r, H - 1)];
            }
#pragma unroll
            for (int j = 0; j < EPD; ++j) v[j] *= inv;
            if (r >= H) continue;
            if (begins && ends) {
                if (r < cols) write_dword(row, r, g, d, v);
            } else {                                         // divided by its sum, so that one number says what it weighs
#pragma unroll
                for (int j = 0; j < EPD; ++j) put_far(reinterpret_cast<f32x4*>(global) + (d * EPD + j) * 4 * H + g * H + r, v[j]);
            }
        }
        if (wave == 0 && g == 0 && r < H) {
            if (!(begins && ends)) put_far(global + H * D + r, log2_sum);
            else if (a.lse && r < cols) a.lse[place_of(row, r)] = log2_sum * 0.69314718055994530942f;
        }
        if (!(begins && ends) && threadIdx.x == 0) s_shared[begins ? 1 : 0] = s_split[i0];
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
            int run0;
            const int n = runs_within(dealt, w.start, w.tiles, a.runs, run0);
            last = atomicAdd(counters + run0, 1) == n - 1;
        }
        s_last[threadIdx.x] = last;
    }
    __syncthreads();
    for (int which = 0; which < 2; ++which) {
        if (!s_last[which]) continue;
        const Split w = s_shared[which];
        int run0;
        const int n = runs_within(dealt, w.start, w.tiles, a.runs, run0);
        const float* const chain = a.parts + ((size_t)hx * a.runs + run0) * 2 * part_room;     // part k: the second slot of run0, the first of the others
        auto part_of = [&](int k) __attribute__((always_inline)) { return chain + (k ? (size_t)k * 2 : 1) * part_room; };
        // A thread has four values of every part, or of every second, third, .. where there are threads enough; many are loaded at a
        // time, since each load takes a microsecond.
        constexpr int AT_ONCE = 16;
        const int quads = E * 4 * H, strands = max(1, kThreads / quads);
        f32x4* const sums = reinterpret_cast<f32x4*>(s_parts);          // [strand][quads], then what they weigh: greatest exponent, sum
        float* const weigh = reinterpret_cast<float*>(sums + strands * quads);
        for (int i = threadIdx.x; i < strands * quads; i += kThreads) {
            const int strand = i / quads, quad = i - strand * quads, h = quad % H;
            f32x4 v{0.f, 0.f, 0.f, 0.f};
            float top = -INFINITY, sum = 0.f;
            for (int k0 = strand; k0 < n; k0 += AT_ONCE * strands) {
                f32x4 x[AT_ONCE];
                float e[AT_ONCE], most = top;
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j) {
                    const int k = k0 + j * strands;
                    e[j] = -INFINITY;
                    x[j] = f32x4{0.f, 0.f, 0.f, 0.f};
                    if (k < n) {
                        x[j] = reinterpret_cast<const f32x4*>(part_of(k))[quad];
                        e[j] = part_of(k)[H * D + h];
                    }
                }
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j) most = fmaxf(most, e[j]);
                const float ref = most == -INFINITY ? 0.f : most, fade = __builtin_amdgcn_exp2f(top - ref);
                v *= fade;
                sum *= fade;
                top = most;
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j) {
                    const float p = __builtin_amdgcn_exp2f(e[j] - ref);
                    sum += p;
                    v += p * x[j];
                }
            }
            sums[i] = v;
            weigh[i * 2] = top;
            weigh[i * 2 + 1] = sum;
        }
        __syncthreads();
        for (int item = threadIdx.x; item < ND * 4 * H; item += kThreads) {
            const int d = item / (4 * H), c = item - d * 4 * H, group = c / H;      // dword d of lane (c % H, c / H)
            f32x4 v[EPD];
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int j = 0; j < EPD; ++j) {
                const int quad = (d * EPD + j) * 4 * H + c;
                v[j] = f32x4{0.f, 0.f, 0.f, 0.f};
                top = -INFINITY;
                sum = 0.f;
                for (int k = 0; k < strands; ++k) top = fmaxf(top, weigh[(k * quads + quad) * 2]);
                const float ref = top == -INFINITY ? 0.f : top;
                for (int k = 0; k < strands; ++k) {
                    const float p = __builtin_amdgcn_exp2f(weigh[(k * quads + quad) * 2] - ref);
                    sum += p * weigh[(k * quads + quad) * 2 + 1];
                    v[j] += p * sums[k * quads + quad];
                }
                v[j] *= sum == 0.f ? 0.f : 1.f / sum;
            }
            if (c - group * H < w.cols) write_dword(w.row, c - group * H, group, d, v);
            if (a.lse && item < w.cols) a.lse[place_of(w.row, item)] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
        }
        if (threadIdx.x == 0) counters[run0] = 0;            // for the next call: nobody else of this one looks at it again
        __syncthreads();
    }
}

// The launch: `runs` blocks for each key/value head and 16 of its query heads.
struct Plan {
    int head_tiles, runs, pack;
    size_t parts_bytes, lds_bytes;
};
Plan plan_of(const moe_kv_shape& s, int32_t R, bool prompts) {
    Plan p;
    const int group = s.n_q / s.n_kv;
    p.pack = prompts && group <= 8 ? 16 / group : 1;
    const int H = std::min(group * p.pack, 16), tile = s.dtype == MOE_DTYPE_BF16 ? Kind<uint16_t>::kTile : Kind<float>::kTile;
    p.head_tiles = (group + 15) / 16;
    const int64_t heads_x = (int64_t)s.n_kv * p.head_tiles;
    const int64_t tiles = R * (((int64_t)s.max_pages * s.page_tokens + tile - 1) / tile);
    // Two for each of the 256 compute units, all of them at once.  us with one, two, four, in an earlier build: 256 requests 365 / 347 / 377,
    // 36 requests 20 / 20 / 24, one request of 131001 tokens 102 / 102 / 126, 830 prompt rows 69 / 49 / 58.
    constexpr int kBlocks = 512;
    p.runs = (int)std::max<int64_t>(1, std::min<int64_t>({kBlocks / heads_x, (tiles + kLeastTiles - 1) / kLeastTiles}));
    p.parts_bytes = (size_t)heads_x * p.runs * 2 * far_floats(s.head_dim, H) * 4;
    p.lds_bytes = (size_t)std::max(kWaves * wave_floats(s.head_dim, H, s.dtype == MOE_DTYPE_BF16 ? 2 : 4), join_floats(s.head_dim, H)) * 4;
    return p;
}

int check_rows(const moe_kv_shape* s, int32_t R) {
    int rc = validate_kv(s);
    if (rc != MOE_OK) return rc;
    const int64_t tiles = ((int64_t)s->max_pages * s->page_tokens + 15) / 16;
    return R < 0 || R * tiles >= (int64_t)1 << 30 ? MOE_ERR_INVALID_ARG : MOE_OK;      // tiles are counted in 32 bits, up to a block's share beyond the last
}

template <class Elem, int D, bool ONCE, bool PACKED>
int launch(const AttnArgs& a, const Plan& p, hipStream_t st) {
    const auto kernel = attn_kernel<Elem, D, ONCE, PACKED>;
    if (p.lds_bytes > 64 * 1024) MOE_HIP_TRY(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)p.lds_bytes));
    hipLaunchKernelGGL(kernel, dim3((uint32_t)p.runs * a.n_kv * p.head_tiles), dim3(kThreads), p.lds_bytes, st, a);
    MOE_HIP_TRY(hipGetLastError());
    return MOE_OK;
}

// Rows with a table row of their own and at most 16 query heads to a key/value head read every key and value once: those loads carry
// the non-temporal hint (us without / with: 256 requests 374 / 347, one request of 131001 tokens 114 / 102).  Rows that name their table row
// may be a prompt's, and share columns where there is room for two.  us, each row by itself / sharing, 32 / 8 heads of 128: 830 rows of six
// prompts 43 / 28, 18636 rows of 128 prompts 767 / 359, a prompt of 4000 tokens 1849 / 564, 2468 rows of 200 prompts of 5 to 20 tokens 38 /
// 35; 20 / 20 heads of 96, prompts of 418, 200 and 60 tokens 91 / 43; float32, 8 / 2 heads, 830 rows 36 / 29, 32 / 8 heads, a prompt of 4000 tokens 5665 / 1627.
// Single tokens that name their table row pay for that: 256 requests of 500 to 5000 tokens 370 where they take 321 without, 36 requests 17.4 / 15.7.
template <class Elem, int D>
int launch(const AttnArgs& a, const Plan& p, hipStream_t st) {
    if (p.pack > 1) return launch<Elem, D, false, true>(a, p, st);
    return a.table_row || a.head_tiles > 1 ? launch<Elem, D, false, false>(a, p, st) : launch<Elem, D, true, false>(a, p, st);
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
    *bytes = MOE_ATTN_COUNTER_BYTES + std::max(plan_of(*s, R, false).parts_bytes, plan_of(*s, R, true).parts_bytes);      // with and without table_row
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
    size_t need = 0;
    (void)moe_attn_workspace_bytes(s, R, &need);
    if (workspace_bytes < need) return MOE_ERR_WORKSPACE_TOO_SMALL;
    const Plan p = plan_of(*s, R, table_row != nullptr);
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
    a.page_magic = division_magic(s->page_tokens, a.page_shift);
    a.R = R;
    a.n_q = s->n_q;
    a.n_kv = s->n_kv;
    a.group = s->n_q / s->n_kv;
    a.head_tiles = p.head_tiles;
    a.pack = p.pack;
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
