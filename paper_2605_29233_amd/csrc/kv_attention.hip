// Softmax attention on rows of 16-bit heads: packed sequences (bb_attention), and branches over a prefix that they share and pages of their own
// (bb_shared_attention).
//
//   out[i] = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(scale q_i k_j - m_i),  j over the keys that query i sees, m_i their largest score
//
// in one pass over the keys: running maximum, sum and output (online softmax), all fp32, the output rounded once.  The query heads that share a kv head are
// folded into the rows (row = token * each + head of the group), so a tile of K and V serves them all.
//
// Matrix instructions (32x32x16, 16-bit operands, fp32 sums), transposed so that a lane keeps to one row:
//   S^T[key][row]  = K[key][:] . Q[row][:]       A = K from LDS, B = Q in registers
//   O^T[d][row]   += V^T[d][key] . P^T[key][row] A = V^T by transposing LDS reads, B = P out of S^T's own registers: a lane holds keys
//                                                4 h + {0..3} and 8 + 4 h + {0..3} of every 16 (h = lane / 32), and V^T is read in that order
// P is rounded to the operands' type (off by 2^-8 of a weight at most in bf16, 2^-11 in fp16, or 2^-25 of weight 1
// where it is below 2^-14; of random sign), as the matrix cores take it; the sum of weights is not.
#include "heads.h"
#include "lds.h"
#include "sched.h"
#include <cmath>

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class E> struct Half;
template <> struct Half<half_t> {
    typedef half_t x8 __attribute__((ext_vector_type(8)));
    static constexpr unsigned exponent = 0x7C007C00u, one = 0x04000400u;
    static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Half<__bf16> {
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    static constexpr unsigned exponent = 0x7F807F80u, one = 0x00800080u;
    static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

// n / d by a product: exact for 0 <= n < 2^31, 1 <= d < 2^31.
struct Divide {
    unsigned m; int shift;
    static Divide by(unsigned d) {
        int l = 0;
        while ((1u << l) < d) ++l;
        return {(unsigned)(((1ull << (31 + l)) + d - 1) / d), 31 + l};
    }
    __device__ __forceinline__ int operator()(int n) const { return (int)((unsigned long long)(unsigned)n * m >> shift); }
};
struct KvArgs {
    const int *q_starts, *k_starts;                                     // k_starts: packed keys (bb_attention)
    const int *own_pages, *own_lens, *prefix_pages, *prefix_lens, *group_starts;
    const char *q, *k, *v; char* out; float* lse;
    long q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs, k_ps, v_ps;    // elements; k_ps, v_ps: between pages
    long own_ld, prefix_ld;
    int q_tokens, k_tokens, n_seq, n_groups, n_pages, own_width, prefix_width;
    int heads, kv_heads, each, block;
    float scale, lag;                                                   // scale times log2(e); KV_LAG / that
    int own_tiles, own_split, prefix_tiles, prefix_split, halves;       // row tiles that the branches (groups) may have, parts that their keys are cut into.  No prefix tiles: a
                                                                        // branch's items take its group's prefix before its own keys
    Divide by_kv_heads, by_each, by_block, by_own_split, by_prefix_split;
    float* part_o; float2* part_ml;                                     // [part][token][head]: unscaled output; maximum before scale and sum.  Null: a single part
};
#define KV_LEAST_TILES 2                // of 64 keys, a part of as many keys as the plan counts with (a row tile may have fewer)
#define KV_MOST_PARTS 32                // of a branch's own keys, of a prefix
#define KV_FEW_PARTS 6                  // from there on the join takes them four ways
#define KV_MOST_COLUMNS (BB_MAX_TOKENS / BB_PAGE_TOKENS)
#define KV_ROWS 128                     // rows (tokens x heads of a group) of a workgroup
#define KV_LAG 8                        // a row's running maximum is at most 2^KV_LAG behind
#define KV_LARGE 1024.f                 // where products with scale stop being what exponents start from

// Sums over the lanes up to each (in the row's order: within rows of 16, then across them).
static __device__ __forceinline__ int lane_sums(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);     // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);     // row_bcast:15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);     // row_bcast:31 into rows 2 and 3
    return x;
}
// The sequences' row tiles have numbers.  Up to KV_SUMMED sequences: one after the other, found by sums over the sequences, 64 at a look.  More: sequence i (starts[i] .., or with steps
// starts[step[i]] ..) has those from starts[i] * each / ROWS + i on, which leaves it room for all its tiles and now and then one that is none; 64 equal shares of the sequences at a look,
// and on in the last that begins at the number or before.  (A token each of 128, 256, 1024, 4096 branches on 64 keys, 28 heads on 4: sums 8.6, 16.8, 67.5, 526 us, shares 11.9, 18.4, 50.6, 209.)
#define KV_SUMMED 512
// How many numbers there may be.
static long tile_numbers(long rows, long sequences, int rows_per_tile) {
    return sequences <= KV_SUMMED ? (rows + (rows_per_tile - 1) * sequences) / rows_per_tile : (rows + rows_per_tile - 1) / rows_per_tile + sequences - 1;
}
// Of number t: which sequence, its first token, its tokens, which of its tiles; false: none.  Starts are taken as they come but never outside 0 .. q_tokens.  extra(i, x, y): two
// more values of the sequence, loaded with the starts.
struct RowTile { int seq, q0, n, tile, x, y; };
template <int ROWS, class F>
static __device__ __forceinline__ bool find_tile(const KvArgs& a, const int* __restrict__ step, int ranges, int t, int each, RowTile& r, F&& extra) {
    const int lane = threadIdx.x & 63;
    auto start_at = [&](int i) { return min(max(a.q_starts[i], 0), a.q_tokens); };
    auto range = [&](int i, int& s0, int& n, int& x, int& y) {
        int i0 = i, i1 = i + 1;
        if (step) { i0 = min(max(step[i], 0), a.n_seq); i1 = min(max(step[i + 1], i0), a.n_seq); }
        extra(i, x, y);
        s0 = start_at(i0);
        n = max(start_at(i1), s0) - s0;
    };
    auto found = [&](int seq, int l, int s0, int n, int x, int y, int first) {
        r.seq = seq;
        r.q0 = __builtin_amdgcn_readlane(s0, l);
        r.n = __builtin_amdgcn_readlane(n, l);
        r.x = __builtin_amdgcn_readlane(x, l);
        r.y = __builtin_amdgcn_readlane(y, l);
        r.tile = t - __builtin_amdgcn_readlane(first, l);
    };
    auto tiles_of = [&](int n) { return (int)(((unsigned)n * (unsigned)each + ROWS - 1) / ROWS); };
    if (ranges <= KV_SUMMED) {
        for (int b = 0; b < ranges; b += 64) {
            const int i = b + lane;
            int s0 = 0, n = 0, x = 0, y = 0;
            if (i < ranges) range(i, s0, n, x, y);
            const int mine = tiles_of(n), upto = lane_sums(mine);
            const unsigned long long hit = __ballot(upto > t);
            if (hit) {
                const int l = __builtin_ctzll(hit);
                found(b + l, l, s0, n, x, y, upto - mine);
                return true;
            }
            t -= __builtin_amdgcn_readlane(upto, 63);
        }
        return false;
    }
    auto number = [&](int start, int i) { return (int)((unsigned)start * (unsigned)each / ROWS) + i; };
    int b = 0, left = ranges;
    while (left > 64) {
        const int share = (left + 63) / 64, i = lane * share;
        int at = b + min(i, left - 1);
        if (step) at = min(max(step[at], 0), a.n_seq);
        const int k = __builtin_popcountll(__ballot(i < left && number(start_at(at), b + i) <= t));
        if (k == 0) return false;
        b += (k - 1) * share;
        left = min(share, left - (k - 1) * share);
    }
    int s0 = 0, n = 0, x = 0, y = 0;
    if (lane < left) range(b + lane, s0, n, x, y);
    const int first = number(s0, b + lane), l = __builtin_popcountll(__ballot(lane < left && first <= t)) - 1;
    if (l < 0) return false;
    found(b + l, l, s0, n, x, y, first);
    return r.tile >= 0 && r.tile < tiles_of(r.n);
}

// The group a branch belongs to, -1: none.
static __device__ __forceinline__ int find_group(const KvArgs& a, int seq) {
    const int lane = threadIdx.x & 63;
    int b = 0, n = a.n_groups;
    while (n > 64) {                                            // (they ascend: 64 equal shares, and on in the last that starts at the branch or before)
        const int share = (n + 63) / 64, i = lane * share;
        const int k = __builtin_popcountll(__ballot(i < n && a.group_starts[b + i] <= seq));
        if (k == 0) return -1;
        b += (k - 1) * share;
        n = min(share, n - (k - 1) * share);
    }
    const int i = b + lane;
    const unsigned long long hit = __ballot(lane < n && a.group_starts[i] <= seq && seq < a.group_starts[i + 1]);
    return hit ? b + __builtin_ctzll(hit) : -1;
}
static __device__ __forceinline__ int paged_keys(int n, int width) { return min(max(n, 0), width * BB_PAGE_TOKENS); }

// Keys in tiles of KEYS tokens: packed, or pages, those of a prefix before those of its own (a tile never holds both).  The ids of 64 pages at a time stand in a register's
// lanes: a load per tile would have to be waited for, and with it every fetch on its way.  A tile past the end, or of a page that is not in the cache, has no keys (n = 0).
struct KeyTile { const char *k, *v; int key0, n; bool own; };
template <int KEYS> struct Keys {
    const int *prefix, *own;        // page tables (both null: packed)
    const char *k, *v;              // of the kv head; packed: of the next tile's first key, as tiles are asked for in order, `step` apart
    int n_prefix, n_own, step;      // keys
    long k_step, v_step;            // packed: bytes to the next tile
    int ids, ids_at;                // page ids from ids_at on (-1: none yet)
    __device__ __forceinline__ Keys(const KvArgs& a, const int* prefix, const int* own, const char* k, const char* v, int n_prefix, int n_own, int first, int step)
        : prefix(prefix), own(own), k(k), v(v), n_prefix(n_prefix), n_own(n_own), step(step), k_step(0), v_step(0), ids(0), ids_at(-1) {
        if (prefix || own) return;
        this->k += (long)first * KEYS * a.k_ts * 2; this->v += (long)first * KEYS * a.v_ts * 2;
        k_step = (long)step * KEYS * a.k_ts * 2; v_step = (long)step * KEYS * a.v_ts * 2;
    }
    __device__ __forceinline__ KeyTile tile(const KvArgs& a, int i, int end) {
        constexpr int PER_PAGE = BB_PAGE_TOKENS / KEYS;
        KeyTile t{};
        if (i >= end) return t;
        if (!prefix && !own) {
            t.own = true;
            t.key0 = i * KEYS;
            t.k = k; t.v = v;
            k += k_step; v += v_step;
            t.n = max(min(n_own - t.key0, KEYS), 0);            // (the second 32 of the last 64 may be none)
            return t;
        }
        const int prefix_pages = (n_prefix + BB_PAGE_TOKENS - 1) / BB_PAGE_TOKENS, page = i / PER_PAGE, within = i % PER_PAGE * KEYS;
        t.own = i >= prefix_pages * PER_PAGE;
        t.key0 = (t.own ? i - prefix_pages * PER_PAGE : i) * KEYS;
        if (ids_at < 0 || page >= ids_at + 64) {
            ids_at = page;
            const int p = page + (int)(threadIdx.x & 63), of_own = p - prefix_pages;
            ids = of_own < 0 ? prefix[p] : of_own * BB_PAGE_TOKENS < n_own ? own[of_own] : -1;
        }
        const int id = __builtin_amdgcn_readlane(ids, page - ids_at);
        if ((unsigned)id >= (unsigned)a.n_pages) return t;
        t.k = k + ((long)id * a.k_ps + (long)within * a.k_ts) * 2;
        t.v = v + ((long)id * a.v_ps + (long)within * a.v_ts) * 2;
        t.n = max(min((t.own ? n_own : n_prefix) - t.key0, KEYS), 0);
        return t;
    }
};

// Where the 16-byte pieces of a row lie in LDS: piece c of row r at c ^ swizzle(r), so that what a wave reads at once (K: a piece of each of 32 rows; V: 32 bytes of four
// rows, twice) touches all banks evenly.
template <int D> static __device__ __forceinline__ int k_swizzle(int row) { return row & (D / 8 - 1); }
template <int D> static __device__ __forceinline__ int v_swizzle(int row) { return D == 128 ? 4 * (row & 3) : 4 * (row >> 1 & 1); }

// KiB of a tile's K or V on their way into LDS: N of them, every STEP-th from the first-th on.  A lane's offset is that of its row and piece in the first KiB; the rows of the
// next lie `step` bytes further on, and their swizzle is the same, or (K, STEP 1, 16 pieces a row) one of four.
template <int D, bool V, int N, int STEP> struct Fetch {
    static constexpr int PER = D / 8, ROWS = 64 / PER, KINDS = !V && STEP == 1 && D == 128 ? 4 : 1;     // pieces per row, rows per KiB
    unsigned off[KINDS]; long ts2;
    __device__ __forceinline__ static unsigned piece_of(int row) { return (unsigned)(((threadIdx.x & 63) % PER ^ (V ? v_swizzle<D>(row) : k_swizzle<D>(row))) * 16); }
    __device__ __forceinline__ Fetch(long ts, int first) : ts2(ts * 2) {
#pragma unroll
        for (int i = 0; i < KINDS; ++i) {
            const int row = (first + i) * ROWS + (int)(threadIdx.x & 63) / PER;
            off[i] = (unsigned)(row - i * ROWS) * (unsigned)ts2 + piece_of(row);
        }
    }
    // (a buffer load takes the KiB's distance from a scalar register, where a pointer would be added up for each)
    __device__ __forceinline__ void whole(const char* src, unsigned lds, int first) const {
        const unsigned long long at = (unsigned long long)src;
        const u32x4 from = {(unsigned)at, (unsigned)(at >> 32) & 0xFFFFu, 0xFFFFFFFFu, 0x00027000u};
#pragma unroll
        for (int u = 0; u < N; ++u) buffer_to_lds(from, off[u % KINDS], (unsigned)(u * STEP * ROWS) * (unsigned)ts2, lds + (u * STEP + first) * 1024);
    }
    // a tile that ends early: rows past its end as its last one
    __device__ __forceinline__ void some(const char* src, int n, unsigned lds, int first) const {
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));                          // (not worth registers through the loop)
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int row = (u * STEP + first) * ROWS + lane / PER;
            load_to_lds<0>(src, (unsigned)min(row, n - 1) * (unsigned)ts2 + (unsigned)((lane % PER ^ (V ? v_swizzle<D>(row) : k_swizzle<D>(row))) * 16), lds + (u * STEP + first) * 1024);
        }
    }
    __device__ __forceinline__ void operator()(const char* src, int n, int keys, unsigned lds, int first) const {
        if (n == keys) whole(src, lds, first); else some(src, n, lds, first);
    }
};
template <int N> static __device__ __forceinline__ void wait_loads() {      // until N of the wave's fetches are left
    static_assert(N == 0 || N == 4 || N == 8, "");
    if constexpr (N == 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    else if constexpr (N == 4) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
}
static __device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

static __device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
static __device__ __forceinline__ float sum_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Parts of a row: maximum (of the scores before scale) and sum.  A part without a key: (-inf, 0).  One whose scores were all -inf has a finite maximum, so that 0 / 0 comes out as the definition's NaN.
static __device__ __forceinline__ bool no_key(float top, float sum) { return top == -INFINITY && sum == 0.f; }
static __device__ __forceinline__ float rescale(float top, float to, float scale) { return top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((top - to) * scale); }
static __device__ __forceinline__ float log_sum(float top, float sum, float scale) { return no_key(top, sum) ? -INFINITY : (top * scale + __builtin_amdgcn_logf(sum)) * 0.69314718056f; }

// What a lane keeps of its row: the running maximum, what its weights' exponents start from and the score above which the maximum follows (see follow()), its half of the sum, its half
// of the output, whether a key was seen.
template <int D> struct RowState { f32x16 o[D / 32]; float top, from, bar, sum; bool met; };
template <int D> static __device__ __forceinline__ void finish(RowState<D>& r) {
    if (r.met && r.top == -INFINITY && r.sum == 0.f) r.top = -3.402823e38f;
}

// LDS by its byte offset.
template <class T> static __device__ __forceinline__ T lds_at(unsigned offset) { return *(__attribute__((address_space(3))) const T*)(size_t)offset; }
// Where a lane's pieces of a tile lie, from the tile's first byte on: of K (row lane % 32, d = 8 (lane / 32) on) and of V (four keys' d, see values()).  The pieces of the d further on are
// an exclusive or with a constant away, those of the rows further on a sum.
template <int D> static __device__ __forceinline__ unsigned k_piece() {
    const int lane = threadIdx.x & 63, row = lane & 31;
    return row * 2 * D + ((lane >> 5 ^ k_swizzle<D>(row)) * 16);
}
template <int D> static __device__ __forceinline__ unsigned v_piece() {
    const int lane = threadIdx.x & 63, key = 4 * (lane >> 5) + (lane >> 2 & 3), d = (lane >> 4 & 1) * 16 + (lane & 3) * 4;
    return key * 2 * D + (((d >> 3) ^ v_swizzle<D>(key)) * 16) + (d & 7) * 2;
}
// Operands that are on their way from LDS while the matrix cores work; the order is fixed by hand, as the compiler would bring all of them first and spill.
#define AHEAD 4
// Step n of a tile's scores: 16 d (16 (n / NK) on) of 32 keys (32 (n % NK) on).
template <class X8, int D, int NK> static __device__ __forceinline__ X8 key_piece(unsigned kp, unsigned at, int n) { return lds_at<X8>((kp ^ 32 * (n / NK)) + at + n % NK * 64 * D); }
// S^T of 32 NK keys (at LDS offset `at`) and the wave's 32 rows.  kp: k_piece.
template <class E, int D, int NK> static __device__ __forceinline__ void scores(unsigned kp, unsigned at, const typename Half<E>::x8 (&qf)[D / 16], f32x16 (&s)[NK]) {
    typedef typename Half<E>::x8 x8;
    constexpr int STEPS = NK * (D / 16);
    x8 ring[AHEAD];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) ring[n] = key_piece<x8, D, NK>(kp, at, n);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
        s[n % NK] = Half<E>::mfma(ring[n % AHEAD], qf[n / NK], n < NK ? f32x16{} : s[n % NK]);
        if (n + AHEAD < STEPS) ring[n % AHEAD] = key_piece<x8, D, NK>(kp, at, n + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
    }
}
// The rows' maxima follow a tile's scores, each by itself.  PART: not every row sees all of the tile's keys; seen: how many of them the lane's row does.
// One follows only by more than KV_LAG (of 2^KV_LAG), so the output is seldom scaled: a weight is then at most that, of no fewer bits.  (The largest is 1 only where the maximum has just followed; elsewhere
// it is rounded as any other.)
// Weights are exp2(s * by - from).  From is the maximum times scale, rounded: what the rounding is off by, 2^-25 of it, all weights have in common, but from some 2^27 on it leaves the range of
// 16-bit weights, and then of fp32.  Beyond KV_LARGE a row's exponents are (s - maximum) * scale instead, its maximum follows every tile, and the two agree within 2^-15 where a row has both (a
// score's own rounding is off by as much).
template <int D, int NK, bool PART> static __device__ __forceinline__ void follow(RowState<D>& r, f32x16 (&s)[NK], float scale, float lag, int seen, float& by, float& from) {
    const int h2 = (threadIdx.x & 63) >> 5;
    if (PART) {
        r.met |= seen > 0;
#pragma unroll
        for (int i = 0; i < NK; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (32 * i + (e >> 2) * 8 + 4 * h2 + (e & 3) >= seen) s[i][e] = -INFINITY;
    }
    float best = s[0][0];
#pragma unroll
    for (int i = 0; i < NK; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) best = fmaxf(best, s[i][e]);
    best = max_halves(best);
    by = scale;
    if (__ballot(best > r.bar)) {
        const float to = best > r.bar ? fmaxf(best, r.top) : r.top;
        // by 2^126 at most at a time (twice where it is more), so that an infinity in the output stays one
        const float power = (r.top - to) * scale;
        auto scale_by = [&](float keep) {
            r.sum *= keep;
#pragma unroll
            for (int t = 0; t < D / 32; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) r.o[t][e] *= keep;
        };
        const bool more = power < -126.f && r.sum > 0.f;
        scale_by(__builtin_amdgcn_exp2f(fmaxf(power, -126.f)));
        if (__ballot(more)) scale_by(__builtin_amdgcn_exp2f(more ? fmaxf(power + 126.f, -126.f) : 0.f));
        const bool none = to == -INFINITY, large = !none && fabsf(to * scale) >= KV_LARGE;
        r.top = to;
        r.from = none || large ? 0.f : to * scale;
        r.bar = none || large ? -INFINITY : to + lag;
        if (__ballot(large)) {
            const float less = large ? to : 0.f;
#pragma unroll
            for (int i = 0; i < NK; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[i][e] = __builtin_fmaf(s[i][e] - less, scale, -r.from);
            by = 1.f;
            from = 0.f;
            return;
        }
    }
    from = r.from;
}
// Scores -> weights p in the operands' type, elements FROM to TO of all 16 NK.
template <class E, int NK, int FROM, int TO>
static __device__ __forceinline__ void weights(const f32x16 (&s)[NK], float by, float from, float (&sum)[2], typename Half<E>::x8 (&p)[2 * NK]) {
#pragma unroll
    for (int n = FROM; n < TO; ++n) {
        const int i = n >> 4, e = n & 15;
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][e], by, -from));
        sum[n & 1] += w;
        p[n >> 3][n & 7] = (E)w;
    }
}
template <class E, int D, int NK, bool PART>
static __device__ __forceinline__ void weights(RowState<D>& r, f32x16 (&s)[NK], float scale, float lag, int seen, typename Half<E>::x8 (&p)[2 * NK]) {
    float by, from, sum[2] = {0.f, 0.f};
    follow<D, NK, PART>(r, s, scale, lag, seen, by, from);
    weights<E, NK, 0, 16 * NK>(s, by, from, sum, p);
    r.sum += sum[0] + sum[1];
}
// V^T of 16 keys (from 16 st on) and 32 d (from 32 t on), in the order of the weights.  vp: v_piece.
template <class E, int D> static __device__ __forceinline__ typename Half<E>::x8 values(unsigned vp, unsigned at, int st, int t) {
    s16x4 f[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) f[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(size_t)((vp ^ 64 * t) + at + (16 * st + 8 * u) * 2 * D));
    typename Half<E>::x8 v;
    __builtin_memcpy(&v, f, 16);
    return v;
}
// Whether N KiB of LDS, every STEP-th, hold an infinity or a NaN.
template <class E, int N, int STEP> static __device__ __forceinline__ bool any_infinite(unsigned at) {
    unsigned bad = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const u32x4 x = lds_at<u32x4>(at + i * STEP * 1024 + (threadIdx.x & 63) * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) bad |= (x[j] & Half<E>::exponent) + Half<E>::one;
        if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);          // (no more registers than that)
    }
    return __ballot((bad & 0x80008000u) != 0) != 0;
}
// O^T += V^T P^T.  Weight 0 does not hide an infinity or a NaN that a row must not see from the product: in a tile that not every row sees whole (PART) and that holds any (bad),
// the product is made without them, and the rows that see them get them added, key by key (tile: the LDS offset of the tile as a whole).
template <class E, int D, int NK, bool PART>
static __device__ __forceinline__ void weigh(RowState<D>& r, unsigned vp, unsigned at, const typename Half<E>::x8 (&p)[2 * NK], int seen, unsigned tile, bool bad) {
    typedef typename Half<E>::x8 x8;
    constexpr int OT = D / 32, STEPS = 2 * NK * OT;
    asm volatile("" : "+v"(vp));
    x8 ring[AHEAD];
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) ring[n] = values<E, D>(vp, at, n / OT, n % OT);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int n = 0; n < STEPS; ++n) {
        x8 v = ring[n % AHEAD];
        if (PART && bad) {
            u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned b = (w[i] & Half<E>::exponent) + Half<E>::one;
                w[i] &= (b & 0x8000u ? 0u : 0xFFFFu) | (b & 0x80000000u ? 0u : 0xFFFF0000u);
            }
            v = __builtin_bit_cast(x8, w);
        }
        r.o[n % OT] = Half<E>::mfma(v, p[n / OT], r.o[n % OT]);
        if (n + AHEAD < STEPS) ring[n % AHEAD] = values<E, D>(vp, at, (n + AHEAD) / OT, (n + AHEAD) % OT);
        __builtin_amdgcn_sched_barrier(0);
    }
    if (PART && bad) {
#pragma unroll 1
        for (int key = 0; key < 32 * NK; ++key)
#pragma unroll
            for (int t = 0; t < OT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int d = 32 * t + 8 * j + 4 * ((threadIdx.x & 63) >> 5);
                    typedef E x4 __attribute__((ext_vector_type(4)));
                    const x4 v = lds_at<x4>(tile + key * 2 * D + (((d >> 3) ^ v_swizzle<D>(key)) * 16) + (d & 7) * 2);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = (float)v[i];
                        r.o[t][4 * j + i] += key < seen && !(fabsf(x) < INFINITY) ? x : 0.f;
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
    }
}

// A workgroup's item: a row tile of a kv head on a part of the keys of its prefix or of its own.  It has HALVES times four waves.
// A tile of more than 32 rows: a half's four waves take 32 rows each, its tiles of 64 keys (each HALVES-th) pass through two stages of LDS that they share, a barrier per tile.
// Up to 32 rows: every wave has all of them and takes each 4 HALVES-th tile of 32 keys through a slice of LDS of its own (K of the next while it works on V of the last),
// without barriers.  The waves of the same rows are joined at the end, in order.
// One half, two workgroups a CU: where there are items enough (each runs on while the other waits at its barrier).  Two halves, one workgroup a CU: where there are few, so that
// fewer parts of the keys have to be joined through memory (four branches of 120 rows in all on 512 shared and 104 to 128 own keys, 32 heads: 16.7 us, 18.1 with one half).
//
// What bounds it.  16384 causal tokens of 32 heads of 128: 1920 to 2060 us, 1.07 to 1.15 PFLOP/s (a library product of 8192^3 on the same card 1.39): the clock is down to 1.9 GHz for
// power, the matrix pipes are busy for 0.51 of the time and the vector pipes, with the exponentials, conversions and maxima, for 0.52; without the fetches it would take 0.88 of the time, without the
// products 0.65.  The two pipes overlap no better whichever way their instructions are laid out (two tiles of scores at once, halves of a tile by turns, priorities: the same within 1 %, or
// slower).  Short prompts (sixteen of 1 to 1008 tokens, 28 heads on 4: 78 us, 0.6 PFLOP/s) are bound by an item's own time, 11600 cycles besides its tiles: 1700 until its sequence is found, 2000 until
// the first fetch is on its way, the fetch, the join or the barrier, 3300 for its rows' way out.
//
// Why 128 rows by 64 keys: a wave's 32 rows keep queries, weights, scores and output in registers (233 of 256, 236 with pages, so two waves a SIMD), K,V of 64 keys come into LDS once for four
// waves, twice over (64 KiB, two workgroups a CU), and a page is one tile.  K Q^T rather than Q K^T, so that a lane's weights are what the second product takes from it, without a way through LDS.
template <class E, int D, bool PAGED, int HALVES>
__global__ __launch_bounds__(256 * HALVES, 2) void kv_attention_kernel(KvArgs a) {
    typedef typename Half<E>::x8 x8;
    typedef E x4 __attribute__((ext_vector_type(4)));
    constexpr int STAGE = 2 * 64 * D * 2, ST = D / 16, OT = D / 32, WAVES = 4 * HALVES;
    __shared__ __attribute__((aligned(1024))) char lds[HALVES * 2 * STAGE];
    __shared__ float2 ends[WAVES][32];                      // the waves' maxima and sums
    __shared__ __attribute__((aligned(16))) int bad_values[2][WAVES];      // of a stage's V, whether the share that a wave fetched holds an infinity or a NaN
    __shared__ long places[4][32];                          // where a wave's rows go (-1: nowhere)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h2 = lane >> 5, half = HALVES == 1 ? 0 : wave >> 2, w4 = HALVES == 1 ? wave : wave & 3;

    warm_arguments<sizeof(KvArgs)>();
    // Which item: kv head fastest, then the parts of the keys, so that the row tiles of a part of a head's keys go to one XCD (workgroups go to them round robin) wherever their
    // number is a multiple of eight, and share an L2; last row tiles, which see the most keys, first.
    int lin = blockIdx.x;
    const int prefix_items = a.prefix_tiles * a.prefix_split * a.kv_heads;
    const bool prefix = PAGED && lin < prefix_items;
    if (!prefix) lin -= prefix_items;
    const int split = prefix ? a.prefix_split : a.own_split, j = a.by_kv_heads(lin), kvh = lin - j * a.kv_heads, from_last = prefix ? a.by_prefix_split(j) : a.by_own_split(j);
    const int piece = j - from_last * split;
    RowTile r;
    const int* lens = PAGED ? prefix ? a.prefix_lens : a.own_lens : a.k_starts;
    if (!find_tile<KV_ROWS>(a, prefix ? a.group_starts : nullptr, prefix ? a.n_groups : a.n_seq, (prefix ? a.prefix_tiles : a.own_tiles) - 1 - from_last, a.each, r,
                   [&](int i, int& x, int& y) { x = lens[i]; if (!PAGED) y = lens[i + 1]; }))
        return;

    // the lane's row
    const int rows = r.n * a.each, tile_rows = min(rows - r.tile * KV_ROWS, KV_ROWS);
    const bool few = tile_rows <= 32;
    const int row = r.tile * KV_ROWS + (few ? 0 : w4 * 32) + (lane & 31), row_in = min(row, rows - 1);
    const int token = a.by_each(row_in), head = kvh * a.each + row_in - token * a.each;
    x8 qf[ST];
    {
        const char* q = a.q + ((long)(r.q0 + token) * a.q_ts + (long)head * a.q_hs) * 2 + 16 * h2;
#pragma unroll
        for (int s = 0; s < ST; ++s) qf[s] = *reinterpret_cast<const x8*>(q + 32 * s);
    }

    // its keys, and how many of its own the row sees
    const int *prefix_table = nullptr, *own_table = nullptr;
    int n_prefix = 0, m = 0;
    long first = 0;
    if (!PAGED) {
        first = min(max(r.x, 0), a.k_tokens);
        m = min(max(r.y, (int)first), a.k_tokens) - (int)first;
    } else if (prefix) {
        n_prefix = paged_keys(r.x, a.prefix_width);
        prefix_table = a.prefix_pages + (long)r.seq * a.prefix_ld;
    } else {
        m = paged_keys(r.x, a.own_width);
        own_table = a.own_pages + (long)r.seq * a.own_ld;
        const int g = a.n_groups && !prefix_items ? find_group(a, r.seq) : -1;
        if (g >= 0) {
            n_prefix = __builtin_amdgcn_readfirstlane(paged_keys(a.prefix_lens[g], a.prefix_width));
            prefix_table = a.prefix_pages + (long)g * a.prefix_ld;
        }
    }
    int limit = m, tile_limit = m, all_limit = m;               // the lane's row; the last row of the tile; keys that every row of the tile sees
    if (a.block) {
        auto limit_of = [&](int tok) {
            const int p = m - r.n + tok;
            return p < 0 ? 0 : (int)min((long)m, ((long)a.by_block(p) + 1) * a.block);
        };
        limit = limit_of(token);
        tile_limit = limit_of(a.by_each(min(r.tile * KV_ROWS + KV_ROWS - 1, rows - 1)));   // (limits ascend with the token)
        all_limit = limit_of(a.by_each(r.tile * KV_ROWS));
    }
    const int last_limit = __builtin_amdgcn_readlane(limit, 31);
    auto seen = [&](const KeyTile& t) { return t.own ? limit - t.key0 : t.n; };

    RowState<D> st;
#pragma unroll
    for (int t = 0; t < OT; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) st.o[t][e] = 0.f;
    st.top = st.bar = -INFINITY; st.from = st.sum = 0.f; st.met = false;

    const unsigned base = lds_offset(lds);
    const char *kb = a.k + ((long)kvh * a.k_hs + first * a.k_ts) * 2, *vb = a.v + ((long)kvh * a.v_hs + first * a.v_ts) * 2;
    const int n_tiles = (n_prefix + 63) / 64 + (tile_limit + 63) / 64;      // (below 2^25, parts at most 32)
    auto part_from = [&](int of) { return prefix ? a.by_prefix_split(n_tiles * of) : a.by_own_split(n_tiles * of); };
    const int t0 = part_from(piece), t1 = part_from(piece + 1);
    const int whole = n_prefix / 64 + (n_prefix % 64 ? 0 : all_limit / 64);     // tiles that every row sees whole, from the first on
    // The queries have to be there before the loop: left to it, their wait would be one for the fetches that are on their way there, too.
    auto have_queries = [&]() {
#pragma unroll
        for (int i = 0; i < ST; ++i) asm volatile("" : "+v"(qf[i]));
    };
    if (!few) {
        constexpr int N = D / 32;                               // KiB of K (and of V) per wave and tile
        const Fetch<D, false, N, 4> fetch_k(a.k_ts, w4);
        const Fetch<D, true, N, 4> fetch_v(a.v_ts, w4);
        Keys<64> keys(a, prefix_table, own_table, kb, vb, n_prefix, tile_limit, t0 + half, HALVES);
        const unsigned to = base + half * 2 * STAGE, kp = k_piece<D>(), vp = v_piece<D>();
        auto fetch = [&](const KeyTile& t, int stage) {
            if (t.n == 0) return;
            fetch_k(t.k, t.n, 64, to + stage * STAGE, w4);
            fetch_v(t.v, t.n, 64, to + stage * STAGE + STAGE / 2, w4);
        };
        KeyTile cur = keys.tile(a, t0 + half, t1), nxt;
        fetch(cur, 0);
        have_queries();
        const bool live = w4 * 32 < tile_rows;
        const int n_whole = min(max(whole - t0, 0), t1 - t0) / HALVES, n_all = (t1 - t0 + HALVES - 1) / HALVES;    // rounds: of tiles that every row sees whole, all
        int i = 0;
        auto round = [&](auto part, int stage) {
            constexpr bool PART = decltype(part)::value;
            wait_loads<0>();
            if (PART && cur.n) {
                const bool bad = any_infinite<E, N, 4>(to + stage * STAGE + STAGE / 2 + w4 * 1024);
                if (lane == 0) bad_values[stage][wave] = bad;
            }
            __syncthreads();                                    // the round's tiles are there, and all have left those before them: the next on their way into their place
            nxt = keys.tile(a, t0 + half + (i + 1) * HALVES, t1);
            fetch(nxt, 1 - stage);
            if (live && cur.n && (!PART || !cur.own || cur.key0 < last_limit)) {
                const unsigned at = to + stage * STAGE;
                f32x16 s[2];
                x8 p[4];
                int bad = 0;
                if constexpr (PART) {
                    const u32x4 b = *reinterpret_cast<const u32x4*>(&bad_values[stage][half * 4]);
                    bad = __builtin_amdgcn_readfirstlane(b[0] | b[1] | b[2] | b[3]);
                } else st.met = true;
                scores<E, D, 2>(kp, at, qf, s);
                weights<E, D, 2, PART>(st, s, a.scale, a.lag, seen(cur), p);
                weigh<E, D, 2, PART>(st, vp, at + STAGE / 2, p, seen(cur), at + STAGE / 2, bad);
            }
            cur = nxt;
            ++i;
        };
        while (i + 1 < n_whole) { round(std::false_type{}, 0); round(std::false_type{}, 1); }      // (two, so that places in LDS are constants)
        if (i < n_whole) round(std::false_type{}, 0);
        while (i < n_all) round(std::true_type{}, i & 1);
        st.sum = sum_halves(st.sum);
        finish(st);
        if constexpr (HALVES == 2) {
            __syncthreads();
            float4* other = (float4*)(lds + 2 * STAGE) + w4 * 4 * OT * 64;
            if (half) {
                if (h2 == 0) ends[wave][lane] = make_float2(st.top, st.sum);
#pragma unroll
                for (int e = 0; e < 4 * OT; ++e) other[e * 64 + lane] = make_float4(st.o[e >> 2][4 * (e & 3)], st.o[e >> 2][4 * (e & 3) + 1], st.o[e >> 2][4 * (e & 3) + 2], st.o[e >> 2][4 * (e & 3) + 3]);
            }
            __syncthreads();
            if (half) return;
            const float2 theirs = ends[wave + 4][lane & 31];
            const float top = fmaxf(st.top, theirs.x), keep = rescale(st.top, top, a.scale), take = rescale(theirs.x, top, a.scale);
#pragma unroll
            for (int e = 0; e < 4 * OT; ++e) {
                const float4 x = other[e * 64 + lane];
                float* o = (float*)&st.o[e >> 2] + 4 * (e & 3);
                o[0] = o[0] * keep + x.x * take; o[1] = o[1] * keep + x.y * take; o[2] = o[2] * keep + x.z * take; o[3] = o[3] * keep + x.w * take;
            }
            st.sum = st.sum * keep + theirs.y * take;
            st.top = top;
        }
    } else {
        constexpr int N = D / 16;                               // KiB of K (and of V) per tile
        const Fetch<D, false, N, 1> fetch_k(a.k_ts, 0);
        const Fetch<D, true, N, 1> fetch_v(a.v_ts, 0);
        const unsigned to = base + wave * (STAGE / 2), kp = k_piece<D>(), vp = v_piece<D>();
        Keys<32> keys(a, prefix_table, own_table, kb, vb, n_prefix, tile_limit, 2 * t0 + wave, WAVES);
        const int end = 2 * t1;
        int i = 2 * t0 + wave;
        auto next = [&]() {                                     // (tiles without keys are passed over)
            KeyTile t{};
            while (i < end && t.n == 0) { t = keys.tile(a, i, end); i += WAVES; }
            return t;
        };
        KeyTile cur = next(), nxt;
        if (cur.n) {
            fetch_k(cur.k, cur.n, 32, to, 0);
            fetch_v(cur.v, cur.n, 32, to + STAGE / 4, 0);
        }
        have_queries();
        auto step = [&](auto part) {
            constexpr bool PART = decltype(part)::value;
            nxt = next();
            f32x16 s[1];
            x8 p[2];
            if (!PART) st.met = true;
            wait_loads<N>();
            scores<E, D, 1>(kp, to, qf, s);
            wait_lds();
            if (nxt.n) fetch_k(nxt.k, nxt.n, 32, to, 0);
            weights<E, D, 1, PART>(st, s, a.scale, a.lag, seen(cur), p);
            if (nxt.n) wait_loads<N>(); else wait_loads<0>();
            weigh<E, D, 1, PART>(st, vp, to + STAGE / 4, p, seen(cur), to + STAGE / 4, PART && any_infinite<E, N, 1>(to + STAGE / 4));
            wait_lds();
            if (nxt.n) fetch_v(nxt.v, nxt.n, 32, to + STAGE / 4, 0);
            cur = nxt;
        };
        while (cur.n == 32 && (!cur.own || cur.key0 + 32 <= all_limit)) step(std::false_type{});
        while (cur.n) step(std::true_type{});
        // the waves' parts of the same rows: each brings its own to the largest maximum, then each sums its share of the output
        st.sum = sum_halves(st.sum);
        finish(st);
        if (h2 == 0) ends[wave][lane] = make_float2(st.top, st.sum);
        __syncthreads();
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, ends[w][lane & 31].x);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum += ends[w][lane & 31].y * rescale(ends[w][lane & 31].x, top, a.scale);
        const float keep = rescale(st.top, top, a.scale);
        float* all = (float*)lds;
#pragma unroll
        for (int e = 0; e < 16 * OT; ++e) all[(wave * OT * 16 + e) * 64 + lane] = st.o[e >> 4][e & 15] * keep;
        __syncthreads();
        st.top = top; st.sum = sum;
#pragma unroll
        for (int e = 0; e < 16 * OT / WAVES; ++e) {
            float x = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) x += all[(w * OT * 16 + wave * (16 * OT / WAVES) + e) * 64 + lane];
            st.o[e >> 4][e & 15] = x;
        }
    }

    // out, or the part's share of it
    const bool alone = PAGED && !prefix && piece == 0 && a.prefix_split && find_group(a, r.seq) < 0;      // (all lanes look)
    const bool none = no_key(st.top, st.sum), mine = row < rows;
    const float inv = none ? 0.f : 1.f / st.sum;
    const long at_row = (long)(r.q0 + token) * a.heads + head, parts = (long)a.q_tokens * a.heads, slot = prefix ? piece : a.prefix_split + piece;
    if (mine && h2 == 0 && (!few || wave == 0)) {
        if (!a.part_o) {
            if (a.lse) a.lse[at_row] = log_sum(st.top, st.sum, a.scale);
        } else {
            a.part_ml[slot * parts + at_row] = make_float2(st.top, st.sum);
            if (alone)                                          // a branch outside every group: nobody else writes what its prefix would give
                for (int p = 0; p < a.prefix_split; ++p) a.part_ml[p * parts + at_row] = make_float2(-INFINITY, 0.f);
        }
    }
    const long place = a.part_o ? ((slot * parts + at_row) * D) * 4 : ((long)(r.q0 + token) * a.o_ts + (long)head * a.o_hs) * 2;     // (a part without a key: its output is not read)
    char* const out = a.part_o ? (char*)a.part_o : a.out;
    const bool store = mine && !(a.part_o && none);
    if (few) {
        // a lane has runs of four elements of its row (run g: d = 32 (g / 4) + 8 (g % 4) + 4 h2), a wave its share of them
        if (store)
#pragma unroll
            for (int i = 0; i < 4 * OT / WAVES; ++i) {
                const int g = wave * (4 * OT / WAVES) + i, d = 32 * (g >> 2) + 8 * (g & 3) + 4 * h2;
                const float x = st.o[i >> 2][4 * (i & 3)], y = st.o[i >> 2][4 * (i & 3) + 1], z = st.o[i >> 2][4 * (i & 3) + 2], w = st.o[i >> 2][4 * (i & 3) + 3];
                if (a.part_o) *reinterpret_cast<float4*>(out + place + 4 * d) = make_float4(x, y, z, w);
                else *reinterpret_cast<x4*>(out + place + 2 * d) = x4{(E)(x * inv), (E)(y * inv), (E)(z * inv), (E)(w * inv)};
            }
        return;
    }
    // 32 rows a wave, through its slice of LDS, so that whole rows are stored at once (8 bytes of each of 64 rows at a time took an item 2.2 us
    // instead of less than one).  Piece c of row r lies at c ^ r.
    if (HALVES == 1) __syncthreads();                           // (all have left the stages; after the halves' join they have)
    if (h2 == 0) places[w4][lane] = store ? place : -1;
    auto through = [&](auto put, auto bytes_of) {
        constexpr int BYTES = decltype(bytes_of)::value, PER = D * BYTES / 16, ROWS = 64 / PER;      // an element's; pieces a row; rows an instruction
        char* at = lds + w4 * 32 * D * BYTES;
#pragma unroll
        for (int g = 0; g < 4 * OT; ++g) {
            const int d = 32 * (g >> 2) + 8 * (g & 3) + 4 * h2, c = d * BYTES / 16;
            put(at + ((lane & 31) * PER + (c ^ (lane & 31 & (PER - 1)))) * 16 + d * BYTES % 16, st.o[g >> 2][4 * (g & 3)], st.o[g >> 2][4 * (g & 3) + 1], st.o[g >> 2][4 * (g & 3) + 2],
                st.o[g >> 2][4 * (g & 3) + 3]);
        }
        wave_lds_order();
#pragma unroll
        for (int i = 0; i < 32 / ROWS; ++i) {
            const int rr = i * ROWS + lane / PER, c = (lane % PER) ^ (rr & (PER - 1));
            const long to = places[w4][rr];
            const u32x4 x = *reinterpret_cast<const u32x4*>(at + (rr * PER + lane % PER) * 16);
            if (to >= 0) *reinterpret_cast<u32x4*>(out + to + c * 16) = x;
        }
    };
    if (a.part_o) through([](char* at, float x, float y, float z, float w) { *reinterpret_cast<float4*>(at) = make_float4(x, y, z, w); }, IC(4));
    else through([&](char* at, float x, float y, float z, float w) { *reinterpret_cast<x4*>(at) = x4{(E)(x * inv), (E)(y * inv), (E)(z * inv), (E)(w * inv)}; }, IC(2));
}

// The parts of every row, joined: a group of D / 4 lanes takes each WAYS-th of them, AT_ONCE loads on their way while the group's lanes see to the parts' maxima and sums, a part a
// lane; the groups are joined in order.  (Four ways for many parts, which a row's chain of loads would be long for; one, and more rows a workgroup, for few.)
// Memory bounds it: 14000 rows of 128 in four parts 7.7 us (33 MB, 4.2 TB/s); 1792 rows in 25 parts 6.4 us (23 MB), 9.0 with a load after the other.
template <class E, int D, int WAYS> __global__ __launch_bounds__(256) void kv_join_kernel(KvArgs a) {
    typedef E x4 __attribute__((ext_vector_type(4)));
    constexpr int LANES = D / 4, ROWS = 256 / LANES / WAYS, AT_ONCE = WAYS == 1 ? KV_FEW_PARTS - 1 : 8, PER_LANE = 2 * KV_MOST_PARTS / LANES;
    __shared__ float4 outs[WAYS][ROWS][LANES];
    RowTile r;
    if (!find_tile<ROWS>(a, nullptr, a.n_seq, blockIdx.x, a.heads, r, [](int, int&, int&) {})) return;
    const int rows = r.n * a.heads, n_parts = a.prefix_split + a.own_split;
    const int l = threadIdx.x % LANES, i = threadIdx.x / LANES % ROWS, way = threadIdx.x / LANES / ROWS, row = r.tile * ROWS + i;
    const long parts = (long)a.q_tokens * a.heads, at = (long)r.q0 * a.heads + min(row, rows - 1);
    float2 ml[PER_LANE];
#pragma unroll
    for (int n = 0; n < PER_LANE; ++n) ml[n] = l + n * LANES < n_parts ? a.part_ml[(l + n * LANES) * parts + at] : make_float2(-INFINITY, 0.f);
    float4 x[AT_ONCE];
    auto load = [&](int from) {
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
            if (from + u * WAYS < n_parts) x[u] = *reinterpret_cast<const float4*>(a.part_o + ((from + u * WAYS) * parts + at) * D + 4 * l);
    };
    load(way);
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int n = 0; n < PER_LANE; ++n) top = fmaxf(top, ml[n].x);
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    float keep[PER_LANE];                                       // -1: no key, its output was not written
#pragma unroll
    for (int n = 0; n < PER_LANE; ++n) {
        const bool none = no_key(ml[n].x, ml[n].y);
        keep[n] = none ? -1.f : rescale(ml[n].x, top, a.scale);
        sum += none ? 0.f : ml[n].y * keep[n];
    }
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int from = way; from < n_parts; from += AT_ONCE * WAYS) {
        if (from != way) load(from);
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int p = from + u * WAYS;
            float k = keep[0];
#pragma unroll
            for (int n = 1; n < PER_LANE; ++n) k = p / LANES == n ? keep[n] : k;
            k = __shfl(k, p, LANES);
            if (p < n_parts && k >= 0.f) { o.x += x[u].x * k; o.y += x[u].y * k; o.z += x[u].z * k; o.w += x[u].w * k; }
        }
    }
    if (WAYS > 1) {
        outs[way][i][l] = o;
        __syncthreads();
    }
    if (way || row >= rows) return;
#pragma unroll
    for (int w = 1; w < WAYS; ++w) {
        const float4 y = outs[w][i][l];
        o.x += y.x; o.y += y.y; o.z += y.z; o.w += y.w;
    }
    const float inv = no_key(top, sum) ? 0.f : 1.f / sum;
    const int token = row / a.heads, head = row - token * a.heads;
    *reinterpret_cast<x4*>(a.out + ((long)(r.q0 + token) * a.o_ts + (long)head * a.o_hs + 4 * l) * 2) = x4{(E)(o.x * inv), (E)(o.y * inv), (E)(o.z * inv), (E)(o.w * inv)};
    if (a.lse && l == 0) a.lse[at] = log_sum(top, sum, a.scale);
}

template <class E, int D, bool PAGED> static void launch_kv(const KvArgs& a, hipStream_t s) {
    const unsigned grid = (unsigned)((a.prefix_tiles * (long)a.prefix_split + a.own_tiles * (long)a.own_split) * a.kv_heads);
    if (a.halves == 2) kv_attention_kernel<E, D, PAGED, 2><<<grid, 512, 0, s>>>(a); else kv_attention_kernel<E, D, PAGED, 1><<<grid, 256, 0, s>>>(a);
    auto groups = [&](int rows) { return (unsigned)tile_numbers((long)a.q_tokens * a.heads, a.n_seq, rows); };
    if (!a.part_o) return;
    if (a.own_split + a.prefix_split >= KV_FEW_PARTS) kv_join_kernel<E, D, 4><<<groups(64 / (D / 4)), 256, 0, s>>>(a); else kv_join_kernel<E, D, 1><<<groups(256 / (D / 4)), 256, 0, s>>>(a);
}
template <bool PAGED> static void launch_kv(const KvArgs& a, int type, int head_dim, hipStream_t s) {
    if (type == BB_BF16) head_dim == 128 ? launch_kv<__bf16, 128, PAGED>(a, s) : launch_kv<__bf16, 64, PAGED>(a, s);
    else head_dim == 128 ? launch_kv<half_t, 128, PAGED>(a, s) : launch_kv<half_t, 64, PAGED>(a, s);
}

// What a plan, and with it the size of a workspace, depends on.
static bool refuse_common_sizes(long q_tokens, long n_seq, long heads, long kv_heads, long head_dim, long type) {
    return (type != BB_BF16 && type != BB_F16) || (head_dim != 64 && head_dim != 128) || q_tokens < 0 || q_tokens > BB_MAX_TOKENS || n_seq < 0 || n_seq > BB_MAX_TOKENS || heads < 1 ||
           heads > BB_MAX_HEADS || kv_heads < 1 || heads % kv_heads || q_tokens * heads > 1L << 30;
}
// What it does not.
static bool refuse_mask(long block, double scale) { return block < 0 || block > 0x7FFFFFFF || !((float)scale > 0) || !((float)scale * 1.45f < INFINITY); }
// A plan: halves of a workgroup, parts of a branch's keys, of a group's prefix (0: taken by the branches before their own).
struct KvPlan { int halves, own_parts, prefix_parts; };
// How many row tiles there can be, whatever the lengths, and how their keys are shared out: into how many parts, to one or two halves of a workgroup, and whether a prefix is taken once
// for its group, as parts of its own, or again by every branch before its own keys.  Lengths stand on the device: tables count with their width, packed keys with their mean, sequences
// as equally long, the longest somewhat longer.  Lengths that are not so cost time, never results: four branches of 120 rows on 512 shared and 104 to 128 own keys (32 heads) 16.4 us with tables of
// their own width, 18.3 with 16 or 64 columns, 25.9 with 512; 64 tokens on 16381 shared keys (28 heads on 4) 36 and, with 512 columns, 90; one query on 16384 packed keys 12.6, with 31 more on 64 each 95.8, as
// its keys are no longer cut.
// The least of a rough account of the time, us, whose constants were fitted to 38 shapes with up to 50 plans each (what it picked was 1 % slower than the best of them in the mean, 11 % at
// most; the join has become a quarter faster since than JOIN and JOIN_BYTES have it): FIRST for the first loads and the launch, ITEM for a workgroup's own, 64 keys of a row tile ALONE on a CU or
// with another workgroup's (BOTH, 512 at once), or 128 by two HALVES; FEW: times that for tiles of up to 32 rows; the join's launch, and its bytes per us.
static bool plan_parts(KvArgs& a, long own_keys, long prefix_keys, int head_dim, const KvPlan* given) {
    const double FIRST = 3.4, ITEM = 2.8, BOTH = 0.9, ALONE = 1.0, HALVES = 1.5, MERGE = 0.15, FEW = 0.57, LONGEST = 1.2, JOIN = 3.7, JOIN_BYTES = 2.8e6, DIM_64 = 0.53;
    static const int counts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
    const long rows = (long)a.q_tokens * a.each;
    const long own = tile_numbers(rows, a.n_seq, KV_ROWS), pre = prefix_keys > 0 ? tile_numbers(rows, a.n_groups, KV_ROWS) : 0;
    const long own_like = std::max(1L, a.n_seq * ((rows / a.n_seq + KV_ROWS - 1) / KV_ROWS)), pre_like = pre ? std::max(1L, a.n_groups * ((rows / a.n_groups + KV_ROWS - 1) / KV_ROWS)) : 0;
    const long own_cols = std::max(1L, (own_keys + 63) / 64), pre_cols = (prefix_keys + 63) / 64;
    const double scale = head_dim == 64 ? DIM_64 : 1, of = rows / a.n_seq <= 32 ? FEW : 1, pf = pre && rows / a.n_groups <= 32 ? FEW : 1;
    // Launches of less than 2^32 threads (the join's workgroups have two rows at least).
    auto fits = [&](int halves, long op, long pp) { return (own * op + pre * pp) * a.kv_heads < (1L << 24) / halves && (op + pp == 1 || (long)a.q_tokens * a.heads + 2L * a.n_seq < 1L << 25); };
    long own_parts = 1, pre_parts = 0;
    double best = 0;
    a.halves = 1;
    for (int apart = 0; apart <= (pre ? 1 : 0); ++apart)
        for (int halves = 1; halves <= 2; ++halves)
            for (int parts : counts) {
                // (apart: as many for the longer of the two, of that length for the other)
                const long cols = apart ? std::max(own_cols, pre_cols) : own_cols + pre_cols, c = (cols + parts - 1) / parts;
                if (parts > 1 && c < KV_LEAST_TILES) break;
                const long op = apart ? std::min<long>((own_cols + c - 1) / c, parts) : parts, pp = apart ? std::min<long>((pre_cols + c - 1) / c, parts) : 0;
                if (!fits(halves, op, pp)) continue;
                auto rounds = [&](long n, long in) { return (double)(((n + in - 1) / in + halves - 1) / halves); };
                const double oc = rounds(apart ? own_cols : cols, op) * of, pc = apart ? rounds(pre_cols, pp) * pf : 0, oi = (double)own_like * op * a.kv_heads, pi = (double)pre_like * pp * a.kv_heads;
                const bool full = oi + pi > 256;
                const double u = scale * (halves == 2 ? HALVES : full ? BOTH : ALONE), item = ITEM + (halves == 2 ? MERGE : 0);
                const double all = (oi * (item + oc * u) + pi * (item + pc * u)) / (halves == 1 && full ? 512 : 256), longest = item + u * std::max(oc, pc) * (a.n_seq > 1 ? LONGEST : 1);
                const double cost = FIRST + std::max(all, longest) + (op + pp > 1 ? JOIN + (double)rows * a.kv_heads * (op + pp) * head_dim * 8 / JOIN_BYTES : 0);
                if (best == 0 || cost < best) { best = cost; own_parts = op; pre_parts = pp; a.halves = halves; }
            }
    if (given) {
        if (given->halves < 1 || given->halves > 2 || given->own_parts < 1 || given->own_parts > KV_MOST_PARTS || given->prefix_parts < 0 || given->prefix_parts > KV_MOST_PARTS) return false;
        a.halves = given->halves; own_parts = given->own_parts; pre_parts = pre ? given->prefix_parts : 0;
    }
    if (!fits(a.halves, own_parts, pre_parts)) return false;
    a.own_tiles = (int)own; a.own_split = (int)own_parts; a.prefix_tiles = pre_parts ? (int)pre : 0; a.prefix_split = (int)pre_parts;
    a.by_kv_heads = Divide::by(a.kv_heads); a.by_each = Divide::by(a.each); a.by_block = Divide::by(std::max(a.block, 1)); a.by_own_split = Divide::by(a.own_split);
    a.by_prefix_split = Divide::by(std::max(a.prefix_split, 1));
    return true;
}
static size_t parts_bytes(const KvArgs& a, int head_dim) {
    const size_t parts = a.own_split + a.prefix_split;
    return parts > 1 ? align_up((size_t)a.q_tokens * a.heads * parts * head_dim * 4, 256) + align_up((size_t)a.q_tokens * a.heads * parts * 8, 256) : 0;
}
template <bool PAGED> static int run_kv(KvArgs& a, int type, int head_dim, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    const size_t need = parts_bytes(a, head_dim);
    if (need > 0) {
        if (workspace_bytes < need) return BB_ENOMEM;
        if (!workspace_dev || (uintptr_t)workspace_dev % 256) return BB_EINVAL;
        a.part_o = (float*)workspace_dev;
        a.part_ml = (float2*)((char*)workspace_dev + align_up((size_t)a.q_tokens * a.heads * (a.own_split + a.prefix_split) * head_dim * 4, 256));
    }
    launch_kv<PAGED>(a, type, head_dim, (hipStream_t)hip_stream);
    return hipGetLastError() == hipSuccess ? BB_OK : BB_EHIP;
}
// Within a tile offsets are of 32 bits.
static bool far_rows(long ts) { return ts > 1 << 23; }
static bool refuse_ints(const void* p) { return !p || (uintptr_t)p % 4; }

static bool refuse_sizes(const bb_attention_args* x) {
    return !x || refuse_common_sizes(x->q_tokens, x->sequences, x->heads, x->kv_heads, x->head_dim, x->type) || x->k_tokens < 0 || x->k_tokens > BB_MAX_TOKENS;
}
static bool plan(KvArgs& a, const bb_attention_args* x, const KvPlan* given = nullptr) {
    a.n_seq = (int)x->sequences; a.q_tokens = (int)x->q_tokens; a.k_tokens = (int)x->k_tokens; a.heads = (int)x->heads; a.kv_heads = (int)x->kv_heads; a.each = a.heads / a.kv_heads;
    a.block = (int)x->block; a.scale = (float)x->scale * 1.44269504089f; a.lag = KV_LAG / a.scale;
    return plan_parts(a, x->k_tokens / x->sequences, 0, (int)x->head_dim, given);
}
extern "C" size_t bb_attention_workspace_bytes(const bb_attention_args* x) {
    KvArgs a{};
    return refuse_sizes(x) || x->q_tokens == 0 || x->sequences == 0 || !plan(a, x) ? 0 : parts_bytes(a, (int)x->head_dim);
}
static int attention(const bb_attention_args* x, const KvPlan* given, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    if (refuse_sizes(x) || refuse_mask(x->block, x->scale)) return BB_EINVAL;
    if (x->q_tokens == 0 || x->sequences == 0) return BB_OK;
    if (refuse_ints(x->q_starts) || refuse_ints(x->k_starts) || (uintptr_t)x->lse % 4) return BB_EINVAL;
    const int heads = (int)x->heads, kv_heads = (int)x->kv_heads, dim = (int)x->head_dim;
    const HeadView q = heads_view(x->q, x->q_tokens, x->q_token, heads, x->q_head, dim, 2), o = heads_view(x->out, x->q_tokens, x->o_token, heads, x->o_head, dim, 2);
    const HeadView k = heads_view(x->k, x->k_tokens, x->k_token, kv_heads, x->k_head, dim, 2), v = heads_view(x->v, x->k_tokens, x->v_token, kv_heads, x->v_head, dim, 2);
    const HeadView l = heads_view(x->lse, x->q_tokens, heads, heads, 1, 1, 4);
    if (refuse_view(q) || refuse_pieces(q) || refuse_out_view(o) || refuse_pieces(o) || overlap(o, q) || (x->lse && (overlap(l, o) || overlap(l, q)))) return BB_EINVAL;
    if (x->k_tokens > 0) {
        if (refuse_view(k) || refuse_pieces(k) || far_rows(k.s[0]) || refuse_view(v) || refuse_pieces(v) || far_rows(v.s[0])) return BB_EINVAL;
        if (overlap(o, k) || overlap(o, v) || (x->lse && (overlap(l, k) || overlap(l, v)))) return BB_EINVAL;
    }
    KvArgs a{};
    if (!plan(a, x, given)) return BB_EINVAL;
    // (strides as the views have them: none over a single token or head)
    a.q = (const char*)x->q; a.q_ts = q.s[0]; a.q_hs = q.s[1]; a.k = (const char*)x->k; a.k_ts = k.s[0]; a.k_hs = k.s[1]; a.v = (const char*)x->v; a.v_ts = v.s[0]; a.v_hs = v.s[1];
    a.out = (char*)x->out; a.o_ts = o.s[0]; a.o_hs = o.s[1]; a.lse = x->lse; a.q_starts = x->q_starts; a.k_starts = x->k_starts;
    return run_kv<false>(a, (int)x->type, dim, workspace_dev, workspace_bytes, hip_stream);
}

static bool refuse_sizes(const bb_shared_attention_args* x) {
    return !x || refuse_common_sizes(x->q_tokens, x->branches, x->heads, x->kv_heads, x->head_dim, x->type) || x->groups < 0 || x->groups > BB_MAX_TOKENS ||
           x->own_width < 0 || x->own_width > KV_MOST_COLUMNS || (x->groups > 0 && (x->prefix_width < 0 || x->prefix_width > KV_MOST_COLUMNS));
}
static bool plan(KvArgs& a, const bb_shared_attention_args* x, const KvPlan* given = nullptr) {
    a.n_seq = (int)x->branches; a.q_tokens = (int)x->q_tokens; a.heads = (int)x->heads; a.kv_heads = (int)x->kv_heads; a.each = a.heads / a.kv_heads;
    a.block = (int)x->block; a.scale = (float)x->scale * 1.44269504089f; a.lag = KV_LAG / a.scale;
    a.own_width = (int)x->own_width; a.n_groups = (int)x->groups; a.prefix_width = x->groups ? (int)x->prefix_width : 0;
    return plan_parts(a, 64L * a.own_width, 64L * a.prefix_width, (int)x->head_dim, given);
}
extern "C" size_t bb_shared_attention_workspace_bytes(const bb_shared_attention_args* x) {
    KvArgs a{};
    return refuse_sizes(x) || x->q_tokens == 0 || x->branches == 0 || !plan(a, x) ? 0 : parts_bytes(a, (int)x->head_dim);
}
static int shared_attention(const bb_shared_attention_args* x, const KvPlan* given, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    if (refuse_sizes(x) || refuse_mask(x->block, x->scale) || x->pages < 1 || x->pages > BB_MAX_PAGES || (x->branches > 1 && x->own_ld < 0) || (x->groups > 1 && x->prefix_ld < 0) ||
        x->own_ld > HEADS_MAX_STRIDE || (x->groups > 0 && x->prefix_ld > HEADS_MAX_STRIDE)) return BB_EINVAL;
    if (x->q_tokens == 0 || x->branches == 0) return BB_OK;
    if (refuse_ints(x->q_starts) || refuse_ints(x->own_lens) || (x->own_width > 0 && refuse_ints(x->own_pages)) || (uintptr_t)x->lse % 4) return BB_EINVAL;
    if (x->groups > 0 && (refuse_ints(x->prefix_lens) || refuse_ints(x->group_starts) || (x->prefix_width > 0 && refuse_ints(x->prefix_pages)))) return BB_EINVAL;
    const int heads = (int)x->heads, kv_heads = (int)x->kv_heads, dim = (int)x->head_dim;
    const HeadView q = heads_view(x->q, x->q_tokens, x->q_token, heads, x->q_head, dim, 2), o = heads_view(x->out, x->q_tokens, x->o_token, heads, x->o_head, dim, 2);
    const HeadView l = heads_view(x->lse, x->q_tokens, heads, heads, 1, 1, 4);
    const HeadView k = pages_view(x->k_cache, x->pages, x->kc_page, kv_heads, x->kc_head, x->kc_token, dim, 2), v = pages_view(x->v_cache, x->pages, x->vc_page, kv_heads, x->vc_head, x->vc_token, dim, 2);
    if (refuse_view(q) || refuse_pieces(q) || refuse_out_view(o) || refuse_pieces(o) || refuse_view(k) || refuse_pieces(k) || refuse_view(v) || refuse_pieces(v) ||
        far_rows(x->kc_token) || far_rows(x->vc_token) || overlap(o, q) || overlap(o, k) || overlap(o, v) ||
        (x->lse && (overlap(l, o) || overlap(l, q) || overlap(l, k) || overlap(l, v)))) return BB_EINVAL;
    KvArgs a{};
    if (!plan(a, x, given)) return BB_EINVAL;
    a.q = (const char*)x->q; a.q_ts = q.s[0]; a.q_hs = q.s[1]; a.k = (const char*)x->k_cache; a.k_ps = k.s[0]; a.k_hs = k.s[1]; a.k_ts = k.s[2];
    a.v = (const char*)x->v_cache; a.v_ps = v.s[0]; a.v_hs = v.s[1]; a.v_ts = v.s[2]; a.out = (char*)x->out; a.o_ts = o.s[0]; a.o_hs = o.s[1]; a.lse = x->lse;
    a.q_starts = x->q_starts; a.own_pages = x->own_pages; a.own_ld = x->branches > 1 ? x->own_ld : 0; a.own_lens = x->own_lens;
    a.prefix_pages = x->prefix_pages; a.prefix_ld = x->groups > 1 ? x->prefix_ld : 0; a.prefix_lens = x->prefix_lens; a.group_starts = x->group_starts; a.n_pages = (int)x->pages;
    return run_kv<true>(a, (int)x->type, dim, workspace_dev, workspace_bytes, hip_stream);
}

extern "C" int bb_attention(const bb_attention_args* x, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    return attention(x, nullptr, workspace_dev, workspace_bytes, hip_stream);
}
extern "C" int bb_shared_attention(const bb_shared_attention_args* x, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    return shared_attention(x, nullptr, workspace_dev, workspace_bytes, hip_stream);
}

// ---- tests ------------------------------------------------------------------------------------------------------------------------------------
extern "C" int bb_debug_attention(const bb_attention_args* x, int halves, int parts, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    const KvPlan given{halves, parts, 0};
    return attention(x, &given, workspace_dev, workspace_bytes, hip_stream);
}
extern "C" int bb_debug_shared_attention(const bb_shared_attention_args* x, int halves, int own_parts, int prefix_parts, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    const KvPlan given{halves, own_parts, prefix_parts};
    return shared_attention(x, &given, workspace_dev, workspace_bytes, hip_stream);
}
