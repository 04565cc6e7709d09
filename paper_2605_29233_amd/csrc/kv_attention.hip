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
// P is rounded to the operands' type (bf16: 2^-9 of each weight at most, of random sign), as the matrix cores take it; the sum of weights is not.
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

struct KvArgs {
    const char *q, *k, *v; char* out; float* lse;
    long q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs, k_ps, v_ps;    // elements; k_ps, v_ps: between pages
    const int *q_starts, *k_starts;                                     // k_starts: packed keys (bb_attention)
    const int *own_pages, *own_lens, *prefix_pages, *prefix_lens, *group_starts;
    long own_ld, prefix_ld;
    int q_tokens, k_tokens, n_seq, n_groups, n_pages, own_width, prefix_width;
    int heads, each, tiles, block;
    float scale;                                                        // times log2(e)
};

// Of `bound` sequences' row tiles the t-th: which sequence, its first and last token, which of its tiles.  Starts are taken as they come but never outside 0 .. q_tokens.
struct RowTile { int seq, q0, n, tile; };
static __device__ __forceinline__ bool find_tile(const KvArgs& a, int t, int rows_per_tile, RowTile& r) {
    const int lane = threadIdx.x & 63;
    for (int b = 0; b < a.n_seq; b += 64) {
        const int i = b + lane;
        int s0 = 0, n = 0;
        if (i < a.n_seq) {
            s0 = min(max(a.q_starts[i], 0), a.q_tokens);
            n = min(max(a.q_starts[i + 1], s0), a.q_tokens) - s0;
        }
        const int mine = (int)(((long)n * a.each + rows_per_tile - 1) / rows_per_tile);
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int below = __shfl_up(upto, o, 64);
            if (lane >= o) upto += below;
        }
        const unsigned long long hit = __ballot(upto > t);
        if (hit) {
            const int l = __builtin_ctzll(hit);
            r.seq = b + l;
            r.q0 = __builtin_amdgcn_readlane(s0, l);
            r.n = __builtin_amdgcn_readlane(n, l);
            r.tile = t - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l));
            return true;
        }
        t -= __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// Which group a branch belongs to, -1: none.
static __device__ __forceinline__ int find_group(const KvArgs& a, int seq) {
    const int lane = threadIdx.x & 63;
    for (int b = 0; b < a.n_groups; b += 64) {
        const int i = b + lane;
        const unsigned long long hit = __ballot(i < a.n_groups && a.group_starts[i] <= seq && seq < a.group_starts[i + 1]);
        if (hit) return b + __builtin_ctzll(hit);
    }
    return -1;
}

// The keys of a row tile, 64 at a time: pages of the prefix, then pages of its own, or packed keys.  Pages that are not in the cache count as not there.
struct KeyTile { const char *k, *v; int key0, n; bool own; };
struct Keys {
    const int *prefix, *own;        // page tables (null: packed)
    int n_prefix, n_own, i;         // keys; i: the next tile
    const char *k, *v;              // of the kv head (packed: of the sequence's first key)
    __device__ __forceinline__ bool next(const KvArgs& a, KeyTile& t) {
        const int tiles_p = (n_prefix + 63) >> 6, tiles = tiles_p + ((n_own + 63) >> 6);
        while (i < tiles) {
            const int at = i++;
            t.own = at >= tiles_p;
            t.key0 = (t.own ? at - tiles_p : at) << 6;
            t.n = min((t.own ? n_own : n_prefix) - t.key0, 64);
            if (!a.k_starts) {
                const int page = __builtin_amdgcn_readfirstlane((t.own ? own : prefix)[t.key0 >> 6]);
                if ((unsigned)page >= (unsigned)a.n_pages) continue;
                t.k = k + (long)page * a.k_ps * 2;
                t.v = v + (long)page * a.v_ps * 2;
            } else {
                t.k = k + (long)t.key0 * a.k_ts * 2;
                t.v = v + (long)t.key0 * a.v_ts * 2;
            }
            return true;
        }
        return false;
    }
};

template <int D> static __device__ __forceinline__ int k_swizzle(int row) { return row & (D / 8 - 1); }
template <int D> static __device__ __forceinline__ int v_swizzle(int row) { return D == 128 ? 4 * (row & 3) : 4 * (row >> 1 & 1); }

// One tile's K and V on their way into LDS, rows past its end as its last one.
template <int D> static __device__ __forceinline__ void fetch_tile(const KvArgs& a, const KeyTile& t, unsigned lds, int wave, int lane) {
    constexpr int PER = D / 8, ROWS = 64 / PER, UNITS = 64 / ROWS;      // pieces per row, rows per KiB, KiB per tile
#pragma unroll
    for (int u = 0; u < UNITS / 4; ++u) {
        const int unit = u * 4 + wave, row = unit * ROWS + lane / PER, piece = lane % PER, from = min(row, t.n - 1);
        load_to_lds<0>(t.k, (unsigned)(from * (unsigned)a.k_ts * 2 + (unsigned)((piece ^ k_swizzle<D>(row)) * 16)), lds + unit * 1024);
        load_to_lds<0>(t.v, (unsigned)(from * (unsigned)a.v_ts * 2 + (unsigned)((piece ^ v_swizzle<D>(row)) * 16)), lds + 128 * D + unit * 1024);
    }
}

static __device__ __forceinline__ float other_half(float x, float& both) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    both = __uint_as_float(r[1]);
    return __uint_as_float(r[0]);
}
static __device__ __forceinline__ float max_halves(float x) { float y; const float z = other_half(x, y); return fmaxf(z, y); }
static __device__ __forceinline__ float sum_halves(float x) { float y; const float z = other_half(x, y); return z + y; }

template <class E, int D>
__global__ __launch_bounds__(256) void kv_attention_kernel(KvArgs a) {
    typedef typename Half<E>::x8 x8;
    constexpr int STAGE = 2 * 64 * D * 2, ST = D / 16, OT = D / 32;
    __shared__ __attribute__((aligned(1024))) char lds[2 * STAGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h2 = lane >> 5;
    const int kvh = blockIdx.x / a.tiles;
    RowTile r;
    if (!find_tile(a, a.tiles - 1 - (int)(blockIdx.x - kvh * a.tiles), 128, r)) return;

    // the wave's rows
    const int rows = r.n * a.each, row = r.tile * 128 + wave * 32 + (lane & 31);
    const int token = min(row, rows - 1) / a.each, head = kvh * a.each + min(row, rows - 1) - token * a.each;
    x8 qf[ST];
    {
        const char* q = a.q + ((long)(r.q0 + token) * a.q_ts + (long)head * a.q_hs) * 2 + 16 * h2;
#pragma unroll
        for (int s = 0; s < ST; ++s) qf[s] = *reinterpret_cast<const x8*>(q + 32 * s);
    }

    // its keys
    Keys keys{};
    if (a.k_starts) {
        const int s0 = min(max(a.k_starts[r.seq], 0), a.k_tokens);
        keys.n_own = __builtin_amdgcn_readfirstlane(min(max(a.k_starts[r.seq + 1], s0), a.k_tokens) - s0);
        const int k0 = __builtin_amdgcn_readfirstlane(s0);
        keys.k = a.k + ((long)k0 * a.k_ts + (long)kvh * a.k_hs) * 2;
        keys.v = a.v + ((long)k0 * a.v_ts + (long)kvh * a.v_hs) * 2;
    } else {
        keys.n_own = __builtin_amdgcn_readfirstlane(min(max(a.own_lens[r.seq], 0), a.own_width * 64));
        keys.own = a.own_pages + (long)r.seq * a.own_ld;
        const int g = a.n_groups ? find_group(a, r.seq) : -1;
        if (g >= 0) {
            keys.n_prefix = __builtin_amdgcn_readfirstlane(min(max(a.prefix_lens[g], 0), a.prefix_width * 64));
            keys.prefix = a.prefix_pages + (long)g * a.prefix_ld;
        }
        keys.k = a.k + (long)kvh * a.k_hs * 2;
        keys.v = a.v + (long)kvh * a.v_hs * 2;
    }
    const int m_keys = keys.n_own;
    auto limit_of = [&](int tok) {      // how many of its own keys a query sees
        if (a.block == 0) return m_keys;
        const int p = m_keys - r.n + tok;
        return p < 0 ? 0 : (int)min((long)m_keys, ((long)(p / a.block) + 1) * a.block);
    };
    const int limit = limit_of(token);
    const int first_limit = __builtin_amdgcn_readfirstlane(limit);                      // (tokens ascend with the lane)
    const bool live = r.tile * 128 + wave * 32 < rows;
    const int last_limit = __builtin_amdgcn_readlane(limit, 31);
    keys.n_own = limit_of(min(r.tile * 128 + 127, rows - 1) / a.each);                  // beyond it no row of the tile sees any

    f32x16 o[OT];
#pragma unroll
    for (int t = 0; t < OT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float top = -INFINITY, sum = 0.f;
    bool met = false;                                               // a key was seen

    const unsigned base = lds_offset(lds);
    KeyTile cur, nxt;
    bool more = keys.next(a, cur);
    if (more) fetch_tile<D>(a, cur, base, wave, lane);
    for (int stage = 0; more; stage ^= 1) {
        const bool after = keys.next(a, nxt);
        if (after) {
            fetch_tile<D>(a, nxt, base + (stage ^ 1) * STAGE, wave, lane);
            if (D == 128) asm volatile("s_waitcnt vmcnt(8)" ::: "memory"); else asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
        } else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (live && (!cur.own || cur.key0 < last_limit)) {
            const char* kt = lds + stage * STAGE;
            const char* vt = kt + 128 * D;
            f32x16 s[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[i][e] = 0.f;
                const int kr = 32 * i + (lane & 31);
#pragma unroll
                for (int st = 0; st < ST; ++st)
                    s[i] = Half<E>::mfma(*reinterpret_cast<const x8*>(kt + kr * 2 * D + (((2 * st + h2) ^ k_swizzle<D>(kr)) * 16)), qf[st], s[i]);
            }
            const int seen = cur.own ? limit - cur.key0 : cur.n;
            met |= seen > 0;
            const bool part = cur.own ? first_limit < cur.key0 + 64 : cur.n < 64;
            if (part) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (32 * i + (e >> 2) * 8 + 4 * h2 + (e & 3) >= seen) s[i][e] = -INFINITY;
            }
            float best = -INFINITY;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) best = fmaxf(best, s[i][e]);
            best = fmaxf(top, max_halves(best) * a.scale);
            if (__ballot(best > top)) {
                const float keep = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - best);
                sum *= keep;
#pragma unroll
                for (int t = 0; t < OT; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[t][e] *= keep;
                top = best;
            }
            const float from = top == -INFINITY ? 0.f : top;        // (no key seen yet: every weight 0)
            x8 p[4];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][e], a.scale, -from));
                    sum += w;
                    p[2 * i + (e >> 3)][e & 7] = (E)w;
                }
#pragma unroll
            for (int st = 0; st < 4; ++st)
#pragma unroll
                for (int t = 0; t < OT; ++t) {
                    s16x4 f[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int key = 16 * st + 8 * u + 4 * h2 + (lane >> 2 & 3), d = 32 * t + (lane >> 4 & 1) * 16 + (lane & 3) * 4;
                        f[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                            (__attribute__((address_space(3))) s16x4*)(vt + key * 2 * D + (((d >> 3) ^ v_swizzle<D>(key)) * 16) + (d & 7) * 2));
                    }
                    u32x4 vf;
                    __builtin_memcpy(&vf, f, 16);
                    if (part) {
                        // Weight 0 does not hide an infinity or a NaN that a row must not see from the product.  Where V holds any they are taken out, and
                        // given to the rows that see them, by a product of where they are (a NaN: both infinities).
                        unsigned bad = 0;
#pragma unroll
                        for (int i = 0; i < 4; ++i) bad |= (vf[i] & Half<E>::exponent) + Half<E>::one;
                        if (__ballot((bad & 0x80008000u) != 0)) {
                            const x8 all = __builtin_bit_cast(x8, vf);
                            x8 fin, plus, minus, see;
                            f32x16 z;
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const float x = (float)all[e];
                                const bool fine = fabsf(x) < INFINITY;
                                fin[e] = fine ? all[e] : (E)0.f;
                                plus[e] = (E)(fine || x < 0.f ? 0.f : 1.f);
                                minus[e] = (E)(fine || x > 0.f ? 0.f : 1.f);
                                see[e] = (E)(16 * st + (e >> 2) * 8 + 4 * h2 + (e & 3) < seen ? 1.f : 0.f);
                            }
#pragma unroll
                            for (int e = 0; e < 16; ++e) z[e] = 0.f;
                            const f32x16 up = Half<E>::mfma(plus, see, z), down = Half<E>::mfma(minus, see, z);
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                if (up[e] > 0.f) o[t][e] += INFINITY;
                                if (down[e] > 0.f) o[t][e] -= INFINITY;
                            }
                            vf = __builtin_bit_cast(u32x4, fin);
                        }
                    }
                    o[t] = Half<E>::mfma(__builtin_bit_cast(x8, vf), p[st], o[t]);
                }
        }
        __syncthreads();
        cur = nxt;
        more = after;
    }

    sum = sum_halves(sum);
    if (row >= rows) return;
    const float inv = met ? 1.f / sum : 0.f;
    char* out = a.out + ((long)(r.q0 + token) * a.o_ts + (long)head * a.o_hs) * 2;
    typedef E x4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int t = 0; t < OT; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x4 y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = (E)(o[t][4 * j + i] * inv);
            *reinterpret_cast<x4*>(out + (32 * t + 8 * j + 4 * h2) * 2) = y;
        }
    if (a.lse && h2 == 0) a.lse[(long)(r.q0 + token) * a.heads + head] = met ? (top + __builtin_amdgcn_logf(sum)) * 0.69314718056f : -INFINITY;
}

template <class E> static void launch_kv(const KvArgs& a, int kv_heads, int head_dim, hipStream_t s) {
    const unsigned grid = (unsigned)a.tiles * kv_heads;
    if (head_dim == 128) kv_attention_kernel<E, 128><<<grid, 256, 0, s>>>(a);
    else kv_attention_kernel<E, 64><<<grid, 256, 0, s>>>(a);
}

static bool refuse_attention(long q_tokens, int n_seq, int heads, int kv_heads, int head_dim, int type, int block, float scale) {
    return (type != BB_BF16 && type != BB_F16) || (head_dim != 64 && head_dim != 128) || q_tokens < 0 || q_tokens > BB_MAX_TOKENS || n_seq < 0 || n_seq > BB_MAX_TOKENS || heads < 1 ||
           heads > BB_MAX_HEADS || kv_heads < 1 || heads % kv_heads || block < 0 || !(scale > 0) || !(scale < INFINITY);
}
// Tiles of 128 rows: as many as the sequences may need, whatever their lengths.
static bool plan_tiles(KvArgs& a, int kv_heads) {
    const long tiles = ((long)a.q_tokens * a.each + 127) / 128 + a.n_seq, n = tiles * kv_heads;
    if (n > 0x7FFFFFFF) return false;
    a.tiles = (int)tiles;
    return true;
}
// Within a tile offsets are of 32 bits.
static bool far_rows(long ts) { return ts > 1 << 23; }

extern "C" size_t bb_attention_workspace_bytes(long q_tokens, long k_tokens, int n_seq, int heads, int kv_heads, int head_dim) { return 0; }

extern "C" int bb_attention(const void* q_dev, long q_token, long q_head, const void* k_dev, long k_token, long k_head, const void* v_dev, long v_token, long v_head,
                            const int32_t* q_starts_dev, const int32_t* k_starts_dev, int n_seq, long q_tokens, long k_tokens, int heads, int kv_heads, int head_dim,
                            int type, int block, float scale, void* out_dev, long o_token, long o_head, float* lse_dev, void* workspace_dev, size_t workspace_bytes,
                            void* hip_stream) {
    if (refuse_attention(q_tokens, n_seq, heads, kv_heads, head_dim, type, block, scale) || k_tokens < 0 || k_tokens > BB_MAX_TOKENS) return BB_EINVAL;
    if (q_tokens == 0 || n_seq == 0) return BB_OK;
    if (!q_starts_dev || !k_starts_dev || (uintptr_t)q_starts_dev % 4 || (uintptr_t)k_starts_dev % 4 || (uintptr_t)lse_dev % 4) return BB_EINVAL;
    const HeadView q = heads_view(q_dev, q_tokens, q_token, heads, q_head, head_dim, 2), o = heads_view(out_dev, q_tokens, o_token, heads, o_head, head_dim, 2);
    if (refuse_view(q) || refuse_pieces(q) || refuse_out_view(o) || refuse_pieces(o) || overlap(o, q)) return BB_EINVAL;
    if (k_tokens > 0) {
        const HeadView k = heads_view(k_dev, k_tokens, k_token, kv_heads, k_head, head_dim, 2), v = heads_view(v_dev, k_tokens, v_token, kv_heads, v_head, head_dim, 2);
        if (refuse_view(k) || refuse_pieces(k) || refuse_view(v) || refuse_pieces(v) || far_rows(k.s[0]) || far_rows(v.s[0]) || overlap(o, k) || overlap(o, v)) return BB_EINVAL;
    }
    KvArgs a{};
    a.q = (const char*)q_dev; a.q_ts = q_token; a.q_hs = q_head; a.k = (const char*)k_dev; a.k_ts = k_tokens > 1 ? k_token : 0; a.k_hs = k_head;
    a.v = (const char*)v_dev; a.v_ts = k_tokens > 1 ? v_token : 0; a.v_hs = v_head; a.out = (char*)out_dev; a.o_ts = o_token; a.o_hs = o_head; a.lse = lse_dev;
    a.q_starts = q_starts_dev; a.k_starts = k_starts_dev; a.n_seq = n_seq; a.q_tokens = (int)q_tokens; a.k_tokens = (int)k_tokens;
    a.heads = heads; a.each = heads / kv_heads; a.block = block; a.scale = scale * 1.44269504089f;
    if (!plan_tiles(a, kv_heads)) return BB_EINVAL;
    if (type == BB_BF16) launch_kv<__bf16>(a, kv_heads, head_dim, (hipStream_t)hip_stream); else launch_kv<half_t>(a, kv_heads, head_dim, (hipStream_t)hip_stream);
    return hipGetLastError() == hipSuccess ? BB_OK : BB_EHIP;
}

extern "C" size_t bb_shared_attention_workspace_bytes(long q_tokens, int n_branches, int n_groups, int own_width, int prefix_width, int heads, int kv_heads, int head_dim) { return 0; }

extern "C" int bb_shared_attention(const void* q_dev, long q_token, long q_head, const int32_t* q_starts_dev, int n_branches, long q_tokens, const void* k_cache_dev, long kc_page,
                                   long kc_head, long kc_token, const void* v_cache_dev, long vc_page, long vc_head, long vc_token, int n_pages, const int32_t* own_pages_dev,
                                   long own_ld, int own_width, const int32_t* own_lens_dev, const int32_t* prefix_pages_dev, long prefix_ld, int prefix_width,
                                   const int32_t* prefix_lens_dev, const int32_t* group_starts_dev, int n_groups, int heads, int kv_heads, int head_dim, int type, int block,
                                   float scale, void* out_dev, long o_token, long o_head, float* lse_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    if (refuse_attention(q_tokens, n_branches, heads, kv_heads, head_dim, type, block, scale) || n_groups < 0 || n_groups > BB_MAX_TOKENS || n_pages < 1 || n_pages > BB_MAX_PAGES ||
        own_width < 0 || own_width > BB_MAX_PAGES || prefix_width < 0 || prefix_width > BB_MAX_PAGES || (n_branches > 1 && own_ld < 0) || (n_groups > 1 && prefix_ld < 0))
        return BB_EINVAL;
    if (q_tokens == 0 || n_branches == 0) return BB_OK;
    if (!q_starts_dev || !own_lens_dev || (own_width > 0 && !own_pages_dev) || (uintptr_t)q_starts_dev % 4 || (uintptr_t)own_pages_dev % 4 || (uintptr_t)own_lens_dev % 4 ||
        (uintptr_t)lse_dev % 4) return BB_EINVAL;
    if (n_groups > 0 && (!prefix_lens_dev || !group_starts_dev || (prefix_width > 0 && !prefix_pages_dev) || (uintptr_t)prefix_pages_dev % 4 || (uintptr_t)prefix_lens_dev % 4 ||
                         (uintptr_t)group_starts_dev % 4)) return BB_EINVAL;
    const HeadView q = heads_view(q_dev, q_tokens, q_token, heads, q_head, head_dim, 2), o = heads_view(out_dev, q_tokens, o_token, heads, o_head, head_dim, 2);
    const HeadView k = pages_view(k_cache_dev, n_pages, kc_page, kv_heads, kc_head, kc_token, head_dim, 2);
    const HeadView v = pages_view(v_cache_dev, n_pages, vc_page, kv_heads, vc_head, vc_token, head_dim, 2);
    if (refuse_view(q) || refuse_pieces(q) || refuse_out_view(o) || refuse_pieces(o) || refuse_view(k) || refuse_pieces(k) || refuse_view(v) || refuse_pieces(v) ||
        far_rows(kc_token) || far_rows(vc_token) || overlap(o, q) || overlap(o, k) || overlap(o, v)) return BB_EINVAL;
    KvArgs a{};
    a.q = (const char*)q_dev; a.q_ts = q_token; a.q_hs = q_head; a.k = (const char*)k_cache_dev; a.k_ps = kc_page; a.k_ts = kc_token; a.k_hs = kc_head;
    a.v = (const char*)v_cache_dev; a.v_ps = vc_page; a.v_ts = vc_token; a.v_hs = vc_head; a.out = (char*)out_dev; a.o_ts = o_token; a.o_hs = o_head; a.lse = lse_dev;
    a.q_starts = q_starts_dev; a.n_seq = n_branches; a.q_tokens = (int)q_tokens; a.own_pages = own_pages_dev; a.own_ld = own_ld; a.own_lens = own_lens_dev; a.own_width = own_width;
    a.prefix_pages = prefix_pages_dev; a.prefix_ld = prefix_ld; a.prefix_lens = prefix_lens_dev; a.prefix_width = prefix_width; a.group_starts = group_starts_dev; a.n_groups = n_groups;
    a.n_pages = n_pages; a.heads = heads; a.each = heads / kv_heads; a.block = block; a.scale = scale * 1.44269504089f;
    if (!plan_tiles(a, kv_heads)) return BB_EINVAL;
    if (type == BB_BF16) launch_kv<__bf16>(a, kv_heads, head_dim, (hipStream_t)hip_stream); else launch_kv<half_t>(a, kv_heads, head_dim, (hipStream_t)hip_stream);
    return hipGetLastError() == hipSuccess ? BB_OK : BB_EHIP;
}
