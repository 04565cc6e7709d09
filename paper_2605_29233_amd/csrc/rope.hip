// Rotary positions: of a head's first `rot` elements pair j, (x[j], x[j + rot/2]) or (x[2j], x[2j+1]), is turned by the angle position * f_j,
//   (a, b) -> (a cos - b sin, a sin + b cos) * magnitude,
// the rest of the head stays as it is.  With a cache the turned keys and the values go to their tokens' slots (bb_rope_append).
//
// The angle is taken in 64 bits: at position 2^20 an fp32 product is off by up to 0.06 rad.  What is left after whole turns is below half a turn and is
// exact enough in fp32 (2^-25 turns) for sine and cosine there.  The turn itself is in fp32, rounded once to the rows' type.
#include "heads.h"

struct RopeArgs {
    const char *q, *k, *v; char *qo, *ko, *vo;      // vo: null without a cache
    long q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, qo_ts, qo_hs, ko_ps, ko_ts, ko_hs, vo_ps, vo_ts, vo_hs;    // (ko_ps, vo_ps: between a cache's pages)
    const int *positions, *slots; const double* freqs;
    long tokens, n_slots;
    int q_heads, k_heads, dim, rot, interleaved;
    float magnitude;
    // pieces: units of a token and of a head, with 2^32 / them rounded up; tokens of a workgroup, units that it takes of them
    int units, head_units, per_group, per_slice; unsigned by_units, by_head;
};
#define ROPE_TURNS 1024

static __device__ __forceinline__ float2 turn_of(double position, double freq, float magnitude) {
    double turns = position * freq * 0.15915494309189533577;           // 1 / (2 pi)
    turns -= rint(turns);
    float s, c;
    sincospif(2.f * (float)turns, &s, &c);
    return make_float2(c * magnitude, s * magnitude);
}
// The tokens of a slot: where its key and value go.
struct RopePlace { long k_at, v_at; bool kept; };
static __device__ __forceinline__ RopePlace place_of(const RopeArgs& a, long t) {
    if (!a.slots) return {t * a.ko_ts, 0, true};
    const long slot = a.slots[t];
    if (slot < 0 || slot >= a.n_slots) return {0, 0, false};           // kept out of the cache
    return {(slot >> 6) * a.ko_ps + (slot & 63) * a.ko_ts, (slot >> 6) * a.vo_ps + (slot & 63) * a.vo_ts, true};
}

// Rows of 16-byte pieces.  A unit is a piece and the one it is turned with (half: half the turned range further on; interleaved: a piece holds its pairs), or a piece of what is
// not turned; values move in the same units.  A thread takes units of all its workgroup's tokens' heads, its loads on their way while the angles are made.
// Memory bounds it where there is much: 20480 tokens of 32 heads of 128 bf16 into a cache 191 us, 5.3 TB/s of 1.0 GB (a copy of 1 GiB runs at 5.1; element by element,
// as below, 466 us).  Little (one token 2.7 us, 112 of 28 heads 3.3) is a launch, the position's load and its angles' 64-bit product behind one another.
template <class E, bool INTER> __global__ __launch_bounds__(256) void rope_pieces_kernel(RopeArgs a) {
    constexpr int VEC = 16 / sizeof(E), AT_ONCE = 4;
    typedef E vec __attribute__((ext_vector_type(VEC)));
    __shared__ __attribute__((aligned(16))) float2 turn[ROPE_TURNS];
    const int half = a.rot >> 1, turned = INTER ? a.rot / VEC : half / VEC;
    const long t0 = (long)blockIdx.x * a.per_group;
    const int tokens = (int)min((long)a.per_group, a.tokens - t0), units = a.units, all = tokens * units;
    const int from = blockIdx.y * a.per_slice, to = min(from + a.per_slice, all);
    bool first = true;
    for (int i0 = from; i0 < to; i0 += 256 * AT_ONCE) {
        vec x[AT_ONCE][2];
        E *y[AT_ONCE];
        int pair[AT_ONCE];                                          // which turns; -1: a copy of both, -2: of the first piece, -3: nothing
#pragma unroll
        for (int n = 0; n < AT_ONCE; ++n) {
            const int i = i0 + n * 256 + (int)threadIdx.x;
            pair[n] = -3;
            if (i >= to) continue;
            const int tk = (int)__umulhi(i, a.by_units), in = i - tk * units, h = (int)__umulhi(in, a.by_head), j = in - h * a.head_units;
            const long t = t0 + tk;
            const int kind = h < a.q_heads ? 0 : h < a.q_heads + a.k_heads ? 1 : 2;
            const RopePlace at = kind ? place_of(a, t) : RopePlace{};
            if (kind && !at.kept) continue;
            const int hk = h - a.q_heads - (kind == 2 ? a.k_heads : 0);
            const E* src = kind == 0 ? (const E*)a.q + t * a.q_ts + h * a.q_hs : kind == 1 ? (const E*)a.k + t * a.k_ts + hk * a.k_hs : (const E*)a.v + t * a.v_ts + hk * a.v_hs;
            E* dst = kind == 0 ? (E*)a.qo + t * a.qo_ts + h * a.qo_hs : kind == 1 ? (E*)a.ko + at.k_at + hk * a.ko_hs : (E*)a.vo + at.v_at + hk * a.vo_hs;
            const bool turn_it = j < turned;
            const int e = turn_it ? j * VEC : a.rot + (j - turned) * VEC;
            y[n] = dst + e;
            x[n][0] = *reinterpret_cast<const vec*>(src + e);
            if (!INTER && turn_it) x[n][1] = *reinterpret_cast<const vec*>(src + e + half);
            pair[n] = !turn_it ? -2 : kind == 2 ? (INTER ? -2 : -1) : tk * half + (INTER ? e >> 1 : e);
        }
        if (first) {
            for (int i = threadIdx.x; i < tokens * half; i += 256) {
                const int tk = i / half;
                turn[i] = turn_of((double)a.positions[t0 + tk], a.freqs[i - tk * half], a.magnitude);
            }
            __syncthreads();
            first = false;
        }
#pragma unroll
        for (int n = 0; n < AT_ONCE; ++n) {
            if (pair[n] == -3) continue;
            vec u = x[n][0], w = x[n][1];
            if (pair[n] >= 0) {
                const float2* cs = turn + pair[n];
                if constexpr (INTER) {
#pragma unroll
                    for (int k = 0; k < VEC / 2; ++k) {
                        const float p = (float)u[2 * k], q = (float)u[2 * k + 1];
                        u[2 * k] = (E)(p * cs[k].x - q * cs[k].y);
                        u[2 * k + 1] = (E)(p * cs[k].y + q * cs[k].x);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < VEC; ++k) {
                        const float p = (float)u[k], q = (float)w[k];
                        u[k] = (E)(p * cs[k].x - q * cs[k].y);
                        w[k] = (E)(p * cs[k].y + q * cs[k].x);
                    }
                }
            }
            *reinterpret_cast<vec*>(y[n]) = u;
            if (!INTER && pair[n] >= -1) *reinterpret_cast<vec*>(y[n] + half) = w;
        }
    }
}

// Rows of any alignment, any number of elements: a workgroup per token, a thread per pair, or per element of what is not turned.
template <class E>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
    __shared__ float2 turn[BB_ROPE_MAX_DIM / 2];
    const int half = a.rot >> 1;
    for (long t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const double p = (double)a.positions[t];
        __syncthreads();
        for (int j = threadIdx.x; j < half; j += 256) turn[j] = turn_of(p, a.freqs[j], a.magnitude);
        __syncthreads();
        const RopePlace at = place_of(a, t);
        const int pairs = half + (a.dim - a.rot);
        const int heads = a.q_heads + (at.kept ? a.k_heads : 0);
        for (int i = threadIdx.x; i < heads * pairs; i += 256) {
            const int h = i / pairs, j = i - h * pairs;
            const bool is_q = h < a.q_heads;
            const E* x = is_q ? (const E*)a.q + t * a.q_ts + h * a.q_hs : (const E*)a.k + t * a.k_ts + (h - a.q_heads) * a.k_hs;
            E* y = is_q ? (E*)a.qo + t * a.qo_ts + h * a.qo_hs : (E*)a.ko + at.k_at + (h - a.q_heads) * a.ko_hs;
            if (j < half) {
                const int e0 = a.interleaved ? 2 * j : j, e1 = a.interleaved ? 2 * j + 1 : j + half;
                const float u = (float)x[e0], w = (float)x[e1];
                const float2 cs = turn[j];
                y[e0] = (E)(u * cs.x - w * cs.y);
                y[e1] = (E)(u * cs.y + w * cs.x);
            } else y[a.rot + j - half] = x[a.rot + j - half];
        }
        if (a.vo && at.kept)
            for (int i = threadIdx.x; i < a.k_heads * a.dim; i += 256) {
                const int h = i / a.dim, d = i - h * a.dim;
                ((E*)a.vo)[at.v_at + h * a.vo_hs + d] = ((const E*)a.v)[t * a.v_ts + h * a.v_hs + d];
            }
    }
}

// Units are numbered below 2^16, so that a product with 2^32 / n rounded up divides them by n exactly (n up to 2^16).
#define ROPE_MOST_UNITS 65536
#define ROPE_MOST_GROUPS (1 << 20)          // of tokens, a launch (one of 2^24 workgroups of 256 threads would be refused)
template <class E> static void launch_rope(RopeArgs& a, hipStream_t s) {
    constexpr int VEC = 16 / sizeof(E);
    const int turned = a.interleaved ? a.rot / VEC : a.rot / 2 / VEC, rest = (a.dim - a.rot) / VEC, heads = a.q_heads + a.k_heads * (a.vo ? 2 : 1);
    const bool whole = a.dim % VEC == 0 && (a.rot / (a.interleaved ? 1 : 2)) % VEC == 0;
    const long units = (long)heads * (turned + rest);
    auto aligned = [&](const void* p, long s0, long s1, long s2) { return (uintptr_t)p % 16 == 0 && s0 % VEC == 0 && s1 % VEC == 0 && s2 % VEC == 0; };
    if (whole && units <= ROPE_MOST_UNITS && (!a.q_heads || (aligned(a.q, a.q_ts, a.q_hs, 0) && aligned(a.qo, a.qo_ts, a.qo_hs, 0))) &&
        (!a.k_heads || (aligned(a.k, a.k_ts, a.k_hs, 0) && aligned(a.ko, a.ko_ps, a.ko_ts, a.ko_hs))) &&
        (!a.vo || (aligned(a.v, a.v_ts, a.v_hs, 0) && aligned(a.vo, a.vo_ps, a.vo_ts, a.vo_hs)))) {
        // one thread a unit while there are few; four, or more, where the chip is full
        a.head_units = turned + rest; a.units = (int)units;
        a.per_group = (int)std::max(1L, std::min<long>(256 / units, a.rot ? ROPE_TURNS / (a.rot / 2) : 256));
        const long at_once = (long)ROPE_MOST_GROUPS * a.per_group, groups = (std::min(a.tokens, at_once) + a.per_group - 1) / a.per_group, in_group = a.per_group * units;
        const long slices = std::max(1L, std::min((in_group + 255) / 256, 1024 / groups));
        a.per_slice = (int)((in_group + slices - 1) / slices + 255) / 256 * 256;
        a.by_units = units > 1 ? (unsigned)((0x100000000ull + units - 1) / units) : 0;
        a.by_head = a.head_units > 1 ? (unsigned)((0x100000000ull + a.head_units - 1) / a.head_units) : 0;
        if (units > 1 && a.head_units > 1) {
            const long all = a.tokens;
            for (long t = 0; t < all; t += at_once) {
                a.tokens = std::min(all - t, at_once);
                const dim3 grid((unsigned)((a.tokens + a.per_group - 1) / a.per_group), (unsigned)((in_group + a.per_slice - 1) / a.per_slice));
                if (a.interleaved) rope_pieces_kernel<E, true><<<grid, 256, 0, s>>>(a); else rope_pieces_kernel<E, false><<<grid, 256, 0, s>>>(a);
                if (all - t <= at_once) return;
                const long bytes = at_once * (long)sizeof(E);
                a.q += a.q_ts * bytes; a.qo += a.qo_ts * bytes; a.k += a.k_ts * bytes; a.v += a.v_ts * bytes;
                a.positions += at_once;
                if (a.slots) a.slots += at_once; else a.ko += a.ko_ts * bytes;
            }
        }
    }
    rope_kernel<E><<<(unsigned)std::min<long>(a.tokens, 1 << 20), 256, 0, s>>>(a);
}
static int launch_rope(RopeArgs& a, int type, hipStream_t s) {
    if (a.tokens == 1) a.q_ts = a.k_ts = a.v_ts = a.qo_ts = 0;             // (a single token, or head, has no next)
    if (a.q_heads == 1) a.q_hs = a.qo_hs = 0;
    if (a.k_heads == 1) a.k_hs = a.ko_hs = a.v_hs = a.vo_hs = 0;
    if (!a.slots && a.tokens == 1) a.ko_ts = 0;
    if (type == BB_F32) launch_rope<float>(a, s);
    else if (type == BB_BF16) launch_rope<__bf16>(a, s);
    else launch_rope<half_t>(a, s);
    return hipGetLastError() == hipSuccess ? BB_OK : BB_EHIP;
}

extern "C" int bb_rope_frequencies(double* freqs_host, int rot, double base, double factor, double context, double low, double high) {
    if (!freqs_host || rot < 2 || rot > BB_ROPE_MAX_DIM || rot % 2 || !(base > 0) || !(base < INFINITY) || !(factor > 0) || !(factor < INFINITY) || !(context >= 0) ||
        !(context < INFINITY) || (context > 0 && !(low < high)))
        return BB_EINVAL;
    for (int j = 0; j < rot / 2; ++j) {
        const double f = pow(base, -2.0 * j / rot);
        double keep = 0;
        if (context > 0) keep = std::min(1.0, std::max(0.0, (context * f / 6.283185307179586477 - low) / (high - low)));
        freqs_host[j] = f * keep + f / factor * (1 - keep);
    }
    return BB_OK;
}

// What both entries have in common.
static bool refuse_turn(const int32_t* positions, const double* freqs, long rot, double magnitude, long tokens, long q_heads, long kv_heads, long dim, long type) {
    return (type != BB_F32 && type != BB_BF16 && type != BB_F16) || dim < 1 || dim > BB_ROPE_MAX_DIM || rot < 0 || rot > dim || rot % 2 || tokens < 0 || tokens > BB_MAX_TOKENS ||
           q_heads < 0 || kv_heads < 0 || q_heads > BB_MAX_HEADS || kv_heads > BB_MAX_HEADS || !(fabs(magnitude) <= 3e38) ||
           (tokens > 0 && (!positions || (uintptr_t)positions % 4 || (rot > 0 && (!freqs || (uintptr_t)freqs % 8))));
}
template <class A> static void common_args(RopeArgs& a, const A* x) {
    a.q = (const char*)x->q; a.q_ts = x->q_token; a.q_hs = x->q_head; a.qo = (char*)x->q_out; a.qo_ts = x->qo_token; a.qo_hs = x->qo_head; a.q_heads = (int)x->q_heads;
    a.k = (const char*)x->k; a.k_ts = x->k_token; a.k_hs = x->k_head;
    a.positions = x->positions; a.freqs = x->freqs; a.rot = (int)x->rot; a.interleaved = x->interleaved != 0; a.magnitude = (float)x->magnitude; a.tokens = x->tokens; a.dim = (int)x->head_dim;
}

extern "C" int bb_rope(const bb_rope_args* x, void* hip_stream) {
    if (!x || refuse_turn(x->positions, x->freqs, x->rot, x->magnitude, x->tokens, x->q_heads, x->k_heads, x->head_dim, x->type)) return BB_EINVAL;
    if (x->tokens == 0 || x->q_heads + x->k_heads == 0) return BB_OK;
    const int size = x->type == BB_F32 ? 4 : 2, dim = (int)x->head_dim;
    const HeadView q = heads_view(x->q, x->tokens, x->q_token, (int)x->q_heads, x->q_head, dim, size), qo = heads_view(x->q_out, x->tokens, x->qo_token, (int)x->q_heads, x->qo_head, dim, size);
    const HeadView k = heads_view(x->k, x->tokens, x->k_token, (int)x->k_heads, x->k_head, dim, size), ko = heads_view(x->k_out, x->tokens, x->ko_token, (int)x->k_heads, x->ko_head, dim, size);
    if (x->q_heads && (refuse_view(q) || refuse_out_view(qo) || (!same_rows(q, qo) && overlap(q, qo)))) return BB_EINVAL;
    if (x->k_heads && (refuse_view(k) || refuse_out_view(ko) || (!same_rows(k, ko) && overlap(k, ko)))) return BB_EINVAL;
    if (x->q_heads && x->k_heads && (overlap(qo, ko) || overlap(q, ko) || overlap(k, qo))) return BB_EINVAL;
    RopeArgs a{};
    common_args(a, x);
    a.ko = (char*)x->k_out; a.ko_ts = x->ko_token; a.ko_hs = x->ko_head; a.k_heads = (int)x->k_heads;
    return launch_rope(a, (int)x->type, (hipStream_t)hip_stream);
}

extern "C" int bb_rope_append(const bb_rope_append_args* x, void* hip_stream) {
    if (!x || refuse_turn(x->positions, x->freqs, x->rot, x->magnitude, x->tokens, x->q_heads, x->kv_heads, x->head_dim, x->type) || x->kv_heads < 1 || x->pages < 1 || x->pages > BB_MAX_PAGES)
        return BB_EINVAL;
    if (x->tokens == 0) return BB_OK;
    const int size = x->type == BB_F32 ? 4 : 2, dim = (int)x->head_dim, kv = (int)x->kv_heads;
    const HeadView q = heads_view(x->q, x->tokens, x->q_token, (int)x->q_heads, x->q_head, dim, size), qo = heads_view(x->q_out, x->tokens, x->qo_token, (int)x->q_heads, x->qo_head, dim, size);
    const HeadView k = heads_view(x->k, x->tokens, x->k_token, kv, x->k_head, dim, size), v = heads_view(x->v, x->tokens, x->v_token, kv, x->v_head, dim, size);
    const HeadView kc = pages_view(x->k_cache, x->pages, x->kc_page, kv, x->kc_head, x->kc_token, dim, size), vc = pages_view(x->v_cache, x->pages, x->vc_page, kv, x->vc_head, x->vc_token, dim, size);
    if (!x->slots || (uintptr_t)x->slots % 4 || refuse_view(k) || refuse_view(v) || refuse_out_view(kc) || refuse_out_view(vc)) return BB_EINVAL;
    if (overlap(kc, vc) || overlap(kc, k) || overlap(kc, v) || overlap(vc, k) || overlap(vc, v)) return BB_EINVAL;
    if (x->q_heads && (refuse_view(q) || refuse_out_view(qo) || (!same_rows(q, qo) && overlap(q, qo)) || overlap(qo, k) || overlap(qo, v) || overlap(qo, kc) || overlap(qo, vc) ||
                       overlap(q, kc) || overlap(q, vc))) return BB_EINVAL;
    RopeArgs a{};
    common_args(a, x);
    a.ko = (char*)x->k_cache; a.ko_ps = x->kc_page; a.ko_ts = x->kc_token; a.ko_hs = x->kc_head; a.k_heads = kv;
    a.v = (const char*)x->v; a.v_ts = x->v_token; a.v_hs = x->v_head; a.vo = (char*)x->v_cache; a.vo_ps = x->vc_page; a.vo_ts = x->vc_token; a.vo_hs = x->vc_head;
    a.slots = x->slots; a.n_slots = x->pages * BB_PAGE_TOKENS;
    return launch_rope(a, (int)x->type, (hipStream_t)hip_stream);
}
