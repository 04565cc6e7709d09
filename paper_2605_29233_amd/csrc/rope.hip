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
};

// A workgroup per token: its angles once, for all heads; then a thread per pair, or per element of what is not turned.
template <class E>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
    __shared__ float2 turn[BB_ROPE_MAX_DIM / 2];
    const int half = a.rot >> 1;
    for (long t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const double p = (double)a.positions[t];
        __syncthreads();
        for (int j = threadIdx.x; j < half; j += 256) {
            double turns = p * a.freqs[j] * 0.15915494309189533577;    // 1 / (2 pi)
            turns -= rint(turns);
            float s, c;
            sincospif(2.f * (float)turns, &s, &c);
            turn[j] = make_float2(c * a.magnitude, s * a.magnitude);
        }
        __syncthreads();
        long k_at = 0, v_at = 0, slot = t;
        if (a.slots) {
            slot = a.slots[t];
            if (slot < 0 || slot >= a.n_slots) slot = -1;           // kept out of the cache
            k_at = (slot >> 6) * a.ko_ps + (slot & 63) * a.ko_ts;
            v_at = (slot >> 6) * a.vo_ps + (slot & 63) * a.vo_ts;
        } else k_at = t * a.ko_ts;
        const int pairs = half + (a.dim - a.rot);
        const int heads = a.q_heads + (slot < 0 ? 0 : a.k_heads);
        for (int i = threadIdx.x; i < heads * pairs; i += 256) {
            const int h = i / pairs, j = i - h * pairs;
            const bool is_q = h < a.q_heads;
            const E* x = is_q ? (const E*)a.q + t * a.q_ts + h * a.q_hs : (const E*)a.k + t * a.k_ts + (h - a.q_heads) * a.k_hs;
            E* y = is_q ? (E*)a.qo + t * a.qo_ts + h * a.qo_hs : (E*)a.ko + k_at + (h - a.q_heads) * a.ko_hs;
            if (j < half) {
                const int e0 = a.interleaved ? 2 * j : j, e1 = a.interleaved ? 2 * j + 1 : j + half;
                const float u = (float)x[e0], w = (float)x[e1];
                const float2 cs = turn[j];
                y[e0] = (E)(u * cs.x - w * cs.y);
                y[e1] = (E)(u * cs.y + w * cs.x);
            } else y[a.rot + j - half] = x[a.rot + j - half];
        }
        if (a.vo && slot >= 0)
            for (int i = threadIdx.x; i < a.k_heads * a.dim; i += 256) {
                const int h = i / a.dim, d = i - h * a.dim;
                ((E*)a.vo)[v_at + h * a.vo_hs + d] = ((const E*)a.v)[t * a.v_ts + h * a.v_hs + d];
            }
    }
}

static int launch_rope(const RopeArgs& a, int type, hipStream_t s) {
    const unsigned grid = (unsigned)std::min<long>(a.tokens, 1 << 20);
    if (type == BB_F32) rope_kernel<float><<<grid, 256, 0, s>>>(a);
    else if (type == BB_BF16) rope_kernel<__bf16><<<grid, 256, 0, s>>>(a);
    else rope_kernel<half_t><<<grid, 256, 0, s>>>(a);
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

static bool refuse_turn(const int32_t* positions, const double* freqs, int rot, float magnitude, long tokens, int q_heads, int kv_heads, int dim, int type) {
    return (type != BB_F32 && type != BB_BF16 && type != BB_F16) || dim < 1 || dim > BB_ROPE_MAX_DIM || rot < 0 || rot > dim || rot % 2 || tokens < 0 || tokens > BB_MAX_TOKENS ||
           q_heads < 0 || kv_heads < 0 || q_heads > BB_MAX_HEADS || kv_heads > BB_MAX_HEADS || !(fabsf(magnitude) < INFINITY) ||
           (tokens > 0 && (!positions || (uintptr_t)positions % 4 || (rot > 0 && (!freqs || (uintptr_t)freqs % 8))));
}

extern "C" int bb_rope(const void* q_dev, long q_token, long q_head, void* q_out_dev, long qo_token, long qo_head, int q_heads, const void* k_dev, long k_token, long k_head,
                       void* k_out_dev, long ko_token, long ko_head, int k_heads, const int32_t* positions_dev, const double* freqs_dev, int rot, int interleaved,
                       float magnitude, long tokens, int head_dim, int type, void* hip_stream) {
    if (refuse_turn(positions_dev, freqs_dev, rot, magnitude, tokens, q_heads, k_heads, head_dim, type)) return BB_EINVAL;
    if (tokens == 0 || q_heads + k_heads == 0) return BB_OK;
    const int size = type == BB_F32 ? 4 : 2;
    const HeadView q = heads_view(q_dev, tokens, q_token, q_heads, q_head, head_dim, size), k = heads_view(k_dev, tokens, k_token, k_heads, k_head, head_dim, size);
    const HeadView qo = heads_view(q_out_dev, tokens, qo_token, q_heads, qo_head, head_dim, size), ko = heads_view(k_out_dev, tokens, ko_token, k_heads, ko_head, head_dim, size);
    if (q_heads && (refuse_view(q) || refuse_out_view(qo) || (!same_rows(q, qo) && overlap(q, qo)))) return BB_EINVAL;
    if (k_heads && (refuse_view(k) || refuse_out_view(ko) || (!same_rows(k, ko) && overlap(k, ko)))) return BB_EINVAL;
    if (q_heads && k_heads && (overlap(qo, ko) || overlap(q, ko) || overlap(k, qo))) return BB_EINVAL;
    RopeArgs a{};
    a.q = (const char*)q_dev; a.q_ts = q_token; a.q_hs = q_head; a.qo = (char*)q_out_dev; a.qo_ts = qo_token; a.qo_hs = qo_head; a.q_heads = q_heads;
    a.k = (const char*)k_dev; a.k_ts = k_token; a.k_hs = k_head; a.ko = (char*)k_out_dev; a.ko_ts = ko_token; a.ko_hs = ko_head; a.k_heads = k_heads;
    a.positions = positions_dev; a.freqs = freqs_dev; a.rot = rot; a.interleaved = interleaved; a.magnitude = magnitude; a.tokens = tokens; a.dim = head_dim;
    return launch_rope(a, type, (hipStream_t)hip_stream);
}

extern "C" int bb_rope_append(const void* q_dev, long q_token, long q_head, void* q_out_dev, long qo_token, long qo_head, int q_heads, const void* k_dev, long k_token, long k_head,
                              const void* v_dev, long v_token, long v_head, int kv_heads, const int32_t* positions_dev, const double* freqs_dev, int rot, int interleaved,
                              float magnitude, const int32_t* slots_dev, void* k_cache_dev, long kc_page, long kc_head, long kc_token, void* v_cache_dev, long vc_page,
                              long vc_head, long vc_token, int n_pages, long tokens, int head_dim, int type, void* hip_stream) {
    if (refuse_turn(positions_dev, freqs_dev, rot, magnitude, tokens, q_heads, kv_heads, head_dim, type) || kv_heads < 1 || n_pages < 1 || n_pages > BB_MAX_PAGES) return BB_EINVAL;
    if (tokens == 0) return BB_OK;
    const int size = type == BB_F32 ? 4 : 2;
    const HeadView q = heads_view(q_dev, tokens, q_token, q_heads, q_head, head_dim, size), qo = heads_view(q_out_dev, tokens, qo_token, q_heads, qo_head, head_dim, size);
    const HeadView k = heads_view(k_dev, tokens, k_token, kv_heads, k_head, head_dim, size), v = heads_view(v_dev, tokens, v_token, kv_heads, v_head, head_dim, size);
    const HeadView kc = pages_view(k_cache_dev, n_pages, kc_page, kv_heads, kc_head, kc_token, head_dim, size);
    const HeadView vc = pages_view(v_cache_dev, n_pages, vc_page, kv_heads, vc_head, vc_token, head_dim, size);
    if (!slots_dev || (uintptr_t)slots_dev % 4 || refuse_view(k) || refuse_view(v) || refuse_out_view(kc) || refuse_out_view(vc)) return BB_EINVAL;
    if (overlap(kc, vc) || overlap(kc, k) || overlap(kc, v) || overlap(vc, k) || overlap(vc, v)) return BB_EINVAL;
    if (q_heads && (refuse_view(q) || refuse_out_view(qo) || (!same_rows(q, qo) && overlap(q, qo)) || overlap(qo, k) || overlap(qo, v) || overlap(qo, kc) || overlap(qo, vc) ||
                    overlap(q, kc) || overlap(q, vc))) return BB_EINVAL;
    RopeArgs a{};
    a.q = (const char*)q_dev; a.q_ts = q_token; a.q_hs = q_head; a.qo = (char*)q_out_dev; a.qo_ts = qo_token; a.qo_hs = qo_head; a.q_heads = q_heads;
    a.k = (const char*)k_dev; a.k_ts = k_token; a.k_hs = k_head; a.ko = (char*)k_cache_dev; a.ko_ps = kc_page; a.ko_ts = kc_token; a.ko_hs = kc_head; a.k_heads = kv_heads;
    a.v = (const char*)v_dev; a.v_ts = v_token; a.v_hs = v_head; a.vo = (char*)v_cache_dev; a.vo_ps = vc_page; a.vo_ts = vc_token; a.vo_hs = vc_head;
    a.positions = positions_dev; a.freqs = freqs_dev; a.rot = rot; a.interleaved = interleaved; a.magnitude = magnitude; a.slots = slots_dev; a.n_slots = (long)n_pages * 64;
    a.tokens = tokens; a.dim = head_dim;
    return launch_rope(a, type, (hipStream_t)hip_stream);
}
