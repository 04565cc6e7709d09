// Rows quantised to int8 with one fp32 scale each: q[c] = rint(127 y[c] / max |y|), ties to even, scale = max |y| / 127, where y is
// the row itself (bb_quantize_rows), RMSNorm of it with the residual's addition (bb_rmsnorm_quantize) or SiLU(gate) * up
// (bb_swiglu_quantize).
//
// The codes are those of the formula in 64 bits whatever the launch.  The norm's 1 / rms is a positive factor of the whole row and falls out
// of y / max |y|, so they depend on p = h * gain alone, which a double holds exactly.  Values are kept in fp32 (v), which for 16-bit types is p
// itself, else off by V_ERR at most; t = v * (127 / max) is off by 127 (V_ERR + 2^-23).  Only where t is that near to a border between two
// codes is it taken again, in double (from memory where v does not hold it, a few elements in 10^5), so that a border that is met exactly (half the
// maximum is 63.5) is seen as one.  So is the maximum itself where fp32 does not hold it.  Sums of squares are in double.
//
// What bounds it: memory.  A row is read once and its values stay in registers between the maximum and the codes.  Read + written, bf16: rows of
// 24576 x 4096 53 us (5.7 TB/s), norm with residual of 20480 x 4096 100 (5.9), SwiGLU of 6143 x 12288 76 (5.0: its exponentials beside the loads);
// a large copy reaches 5.1.  One row of 4096: 2.3, 3.0 and 3.4 us; a fill of one value 1.2.
#include "bb_internal.h"
#include <algorithm>
#include <cstdlib>
#include <type_traits>

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

#define QOP_ROWS 0
#define QOP_NORM 1
#define QOP_SWIGLU 2
#define QOP_PANEL 3             // rows of a packed activation panel of two bf16 terms (what attention leaves for the output projection)

struct QuantArgs {
    const void *x, *x2, *gain;      // NORM: x2 = residual (or null); SWIGLU: x = gate, x2 = up
    void* h;                        // NORM: x + residual
    int8_t* q; float* scale;
    long ldx, ldx2, ldh, ldq;
    long rows; int cols;
    double eps;
    const int* live;                // rows that count, on the device (null: all)
    int mt_total;                   // PANEL
};

struct bf16_t { uint16_t v; };
template <class T> static __device__ __forceinline__ float widen(T v) {
    if constexpr (std::is_same_v<T, bf16_t>) return bf16_to_f32(v.v); else return (float)v;
}
template <class T> static __device__ __forceinline__ T narrow(float v) {
    if constexpr (std::is_same_v<T, bf16_t>) {      // (NaN stays NaN: the rounding of its bits could carry it into infinity)
        return bf16_t{v != v ? (uint16_t)0x7FC0 : f32_to_bf16_rne(v)};
    } else return (T)v;
}

// Eight consecutive elements as they lie in memory, taken apart only where they are used: loads of several groups are then on their way together.
template <class T> struct Eight {
    static constexpr int WORDS = 8 * (int)sizeof(T) / 16;
    u32x4 w[WORDS];
    __device__ __forceinline__ float get(int j) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[j >> 2][j & 3]);
        else if constexpr (std::is_same_v<T, bf16_t>) return __uint_as_float(j & 1 ? w[0][j >> 1] & 0xFFFF0000u : w[0][j >> 1] << 16);
        else return (float)__builtin_bit_cast(half_t, (uint16_t)(w[0][j >> 1] >> (16 * (j & 1))));
    }
    __device__ __forceinline__ void set(int j, float v) {
        const T n = narrow<T>(v);
        if constexpr (sizeof(T) == 4) w[j >> 2][j & 3] = __float_as_uint(n);
        else {
            const unsigned b = __builtin_bit_cast(uint16_t, n);
            w[0][j >> 1] = j & 1 ? (w[0][j >> 1] & 0xFFFFu) | b << 16 : (w[0][j >> 1] & 0xFFFF0000u) | b;
        }
    }
    // any alignment that the type itself has
    __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(w, p, sizeof(w)); }
    __device__ __forceinline__ void store(T* p) const { __builtin_memcpy(p, w, sizeof(w)); }
};

// x / (1 + exp(-x)) for x >= SILU_FAR.  exp(-x) = 2^(-x log2 e): the product in two parts, the second (its rounding, and what a float of log2 e
// leaves out) as a factor 1 + part ln 2.  Halves of a last place: 1 for the product's parts, 2 each for the hardware's exp2 and reciprocal, 1 each for
// the factor, the sum, the product with x: 8, and 1 for the product with `up`.
#define SILU_FAR (-87.0f)
#define SILU_FAR_BITS 0xC2AE0000u
static __device__ __forceinline__ float silu(float x) {
    constexpr float L = -1.44269504088896340736f, L_REST = (float)(-1.44269504088896340736 - (double)L);
    const float hi = x * L, lo = fmaf(x, L_REST, fmaf(x, L, -hi)), e0 = __builtin_amdgcn_exp2f(hi);
    const float e = fabsf(hi) < 126.0f ? fmaf(e0, lo * 0.693147180559945309417f, e0) : e0;     // (beyond, infinity times a small part)
    return x * __builtin_amdgcn_rcpf(1.0f + e);
}
// SiLU(x) * up for x < SILU_FAR, where 1 + exp(-x) nears or leaves fp32's range (and its reciprocal is subnormal) although the product with a large `up` is an
// ordinary value: x exp(x) up (1 + exp(x) is 1 to 2^-125), exp(x) as the square of 2^(x log2 e / 2), `up` between its factors, so that nothing leaves the range
// before the value itself does (below x = -174 the value is under 2^-110 whatever `up` is).  Halves of a last place: 2 for each of the two factors, 4 products, 1 for the second
// part's factor: 9.
static __device__ __forceinline__ float silu_far(float x, float up) {
    constexpr float L = 1.44269504088896340736f, L_REST = (float)(1.44269504088896340736 - (double)L);
    const float least = fmaxf(x, -512.0f), hi = least * L, lo = fmaf(least, L_REST, fmaf(least, L, -hi)), e = __builtin_amdgcn_exp2f(0.5f * hi);
    return x * e * up * (e * fmaf(lo, 0.693147180559945309417f, 1.0f));        // (-infinity times 0 is NaN, as in the formula)
}

// What a row's values are, at column c, in 64 bits, from memory (h once it is written).  ZEROS: products with a zero are likely.
template <int OP, class T, bool ZEROS = false> static __device__ __forceinline__ double exact_value(const QuantArgs& a, long row, int c) {
    if constexpr (OP == QOP_PANEL) {
        auto term = [&](int t) { return (double)widen(((const T*)((const u32x4*)a.x + packA_u4((int)row, c >> 3, a.mt_total, t)))[c & 7]); };
        return term(0) + term(1);
    }
    const double x = widen((OP == QOP_NORM && a.x2 ? (const T*)a.h + row * a.ldh : (const T*)a.x + row * a.ldx)[c]);
    if constexpr (OP == QOP_NORM) return x * (double)widen(((const T*)a.gain)[c]);
    if constexpr (OP == QOP_SWIGLU) {
        const double up = widen(((const T*)a.x2 + row * a.ldx2)[c]);
        if (ZEROS && (x == 0.0 || up == 0.0)) return x * up;
        return x / (1.0 + exp(-x)) * up;
    }
    return x;
}

// THREADS lanes share a row (64: a wave each, four rows a workgroup).  G: groups of eight columns a thread keeps, group i of thread t
// being number t + i THREADS of the row; G = 0: longer rows, read again for the codes.  Of the up to seven columns that make no group thread t takes one.
template <int OP, class T, int THREADS, int G>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void quantize_kernel(QuantArgs a) {
    constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1, KEEP = G ? G : 1;
    constexpr bool V_EXACT = OP == QOP_ROWS || OP == QOP_PANEL || (OP == QOP_NORM && sizeof(T) == 2);
    constexpr bool TOP_IN_DOUBLE = OP == QOP_NORM && std::is_same_v<T, float>;      // v does not hold the maximum, but its factors are at hand
    // 2^-24: one rounding; SiLU * up: 9 of them, allowed 16
    constexpr float V_ERR = OP == QOP_SWIGLU ? 0x1p-20f : 0x1p-24f, NEAR = 0.5f - 127.0f * (V_ERR + 0x1p-22f);
    const int t = threadIdx.x % THREADS;
    const long row = (long)blockIdx.x * ROWS + threadIdx.x / THREADS;
    if ((ROWS > 1 && row >= a.rows) || (a.live && row >= *a.live)) return;          // (whole waves; no barrier follows where rows share a workgroup)
    const T* x = (const T*)a.x + row * a.ldx;
    const T* x2 = a.x2 ? (const T*)a.x2 + row * a.ldx2 : nullptr;
    const T* gain = (const T*)a.gain;
    T* h = (T*)a.h + row * a.ldh;
    const int cols = a.cols, groups = cols >> 3, c_tail = groups * 8 + t;
    const bool tail = t < (cols & 7);

    float v[KEEP][8], v_tail = 0.f;
    double ss = 0.0, top2 = 0.0;
    unsigned top_bits = 0u;                                 // as whole numbers |v| are in order, infinity and NaN at the end
    unsigned low_bits = 0u;                                 // of the lowest gate: as whole numbers negative values come after all others, the lowest last
    Eight<T> kx[KEEP], ky[OP == QOP_ROWS ? 1 : KEEP], kr[OP == QOP_NORM ? KEEP : 1];
    auto fetch = [&](int i, int g, bool again) {            // (nothing that would make a load wait for the one before it)
        const int c = g * 8;
        if constexpr (OP == QOP_PANEL) {
            kx[i].load((const T*)((const u32x4*)a.x + packA_u4((int)row, g, a.mt_total, 0)));
            ky[i].load((const T*)((const u32x4*)a.x + packA_u4((int)row, g, a.mt_total, 1)));
            return;
        }
        kx[i].load((OP == QOP_NORM && again && x2 ? h : x) + c);
        if constexpr (OP == QOP_SWIGLU) ky[i].load(x2 + c);
        if constexpr (OP == QOP_NORM) {
            ky[i].load(gain + c);
            if (x2 && !again) kr[i].load(x2 + c);
        }
    };
    auto value = [&](float f, float w, bool far) {          // far: a gate below SILU_FAR
        float y = f;
        if constexpr (OP == QOP_NORM) {
            y = f * w;
            ss = fma((double)f, (double)f, ss);
            if constexpr (TOP_IN_DOUBLE) top2 = fmax(top2, fabs((double)f * (double)w));
        }
        if constexpr (OP == QOP_SWIGLU) y = far ? silu_far(f, w) : silu(f) * w;
        if constexpr (OP == QOP_PANEL) y = f + w;           // (exact: store_panel8 splits an fp32 value, both terms are multiples of its last place and no larger)
        top_bits = max(top_bits, __float_as_uint(y) & 0x7FFFFFFFu);
        return y;
    };
    auto values = [&](int i, int g, bool again, auto Far) {      // Far: gates below SILU_FAR taken as such; else only noticed
        if constexpr (OP == QOP_NORM)
            if (x2 && !again) {
#pragma unroll
                for (int j = 0; j < 8; ++j) kx[i].set(j, kx[i].get(j) + kr[i].get(j));
                kx[i].store(h + g * 8);
            }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float f = kx[i].get(j);
            if constexpr (OP == QOP_SWIGLU && !decltype(Far)::value) low_bits = max(low_bits, __float_as_uint(f));
            v[i][j] = value(f, OP == QOP_ROWS ? 0.f : ky[OP == QOP_ROWS ? 0 : i].get(j), decltype(Far)::value && f < SILU_FAR);
        }
    };
    const std::false_type near{};
    const std::true_type far{};
    if constexpr (G > 0) {
#pragma unroll
        for (int i = 0; i < G; ++i) if (t + i * THREADS < groups) fetch(i, t + i * THREADS, false);
    }
    if (tail) {
        float f = widen(x[c_tail]);
        if constexpr (OP == QOP_NORM)
            if (x2) {
                const T n = narrow<T>(f + widen(x2[c_tail]));
                h[c_tail] = n;
                f = widen(n);
            }
        v_tail = value(f, OP == QOP_NORM ? widen(gain[c_tail]) : OP == QOP_SWIGLU ? widen(x2[c_tail]) : 0.f, f < SILU_FAR);
    }
    if constexpr (G > 0) {
#pragma unroll
        for (int i = 0; i < G; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
            if (t + i * THREADS < groups) values(i, t + i * THREADS, false, near);
        }
    } else
        for (int g = t; g < groups; g += THREADS) { fetch(0, g, false); values(0, g, false, near); }
    // Gates below SILU_FAR are rare: they are only noticed above, and a wave that met one reads its groups again
    // (6143 x 12288 bf16 75 us without any, 125 with some in every row).
    bool careful = false;
    if constexpr (OP == QOP_SWIGLU) {
        careful = __any(low_bits > SILU_FAR_BITS);
        if (__builtin_expect(careful, 0)) {
            top_bits = __float_as_uint(v_tail) & 0x7FFFFFFFu;
            if constexpr (G > 0) {
#pragma unroll
                for (int i = 0; i < G; ++i) if (t + i * THREADS < groups) { fetch(i, t + i * THREADS, true); values(i, t + i * THREADS, true, far); }
            } else
                for (int g = t; g < groups; g += THREADS) { fetch(0, g, true); values(0, g, true, far); }
        }
    }
    auto values_again = [&](int g) {                        // (G = 0)
        fetch(0, g, true);
        if (careful) values(0, g, true, far); else values(0, g, true, near);
    };

    // ---- the row's maximum (and sum of squares) ----------------------------------------------------------------------------------------
    __shared__ double sh_ss[16], sh_top[16];
    __shared__ unsigned sh_bits[16];
    auto reduce = [&]() {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            top_bits = max(top_bits, (unsigned)__shfl_xor((int)top_bits, o, 64));
            if constexpr (OP == QOP_NORM) ss += __shfl_xor(ss, o, 64);
            if constexpr (TOP_IN_DOUBLE) top2 = fmax(top2, __shfl_xor(top2, o, 64));
        }
        if constexpr (THREADS > 64) {
            if ((t & 63) == 0) { sh_bits[t >> 6] = top_bits; if (OP == QOP_NORM) sh_ss[t >> 6] = ss; if (TOP_IN_DOUBLE) sh_top[t >> 6] = top2; }
            __syncthreads();
            ss = 0.0;
#pragma unroll
            for (int w = 0; w < THREADS / 64; ++w) {
                top_bits = max(top_bits, sh_bits[w]);
                if constexpr (OP == QOP_NORM) ss += sh_ss[w];
                if constexpr (TOP_IN_DOUBLE) top2 = fmax(top2, sh_top[w]);
            }
        }
    };
    auto reduce_top = [&](double d) {                       // the maximum of d over the row
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) d = fmax(d, __shfl_xor(d, o, 64));
        if constexpr (THREADS > 64) {
            __syncthreads();
            if ((t & 63) == 0) sh_top[t >> 6] = d;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < THREADS / 64; ++w) d = fmax(d, sh_top[w]);
        }
        return d;
    };
    reduce();
    double top = TOP_IN_DOUBLE ? top2 : (double)__uint_as_float(top_bits);
    // Rows so large or small that fp32 products would not do (and those that hold an infinity or a NaN): everything in double.
    const bool hard = !(top_bits > 0x0D800000u && top_bits < 0x71800000u);     // 2^-100, 2^100
    bool bad = false;
    // (zeros that v holds exactly need no second look; a norm's or SwiGLU's products below fp32's range do)
    if (hard && (top_bits != 0u || (OP == QOP_NORM && ss > 0.0) || OP == QOP_SWIGLU)) {
        double d = 0.0;
        int b = 0;
        auto look = [&](int c) {                            // (columns of this thread's own: h is as it wrote it)
            const double y = fabs(exact_value<OP, T, true>(a, row, c));
            b |= !(y < INFINITY);
            d = fmax(d, y);
        };
        // (a row of zeros as gates, which pads a batch, is nothing but zeros: 70 us for 6143 x 12288 of them, 177 with a look at each)
        const bool zeros = OP == QOP_SWIGLU && top_bits == 0u && low_bits == 0u;
        for (int g = zeros ? groups : t; g < groups; g += THREADS)
#pragma unroll 1
            for (int j = 0; j < 8; ++j) look(g * 8 + j);
        if (tail) look(c_tail);
        top = reduce_top(b ? INFINITY : d);
        bad = !(top < INFINITY);
    } else if (OP == QOP_SWIGLU && top_bits != 0u) {        // the largest of those that may be the maximum
        double d = 0.0;
        const float least = (float)top * (1.0f - 4.0f * V_ERR);
        auto look = [&](int i, int g) {
            unsigned near = 0u;
#pragma unroll
            for (int j = 0; j < 8; ++j) near |= fabsf(v[i][j]) >= least ? 1u << j : 0u;
#pragma unroll 1
            for (; near; near &= near - 1u) d = fmax(d, fabs(exact_value<OP, T>(a, row, g * 8 + __ffs((int)near) - 1)));
        };
        if constexpr (G > 0) {
#pragma unroll
            for (int i = 0; i < G; ++i) look(i, t + i * THREADS);       // (groups that do not exist hold zeros)
        } else
            for (int g = t; g < groups; g += THREADS) { values_again(g); look(0, g); }
        if (fabsf(v_tail) >= least) d = fmax(d, fabs(exact_value<OP, T>(a, row, c_tail)));
        top = reduce_top(d);
    }
    if constexpr (OP == QOP_NORM) bad |= !(ss < INFINITY);
    // a row that holds a NaN or an infinity has the scale NaN (and codes 0); one of zeros the scale 0
    if (t == 0) {
        const double rms = OP == QOP_NORM ? sqrt(ss / cols + a.eps) : 1.0;
        a.scale[row] = bad ? NAN : top == 0.0 ? 0.0f : (float)(top / rms / 127.0);
    }

    // ---- the codes ---------------------------------------------------------------------------------------------------------------------
    const bool none = bad || top == 0.0;
    const float per = none || hard ? 0.0f : 127.0f / (float)top;     // (the rounding of top, the quotient and the product: under 2^-22)
    int8_t* q = a.q + row * a.ldq;
    // adding 1.5 * 2^23 rounds to a whole number, whose low byte is the code; far: how far from it, half at a border
    auto code_bits = [&](float y, float& far) {
        const float u = y * per, r = u + 12582912.0f;
        far = fabsf(u - (r - 12582912.0f));
        return __float_as_uint(r);
    };
    auto exact_code = [&](double y) { return (unsigned)(int)rint(127.0 * y / top) & 0xFFu; };
    // For a y that v holds: which side of the border next to u it is on.  Both products are exact.  (16-bit types meet borders often: of
    // normal bf16 values one in 600 is half the row's maximum.)
    auto side_of_border = [&](float y) {
        const float u = y * per, r = rintf(u), border = r + (u > r ? 0.5f : -0.5f);
        const double l = 127.0 * (double)y, b = (double)border * top;
        const float below = border - 0.5f, above = border + 0.5f;
        const float code = l > b ? above : l < b ? below : rintf(border);
        return (unsigned)(int)code & 0xFFu;
    };
    auto codes = [&](int i, int g) {
        unsigned bits[8], out[2];
        float far[8], most = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) { bits[j] = code_bits(v[i][j], far[j]); most = fmaxf(most, far[j]); }
        unsigned again = 0u;            // the codes to take from the values in memory
        if (hard && !none) again = 0xFFu;
        else if (most > NEAR && !none) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (V_EXACT) { if (far[j] > NEAR) bits[j] = side_of_border(v[i][j]); }
                else again |= far[j] > NEAR ? 1u << j : 0u;
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
            out[k] = __builtin_amdgcn_perm(bits[4 * k + 1], bits[4 * k], 0x0C0C0400u) | __builtin_amdgcn_perm(bits[4 * k + 3], bits[4 * k + 2], 0x04000C0Cu);
        if (none) out[0] = out[1] = 0u;
#pragma unroll 1
        for (; again; again &= again - 1u) {
            const int j = __ffs((int)again) - 1, at = 8 * (j & 3);
            const unsigned code = exact_code(exact_value<OP, T>(a, row, g * 8 + j)) << at, mask = ~(0xFFu << at);
            if (j < 4) out[0] = (out[0] & mask) | code; else out[1] = (out[1] & mask) | code;
        }
        __builtin_memcpy(q + g * 8, out, 8);
    };
    if constexpr (G > 0) {
#pragma unroll
        for (int i = 0; i < G; ++i) if (t + i * THREADS < groups) codes(i, t + i * THREADS);
    } else
        for (int g = t; g < groups; g += THREADS) { values_again(g); codes(0, g); }
    if (tail) {
        float far;
        const unsigned b = code_bits(v_tail, far);
        q[c_tail] = (int8_t)(none ? 0u : hard || far > NEAR ? exact_code(exact_value<OP, T>(a, row, c_tail)) : b & 0xFFu);
    }
}

template <int OP, class T, int THREADS, int G> static void launch_body(const QuantArgs& a, hipStream_t s) {
    constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1;
    quantize_kernel<OP, T, THREADS, G><<<dim3((unsigned)((a.rows + ROWS - 1) / ROWS)), THREADS < 256 ? 256 : THREADS, 0, s>>>(a);
}
// Lanes per row: with many rows as few as keep a row in registers without costing occupancy (fewer partial sums to put together), with few
// rows as many as shorten one row's time.  us, bf16 rows: 20480 x 4096 256 lanes 47, 512 54, 64 53; 6143 x 12288 256 lanes 45, 512 43, 1024 47
// (SwiGLU 83, 95, 129); 120 x 12288 1024 lanes 5.1, 512 6.0, 256 8.3; 20480 x 512 64 lanes 9.6, 256 17.
template <int OP, class T> static void launch_quantize(const QuantArgs& a, hipStream_t s) {
    const int groups = a.cols / 8;
    const bool many = a.rows >= 1024;
    if (groups <= 64) launch_body<OP, T, 64, 1>(a, s);
    else if (groups <= 128 && many) launch_body<OP, T, 64, 2>(a, s);
    else if (groups <= 256) launch_body<OP, T, 256, 1>(a, s);
    else if (groups <= 512) { if (many) launch_body<OP, T, 256, 2>(a, s); else launch_body<OP, T, 512, 1>(a, s); }
    else if (groups <= 1024) { if (many) launch_body<OP, T, 256, 4>(a, s); else launch_body<OP, T, 1024, 1>(a, s); }
    else if (groups <= 1536 && many) launch_body<OP, T, 256, 6>(a, s);
    else if (groups <= 2048 && !many) launch_body<OP, T, 1024, 2>(a, s);
    else if (groups <= 2560 && many) launch_body<OP, T, 512, 5>(a, s);
    else if (groups <= 4096) launch_body<OP, T, 1024, 4>(a, s);
    else launch_body<OP, T, 1024, 0>(a, s);
}

// (a launch holds under 2^32 threads: rows by parts)
template <int OP> static int quantize(int type, QuantArgs a, hipStream_t s) {
    const long rows = a.rows, most = 1L << 21, size = type == BB_F32 ? 4 : 2;
    auto skip = [&](const void*& p, long ld) { if (p) p = (const char*)p + most * ld * size; };
    for (long r = 0; r < rows; r += most) {
        a.rows = std::min(most, rows - r);
        switch (type) {
            case BB_F32: launch_quantize<OP, float>(a, s); break;
            case BB_BF16: launch_quantize<OP, bf16_t>(a, s); break;
            default: launch_quantize<OP, half_t>(a, s); break;
        }
        skip(a.x, a.ldx); skip(a.x2, a.ldx2);
        if (a.h) a.h = (char*)a.h + most * a.ldh * size;
        a.q += most * a.ldq; a.scale += most;
    }
    return hipGetLastError() == hipSuccess ? BB_OK : BB_EHIP;
}

// What the three calls refuse alike: an output row has to end before the next begins; elements lie at multiples of their size.
static bool refuse_sizes(int type, long rows, int cols) {
    return (type != BB_F32 && type != BB_BF16 && type != BB_F16) || rows < 0 || rows > BB_QUANTIZE_MAX_ROWS || cols < 1;
}
static bool refuse_out(const void* q, long ldq, const void* scale, long rows, int cols) {
    return !q || !scale || (uintptr_t)scale % 4 || (rows > 1 && ldq < cols);
}
static bool refuse_rows(const void* p, int type, long rows, long ld) {
    return !p || (uintptr_t)p % (type == BB_F32 ? 4 : 2) || (rows > 1 && ld < 0);
}
// Rows that are written (w, ldw >= cols) while others (r) are read: right where they are the same rows, or have no element in common (apart, or between each
// other: column ranges or alternate rows of one tensor).
static bool refuse_overlap(const void* r, long ldr, const void* w, long ldw, long rows, int cols, int type) {
    const long size = type == BB_F32 ? 4 : 2, n = cols * size, r0 = (long)(uintptr_t)r, w0 = (long)(uintptr_t)w;
    if (rows == 1) ldr = ldw = cols;
    if (r0 == w0 && ldr == ldw) return false;
    ldr *= size; ldw *= size;
    const long r1 = r0 + (rows - 1) * ldr + n, w1 = w0 + (rows - 1) * ldw + n;
    if (r1 <= w0 || w1 <= r0) return false;
    if (ldr == ldw) {                                       // (how far a row is from the next one before it)
        const long apart = labs(r0 - w0) % ldw;
        return apart < n || ldw - apart < n;
    }
    if (ldr <= n) {                                         // rows without gaps: a single run
        const long i = std::max(0L, (r0 - w0) / ldw);       // the last row of w that begins at or before it, or the first
        return (w0 + i * ldw < r1 && w0 + i * ldw + n > r0) || (i + 1 < rows && w0 + (i + 1) * ldw < r1);
    }
    for (long i = 0; i < rows; ++i) {
        const long at = w0 + i * ldw, j = at < r0 ? 0 : std::min(rows - 1, (at - r0) / ldr);
        if ((r0 + j * ldr < at + n && at < r0 + j * ldr + n) || (j + 1 < rows && r0 + (j + 1) * ldr < at + n)) return true;
    }
    return false;
}

// The layers of a forward: fp32 rows, of which *live count.
void launch_rmsnorm_quantize(const float* x, float* residual, const float* gain, float eps, int8_t* q, long ldq, float* scale, long rows, int cols,
                             const int* live, hipStream_t s) {
    QuantArgs a{};
    a.x = x; a.ldx = cols; a.x2 = residual; a.ldx2 = cols; a.h = residual; a.ldh = cols; a.gain = gain; a.eps = eps;
    a.q = q; a.ldq = ldq; a.scale = scale; a.rows = rows; a.cols = cols; a.live = live;
    launch_quantize<QOP_NORM, float>(a, s);
}
void launch_swiglu_quantize(const float* gate, const float* up, long ld, int8_t* q, long ldq, float* scale, long rows, int cols, const int* live, hipStream_t s) {
    QuantArgs a{};
    a.x = gate; a.ldx = ld; a.x2 = up; a.ldx2 = ld; a.q = q; a.ldq = ldq; a.scale = scale; a.rows = rows; a.cols = cols; a.live = live;
    launch_quantize<QOP_SWIGLU, float>(a, s);
}
void launch_panel_quantize(const u32x4* Apk, int mt_total, int8_t* q, long ldq, float* scale, long rows, int cols, const int* live, hipStream_t s) {
    QuantArgs a{};
    a.x = Apk; a.mt_total = mt_total; a.q = q; a.ldq = ldq; a.scale = scale; a.rows = rows; a.cols = cols; a.live = live;
    launch_quantize<QOP_PANEL, bf16_t>(a, s);
}

extern "C" int bb_quantize_rows(const void* x_dev, long ldx, int8_t* q_dev, long ldq, float* scale_dev, long rows, int cols, int type, void* hip_stream) {
    if (refuse_sizes(type, rows, cols)) return BB_EINVAL;
    if (rows == 0) return BB_OK;
    if (refuse_out(q_dev, ldq, scale_dev, rows, cols) || refuse_rows(x_dev, type, rows, ldx)) return BB_EINVAL;
    QuantArgs a{};
    a.x = x_dev; a.ldx = ldx; a.q = q_dev; a.ldq = ldq; a.scale = scale_dev; a.rows = rows; a.cols = cols;
    return quantize<QOP_ROWS>(type, a, (hipStream_t)hip_stream);
}

extern "C" int bb_rmsnorm_quantize(const void* x_dev, long ldx, const void* residual_dev, long ldr, void* residual_out_dev, long ldo, const void* gain_dev,
                                   float eps, int8_t* q_dev, long ldq, float* scale_dev, long rows, int cols, int type, void* hip_stream) {
    if (refuse_sizes(type, rows, cols)) return BB_EINVAL;
    if (rows == 0) return BB_OK;
    if (refuse_out(q_dev, ldq, scale_dev, rows, cols) || refuse_rows(x_dev, type, rows, ldx) || refuse_rows(gain_dev, type, rows, 0)) return BB_EINVAL;
    if (!(eps >= 0.f) || !(eps < INFINITY) || !residual_dev != !residual_out_dev) return BB_EINVAL;
    if (residual_dev && (refuse_rows(residual_dev, type, rows, ldr) || refuse_rows(residual_out_dev, type, rows, ldo) || (rows > 1 && ldo < cols) ||
                         refuse_overlap(x_dev, ldx, residual_out_dev, ldo, rows, cols, type) || refuse_overlap(residual_dev, ldr, residual_out_dev, ldo, rows, cols, type)))
        return BB_EINVAL;
    QuantArgs a{};
    a.x = x_dev; a.ldx = ldx; a.x2 = residual_dev; a.ldx2 = ldr; a.h = residual_out_dev; a.ldh = ldo; a.gain = gain_dev; a.eps = eps;
    a.q = q_dev; a.ldq = ldq; a.scale = scale_dev; a.rows = rows; a.cols = cols;
    return quantize<QOP_NORM>(type, a, (hipStream_t)hip_stream);
}

extern "C" int bb_swiglu_quantize(const void* gate_dev, long ldg, const void* up_dev, long ldu, int8_t* q_dev, long ldq, float* scale_dev, long rows,
                                  int cols, int type, void* hip_stream) {
    if (refuse_sizes(type, rows, cols)) return BB_EINVAL;
    if (rows == 0) return BB_OK;
    if (refuse_out(q_dev, ldq, scale_dev, rows, cols) || refuse_rows(gate_dev, type, rows, ldg) || refuse_rows(up_dev, type, rows, ldu)) return BB_EINVAL;
    QuantArgs a{};
    a.x = gate_dev; a.ldx = ldg; a.x2 = up_dev; a.ldx2 = ldu; a.q = q_dev; a.ldq = ldq; a.scale = scale_dev; a.rows = rows; a.cols = cols;
    return quantize<QOP_SWIGLU>(type, a, (hipStream_t)hip_stream);
}

// ---- tests ------------------------------------------------------------------------------------------------------------------------------------
extern "C" int bb_debug_panel_quantize(const float* x_dev, int rows, int cols, void* panel_dev, size_t panel_bytes, int8_t* q_dev, float* scale_dev, const int* live_dev,
                                       void* hip_stream) {
    if (!x_dev || !panel_dev || !q_dev || !scale_dev || rows < 1 || rows > 1 << 20 || cols < 16 || cols > 1 << 20 || cols % 16 || (uintptr_t)panel_dev % 16) return BB_EINVAL;
    const int mt = (rows + 31) / 32;
    if (panel_bytes < (size_t)mt * 32 * ((cols + 63) / 64 * 64) * 2 * BB_SPLIT) return BB_ENOMEM;
    launch_pack_rows(x_dev, rows, cols, (u32x4*)panel_dev, mt, (hipStream_t)hip_stream);
    launch_panel_quantize((const u32x4*)panel_dev, mt, q_dev, cols, scale_dev, rows, cols, live_dev, (hipStream_t)hip_stream);
    return hipGetLastError() == hipSuccess ? BB_OK : BB_EHIP;
}
