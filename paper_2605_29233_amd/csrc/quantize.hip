// Rows quantised to int8 with one fp32 scale each: q[c] = rint(127 y[c] / max |y|), ties to even, scale = max |y| / 127, where y is
// the row itself (bb_quantize_rows), RMSNorm of it with the residual's addition (bb_rmsnorm_quantize) or SiLU(gate) * up
// (bb_swiglu_quantize).
//
// The codes are those of the formula whatever the launch: the norm's 1 / rms is a positive factor of the whole row and falls out of
// y / max |y|, so they depend on p = h * gain alone, which a double holds exactly; 127 p / max |p| is formed in double too, as a
// product with 127 / max |p| and, within 1e-12 of a border between two codes, again as a correctly rounded quotient (a border that
// is met exactly, like half the maximum, is thereby seen as one).  SiLU is computed in fp32: its y is off by a few 2^-24 and a code
// can so differ by one where y is that near to a border.  Sums of squares are in double.
//
// What bounds it: memory.  A row is read once and kept in registers (as it came) between the maximum and the codes.
#include "bb_internal.h"
#include <algorithm>
#include <type_traits>

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

#define QOP_ROWS 0
#define QOP_NORM 1
#define QOP_SWIGLU 2

struct QuantArgs {
    const void *x, *x2, *gain;      // NORM: x2 = residual (or null); SWIGLU: x = gate, x2 = up
    void* h;                        // NORM: x + residual
    int8_t* q; float* scale;
    long ldx, ldx2, ldh, ldq;
    long rows; int cols;
    double eps;
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

// Eight consecutive elements; any alignment that the type itself has (the hardware takes such loads and stores).
template <class T> struct Eight { T e[8]; };
template <class T> static __device__ __forceinline__ Eight<T> load8(const T* p) { Eight<T> r; __builtin_memcpy(&r, p, sizeof(r)); return r; }
template <class T> static __device__ __forceinline__ Eight<T> load8(const T* p, int n) {
    Eight<T> r;
#pragma unroll
    for (int j = 0; j < 8; ++j) r.e[j] = j < n ? p[j] : T{};
    return r;
}

struct RowSums { double top, ss; bool bad; };

// THREADS lanes share a row (64: a wave each, four rows a workgroup).  G: groups of eight columns a thread keeps, group i of thread t
// being number t + i THREADS of the row; G = 0: rows of more than 32768 columns, read a second time for the codes.
template <int OP, class T, int THREADS, int G>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void quantize_kernel(QuantArgs a) {
    constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1, KEEP = G ? G : 1;
    const int t = threadIdx.x % THREADS;
    const long row = (long)blockIdx.x * ROWS + threadIdx.x / THREADS;
    if (ROWS > 1 && row >= a.rows) return;                  // (whole waves; no barrier follows where rows share a workgroup)
    const T* x = (const T*)a.x + row * a.ldx;
    const T* x2 = a.x2 ? (const T*)a.x2 + row * a.ldx2 : nullptr;
    const T* gain = (const T*)a.gain;
    T* h = (T*)a.h + row * a.ldh;
    const int cols = a.cols, groups = (cols + 7) >> 3;

    Eight<T> kx[KEEP], kx2[OP == QOP_SWIGLU ? KEEP : 1], kg[OP == QOP_NORM ? KEEP : 1];
    auto fetch = [&](int i, int g, bool again) {
        const int c = g * 8, n = cols - c;
        auto get = [&](const T* p) { return n >= 8 ? load8(p + c) : load8(p + c, n); };
        kx[i] = get(OP == QOP_NORM && again && x2 ? h : x);
        if constexpr (OP == QOP_SWIGLU) kx2[i] = get(x2);
        if constexpr (OP == QOP_NORM) {
            kg[i] = get(gain);
            if (x2 && !again) {
                const Eight<T> r = get(x2);
#pragma unroll
                for (int j = 0; j < 8; ++j) kx[i].e[j] = narrow<T>(widen(kx[i].e[j]) + widen(r.e[j]));
                if (n >= 8) __builtin_memcpy(h + c, &kx[i], sizeof(kx[i]));
                else for (int j = 0; j < n; ++j) h[c + j] = kx[i].e[j];
            }
        }
    };
    auto value = [&](int i, int j) -> double {
        const float v = widen(kx[i].e[j]);
        if constexpr (OP == QOP_ROWS) return v;
        if constexpr (OP == QOP_NORM) return (double)v * (double)widen(kg[i].e[j]);
        if constexpr (OP == QOP_SWIGLU) return v / (1.0f + expf(-v)) * widen(kx2[i].e[j]);
    };
    RowSums s = {0.0, 0.0, false};
    auto look = [&](int i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const double y = fabs(value(i, j));
            s.bad |= !(y < INFINITY);
            s.top = fmax(s.top, y);
            if constexpr (OP == QOP_NORM) { const double v = widen(kx[i].e[j]); s.ss = fma(v, v, s.ss); }
        }
    };
    if constexpr (G > 0) {
#pragma unroll
        for (int i = 0; i < G; ++i) if (t + i * THREADS < groups) fetch(i, t + i * THREADS, false);
#pragma unroll
        for (int i = 0; i < G; ++i) if (t + i * THREADS < groups) look(i);
    } else
        for (int g = t; g < groups; g += THREADS) { fetch(0, g, false); look(0); }

    int bad = s.bad;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        s.top = fmax(s.top, __shfl_xor(s.top, o, 64));
        if constexpr (OP == QOP_NORM) s.ss += __shfl_xor(s.ss, o, 64);
        bad |= __shfl_xor(bad, o, 64);
    }
    if constexpr (THREADS > 64) {
        __shared__ double tops[THREADS / 64], sums[THREADS / 64];
        __shared__ int bads[THREADS / 64];
        if ((t & 63) == 0) { tops[t >> 6] = s.top; sums[t >> 6] = s.ss; bads[t >> 6] = bad; }
        __syncthreads();
        s.top = 0.0; s.ss = 0.0; bad = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) { s.top = fmax(s.top, tops[w]); s.ss += sums[w]; bad |= bads[w]; }
    }
    // a row that holds a NaN or an infinity has the scale NaN (and codes 0); one of zeros the scale 0
    if constexpr (OP == QOP_NORM) bad |= !(s.ss < INFINITY);
    if (t == 0) {
        const double rms = OP == QOP_NORM ? sqrt(s.ss / cols + a.eps) : 1.0;
        a.scale[row] = bad ? NAN : s.top == 0.0 ? 0.0f : (float)(s.top / rms / 127.0);
    }
    const bool none = bad || s.top == 0.0;
    const double per = none ? 0.0 : 127.0 / s.top;
    int8_t* q = a.q + row * a.ldq;
    auto codes = [&](int i, int g) {
        const int c = g * 8, n = cols - c;
        unsigned out[2] = {0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const double p = none ? 0.0 : value(i, j), u = p * per;
            double r = rint(u);
            if (fabs(u - r) > 0.5 - 1e-12) r = rint(127.0 * p / s.top);
            out[j >> 2] |= ((unsigned)(int)r & 0xFFu) << (8 * (j & 3));
        }
        if (n >= 8) __builtin_memcpy(q + c, out, 8);
        else for (int j = 0; j < n; ++j) q[c + j] = (int8_t)(out[j >> 2] >> (8 * (j & 3)));
    };
    if constexpr (G > 0) {
#pragma unroll
        for (int i = 0; i < G; ++i) if (t + i * THREADS < groups) codes(i, t + i * THREADS);
    } else
        for (int g = t; g < groups; g += THREADS) { fetch(0, g, true); codes(0, g); }
}

template <int OP, class T> static void launch_quantize(const QuantArgs& a, hipStream_t s) {
    const int groups = (a.cols + 7) / 8;
#define QLAUNCH(THREADS, G) quantize_kernel<OP, T, THREADS, G><<<dim3((unsigned)((a.rows + (THREADS < 256 ? 256 / THREADS : 1) - 1) / (THREADS < 256 ? 256 / THREADS : 1))), THREADS < 256 ? 256 : THREADS, 0, s>>>(a)
    if (groups <= 64) QLAUNCH(64, 1);
    else if (groups <= 256) QLAUNCH(256, 1);
    else if (groups <= 512) QLAUNCH(256, 2);
    else if (groups <= 1024) QLAUNCH(1024, 1);
    else if (groups <= 4096) QLAUNCH(1024, 4);
    else QLAUNCH(1024, 0);
#undef QLAUNCH
}

template <int OP> static int quantize(int type, const QuantArgs& a, hipStream_t s) {
    switch (type) {
        case BB_F32: launch_quantize<OP, float>(a, s); break;
        case BB_BF16: launch_quantize<OP, bf16_t>(a, s); break;
        default: launch_quantize<OP, half_t>(a, s); break;
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
    if (residual_dev && (refuse_rows(residual_dev, type, rows, ldr) || refuse_rows(residual_out_dev, type, rows, ldo) || (rows > 1 && ldo < cols))) return BB_EINVAL;
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
