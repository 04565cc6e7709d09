// bb_gemm_int8: C[m][n] = (sum_k A[m][k] W[n][k]) * a_scale[m] * w_scale[n] + bias[n], A and W int8, both with k contiguous.
//
// The sum is exact (int32; K <= 131071 keeps it below 2^31 even for codes of -128), so results do not depend on the tile, the split
// of k or the order; it is rounded to fp32 once, scaled in fp32 and rounded to C's type.
//
// MFMA operands: the matrix cores take 16 rows x 64 k, lane l holding the 16 bytes k = 16 (l / 16) .. + 15 of row l % 16, so row-major
// operands need no re-tiling: 16-byte pieces of their rows are what a lane wants.  W is the first operand: a lane then holds four
// consecutive columns of one row of C.
#include "bb_internal.h"
#include <algorithm>

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct GemmInt8Args {
    const int8_t *A, *W; const float *sa, *sw, *bias; void* C;
    long lda, ldw, ldc;
    int M, N, K, type;
};

// Four consecutive columns of a row of C, as far as they exist.
static __device__ __forceinline__ void store_c4(const GemmInt8Args& a, int m, int n, const i32x4& acc) {
    if (m >= a.M || n >= a.N) return;
    const float sa = a.sa[m];
    const int cnt = min(4, a.N - n);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (r >= cnt) break;
        float v = (float)acc[r] * sa * a.sw[n + r];
        if (a.bias) v += a.bias[n + r];
        const size_t at = (size_t)m * a.ldc + n + r;
        if (a.type == BB_F32) ((float*)a.C)[at] = v;
        else if (a.type == BB_F16) ((half_t*)a.C)[at] = (half_t)v;
        else ((uint16_t*)a.C)[at] = v != v ? (uint16_t)0x7FC0 : f32_to_bf16_rne(v);
    }
}

// 16 bytes of a row from k on; zeros past its end.  Any alignment.
static __device__ __forceinline__ u32x4 load16(const int8_t* row, int k, int K) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if (k + 16 <= K) __builtin_memcpy(&v, row + k, 16);
    else
        for (int j = 0; j < 16; ++j)
            if (k + j < K) v[j >> 2] |= (unsigned)(uint8_t)row[k + j] << (8 * (j & 3));
    return v;
}

// 64 x 64 of C per workgroup, 64 k at a time through LDS (rows 80 bytes apart: 16 lanes' pieces fall into different banks); four waves of 32 x 32.
__global__ __launch_bounds__(256) void gemm_int8_kernel(GemmInt8Args a) {
    __shared__ __attribute__((aligned(16))) char lds[2][64 * 80];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, c16 = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 64, m0 = blockIdx.y * 64;
    const int wn = (wave & 1) * 32, wm = (wave >> 1) * 32;
    const int8_t* wrow = a.W + (long)min(n0 + (t >> 2), a.N - 1) * a.ldw;
    const int8_t* arow = a.A + (long)min(m0 + (t >> 2), a.M - 1) * a.lda;
    i32x4 acc[2][2] = {};
    for (int k = 0; k < a.K; k += 64) {
        const u32x4 w = load16(wrow, k + (t & 3) * 16, a.K), b = load16(arow, k + (t & 3) * 16, a.K);
        __syncthreads();
        *reinterpret_cast<u32x4*>(&lds[0][(t >> 2) * 80 + (t & 3) * 16]) = w;
        *reinterpret_cast<u32x4*>(&lds[1][(t >> 2) * 80 + (t & 3) * 16]) = b;
        __syncthreads();
        i32x4 fw[2], fa[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            fw[i] = *reinterpret_cast<const i32x4*>(&lds[0][(wn + i * 16 + c16) * 80 + g * 16]);
            fa[i] = *reinterpret_cast<const i32x4*>(&lds[1][(wm + i * 16 + c16) * 80 + g * 16]);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[i], fa[j], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) store_c4(a, m0 + wm + j * 16 + c16, n0 + wn + i * 16 + 4 * g, acc[i][j]);
}

extern "C" size_t bb_gemm_int8_workspace_bytes(int M, int N, int K) {
    (void)M; (void)N; (void)K;
    return 0;
}

extern "C" int bb_gemm_int8(const int8_t* A_dev, long lda, const float* a_scale_dev, const int8_t* W_dev, long ldw, const float* w_scale_dev,
                            const float* bias_dev, void* C_dev, long ldc, int c_type, int M, int N, int K, void* workspace_dev,
                            size_t workspace_bytes, void* hip_stream) {
    if (M < 0 || N < 0 || K < 1 || K > BB_GEMM_INT8_MAX_K || (c_type != BB_F32 && c_type != BB_BF16 && c_type != BB_F16)) return BB_EINVAL;
    if (M == 0 || N == 0) return BB_OK;
    if (!A_dev || !a_scale_dev || !W_dev || !w_scale_dev || !C_dev || (M > 1 && (lda < 0 || ldc < N)) || (N > 1 && ldw < 0)) return BB_EINVAL;
    if ((uintptr_t)a_scale_dev % 4 || (uintptr_t)w_scale_dev % 4 || (uintptr_t)bias_dev % 4 || (uintptr_t)C_dev % (c_type == BB_F32 ? 4 : 2)) return BB_EINVAL;
    if (workspace_bytes < bb_gemm_int8_workspace_bytes(M, N, K)) return BB_ENOMEM;
    (void)workspace_dev;
    GemmInt8Args a{A_dev, W_dev, a_scale_dev, w_scale_dev, bias_dev, C_dev, lda, ldw, ldc, M, N, K, c_type};
    gemm_int8_kernel<<<dim3((N + 63) / 64, (M + 63) / 64), 256, 0, (hipStream_t)hip_stream>>>(a);
    return hipGetLastError() == hipSuccess ? BB_OK : BB_EHIP;
}
