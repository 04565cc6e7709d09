// bb_gemm_int8: C[m][n] = (sum_k A[m][k] W[n][k]) * a_scale[m] * w_scale[n] + bias[n], A and W int8, both with k contiguous.
//
// The sum is exact (int32; K <= 131071 keeps it below 2^31 even for codes of -128), so results do not depend on the tile, the split
// of k or the order; it is rounded to fp32 once, scaled in fp32 and rounded to C's type.
//
// The operands: the matrix cores take 16 rows x 64 k, lane l holding the 16 bytes k = 16 (l / 16) .. + 15 of row l % 16, so row-major
// operands need no re-tiling: 16-byte pieces of their rows are what a lane wants.  W is the first operand: a lane then holds four
// consecutive columns of one row of C.
//
// What bounds it.  Large products: what the L2s deliver, at the clock that power allows.  MFMAs alone on such operands run at 4.1 POP/s (1.95 GHz);
// with the LDS reads 3.6-3.8; with the loads too 2.9 in the loop over k of a 256 x 256 tile (64 KB per CU and chunk of 128 k, 1.36 us, of 47 KB/us; the
// matrix pipes are busy 0.67 of the time at 1.88 GHz), and 2.4 over 8192 x 8192 x 8192 (459 us) and 8192 x 24576 x 4096 (0.68 ms), with the
// tiles' ends.  Loads by 64-byte runs reach half the rate of whole lines (66 against 130 KB/us and CU from an L2): hence chunks of 128 k, and
// rows at multiples of 128 bytes are fastest (1402 x 4610 rows of 3592 k 41 us, of 3584 34).  Few rows: the stream of W, 19.3 us of 101 MB
// at one row (5.2 TB/s, partly out of the cache behind the L2s); between them (120 rows, 50 MB) 14 us beside 4 us that join four splits of k.
#include "bb_internal.h"
#include "lds.h"
#include "sched.h"
#include <algorithm>
#include <cmath>
#include <type_traits>

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct GemmInt8Args {
    const int8_t *A, *W; const float *sa, *sw, *bias; void* C;
    long lda, ldw, ldc;
    int M, N, K, type;
    const int* live;                // rows of A that count, on the device (null: all M; only the tiled kernel is asked for fewer)
};

// Which column of a wave's 16 T row i of MFMA tile t is: of a pair of tiles a lane, which holds rows 4 (lane / 16) .. + 3 of each, gets eight columns
// in a row, which it stores whole.  (The last of an odd number of tiles: as they come.)
template <int T> static __device__ __forceinline__ constexpr int column_of(int t, int i) {
    return t < T / 2 * 2 ? t / 2 * 32 + i / 4 * 8 + t % 2 * 4 + i % 4 : t * 16 + i;
}
// N consecutive values of a row of C, scaled and rounded, as far as the row goes.
template <int N, class E> static __device__ __forceinline__ void store_values(const float (&v)[N], E* at, int left) {
    typedef float fN __attribute__((ext_vector_type(N)));
    typedef E eN __attribute__((ext_vector_type(N)));
    fN f;
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = v[j];
    const eN e = __builtin_convertvector(f, eN);
    if (left >= N) {
        typedef E eU __attribute__((ext_vector_type(N), aligned(sizeof(E))));
        __builtin_nontemporal_store(e, reinterpret_cast<eU*>(at));
    } else
#pragma unroll
        for (int j = 0; j < N - 1; ++j) if (j < left) at[j] = e[j];
}
// Columns of tile(s) t (and t + 1) of R rows of MFMA tiles; sw, bias: the scales of the wave's columns in LDS; sa: of the rows lane % 16 of each tile row.
template <int T, int R, int t, class E>
static __device__ __forceinline__ void store_columns(const GemmInt8Args& a, int m, int n, const i32x4 (&acc)[R][T], const float (&sa)[R], const float* sw, const float* bias) {
    constexpr int N = t < T / 2 * 2 ? 8 : 4;
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));                          // (addresses are not worth keeping through the loop over k)
    const int col = column_of<T>(t, 4 * (lane >> 4));
    float s[N], bs[N];
#pragma unroll
    for (int j = 0; j < N; ++j) { s[j] = sw[col + j]; bs[j] = a.bias ? bias[col + j] : 0.f; }
    const int row = m + (lane & 15), left = a.N - n - col;
    E* at = (E*)a.C + (size_t)row * a.ldc + n + col;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float v[N];
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = (float)acc[r][t + j / 4][j % 4] * sa[r] * s[j];
        if (a.bias)
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] += bs[j];
        if (row + 16 * r < a.M) store_values<N, E>(v, at, left);
        at += 16 * a.ldc;
        __builtin_amdgcn_sched_barrier(0);
    }
}
template <int T, int R> static __device__ __forceinline__ void store_tile(const GemmInt8Args& a, int m, int n, const i32x4 (&acc)[R][T], const float (&sa)[R], const float* sw, const float* bias) {
    auto as = [&](auto e) {
        typedef decltype(e) E;
        unroll<(T + 1) / 2>([&](auto P) { store_columns<T, R, 2 * decltype(P)::value, E>(a, m, n, acc, sa, sw, bias); });
    };
    if (a.type == BB_F32) as(0.f); else if (a.type == BB_F16) as((half_t)0); else as((__bf16)0.f);
}

// 16 bytes of a row from k on; zeros past its end.  Any alignment.  A piece that the end cuts is shifted down out of the row's last 16 bytes, so
// that every lane makes one load and none waits for another's (K >= 16).
static __device__ __forceinline__ u32x4 load16(const int8_t* row, int k, int K) {
    typedef unsigned long long u64x2 __attribute__((ext_vector_type(2)));
    const int from = min(k, K - 16);
    u64x2 w;
    __builtin_memcpy(&w, row + from, 16);
    int sh = 8 * min(k - from, 16);                         // 0: whole; 128: nothing left
    const bool upper = sh >= 64;
    unsigned long long lo = upper ? w[1] : w[0], hi = upper ? 0 : w[1];
    sh -= upper ? 64 : 0;
    const bool none = sh >= 64;
    sh = none ? 0 : sh;
    lo = lo >> sh | hi << 1 << (63 - sh);
    hi >>= sh;
    return __builtin_bit_cast(u32x4, u64x2{none ? 0 : lo, none ? 0 : hi});
}

// Rows of fewer than 16 bytes: a thread per value of C.
__global__ __launch_bounds__(256) void gemm_int8_short_kernel(GemmInt8Args a) {
    const size_t values = (size_t)a.M * a.N;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < values; i += (size_t)gridDim.x * 256) {
        const int m = (int)(i / a.N), n = (int)(i % a.N);
        int acc = 0;
        for (int k = 0; k < a.K; ++k) acc += (int)a.A[m * a.lda + k] * (int)a.W[n * a.ldw + k];
        float v = (float)acc * a.sa[m] * a.sw[n];
        if (a.bias) v += a.bias[n];
        const size_t at = (size_t)m * a.ldc + n;
        if (a.type == BB_F32) ((float*)a.C)[at] = v;
        else if (a.type == BB_F16) ((half_t*)a.C)[at] = (half_t)v;
        else ((__bf16*)a.C)[at] = (__bf16)v;
    }
}

// Rows of any alignment -> rows of whole 16-byte pieces with zeros past K, for the tiled kernel.
__global__ __launch_bounds__(256) void align_rows_kernel(const int8_t* __restrict__ src, long ld, u32x4* __restrict__ dst, size_t pieces, int per_row, int K) {
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (size_t)gridDim.x * 256) {
        const size_t row = i / per_row;
        dst[i] = load16(src + (long)row * ld, (int)(i - row * per_row) * 16, K);
    }
}

// The tiled kernel: operands whose rows are 16-byte aligned.  A workgroup of four waves (WM of them along m) owns 16 R WM rows x 16 T (4 / WM)
// columns, a wave 16 R x 16 T of them.  Both operands pass through LDS in chunks of 128 k: a direct-to-LDS load brings a unit of eight rows x
// 128 k (1 KiB), eight lanes a row, so that whole 128-byte lines are asked for at once, into a ring of NS chunks; fragments of the next
// half chunk move into registers while the matrix cores work on the present one.  In unit u piece c (16 bytes) of row r lies at
// 8 r + (c ^ r ^ 4 (u % 2)): eight lanes that read one piece of eight rows, of one unit or of half of two (see column_of), touch all banks once.
// Workgroups are as many as run at once and take item after item (a tile, or a split's part of its k): the chunks of all their items pass
// through the ring as one stream, so that the next item's are on their way while a tile is stored.
// The chunk of a ragged end of k (K % 128) is brought through registers, with zeros past the end.
struct TiledArgs { GemmInt8Args g; int tiles_m, tiles_n, chunks, split; i32x4* part; };
struct Item { int m0, n0, c0, c1; };
#define I8_BAND 4
// Items are numbered split by split, tiles in bands of four row groups, row group fastest.
template <int BM, int BN> static __device__ __forceinline__ Item item_of(const TiledArgs& ta, int item) {
    const int tiles = ta.tiles_m * ta.tiles_n, split_id = item / tiles, tile = item % tiles;
    const int band = tile / (I8_BAND * ta.tiles_n), in_band = tile % (I8_BAND * ta.tiles_n), band_h = min(I8_BAND, ta.tiles_m - band * I8_BAND);
    Item it;
    it.m0 = __builtin_amdgcn_readfirstlane((band * I8_BAND + in_band % band_h) * BM);
    it.n0 = __builtin_amdgcn_readfirstlane(in_band / band_h * BN);
    it.c0 = __builtin_amdgcn_readfirstlane(ta.chunks * split_id / ta.split);
    it.c1 = __builtin_amdgcn_readfirstlane(ta.chunks * (split_id + 1) / ta.split);
    return it;
}

static __device__ __forceinline__ void only_live(TiledArgs& ta, int bm) {
    if (!ta.g.live) return;
    ta.g.M = __builtin_amdgcn_readfirstlane(min(ta.g.M, *ta.g.live));
    ta.tiles_m = (ta.g.M + bm - 1) / bm;
}

template <int R, int T, int WM, int NS, int PER_CU>
__global__ __launch_bounds__(256, PER_CU) void gemm_int8_tiled_kernel(TiledArgs ta) {
    constexpr int WN = 4 / WM, FA = R * WM, FW = T * WN, BM = 16 * FA, BN = 16 * FW, U = 2 * (FA + FW), L = U / 4, LA = FA / 2, SLOT = U * 1024;
    static_assert(FA % 2 == 0, "every wave brings as many units of A, and of W");
    constexpr int SM = (BM + 63) / 64 * 64, SN = (BN + 63) / 64 * 64, SCALES = SM + 2 * SN;        // scales of an item: rows', columns', biases
    __shared__ __attribute__((aligned(16))) char lds[NS * SLOT + (NS + 2) * SCALES * 4];
    float* const scales = reinterpret_cast<float*>(lds + NS * SLOT);
    only_live(ta, BM);
    const GemmInt8Args& a = ta.g;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, c16 = lane & 15, g = lane >> 4;
    const int wm = wave % WM, wn = wave / WM;
    const int items = ta.tiles_m * ta.tiles_n * ta.split, whole = a.K / 128;        // whole chunks: the one after them is ragged
    // workgroups go to the eight XCDs round robin: of every round of items each XCD gets a contiguous run
    auto item_at = [&](int base) {
        const int n_round = min((int)gridDim.x, items - base), lin = blockIdx.x, e = lin & 7;
        return lin < n_round ? __builtin_amdgcn_readfirstlane(base + e * (n_round >> 3) + min(e, n_round & 7) + (lin >> 3)) : -1;
    };

    // ---- the loads: wave w brings the units w, w + 4, ... of a chunk, first A's, then W's -------------------------------
    const unsigned lds0 = lds_offset(lds), lda = (unsigned)a.lda, ldw = (unsigned)a.ldw;
    const int lr = lane >> 3, piece = ((lane & 7) ^ lr ^ ((wave & 1) * 4)) * 16;
    const unsigned offA = (wave * 8 + lr) * lda + piece, offW = (wave * 8 + lr) * ldw + piece;
    auto uniform = [](const void* q) {
        const size_t v = (size_t)q;
        return (const char*)(((size_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)v));
    };
    // The chunk to ask for next: its round of items, number and the item's end; its first row and k; the last row (rows past the operand's
    // end read that).  What is not to be read directly, the ragged chunk and what follows the last item, is one address for all lanes.
    int f_base = 0, f_c = 0, f_end = 0, f_scales = 0, f_m0 = 0, f_n0 = 0;
    const char *pA = uniform(a.A), *pW = uniform(a.W);
    unsigned maxA = 0, maxW = 0, runA = 0, runW = 0;        // (run: offsets of the next unit's lanes)
    unsigned wr = 0, rd = 0;                                // byte offsets of the ring's slots
    auto bump = [&](unsigned& o) { o = o + SLOT == NS * SLOT ? 0u : o + SLOT; };
    auto indirect = [&]() { pA = uniform(a.A); pW = uniform(a.W); maxA = maxW = 0; };
    auto open_item = [&]() {
        const int item = f_base < items ? item_at(f_base) : -1;
        if (item < 0) { indirect(); f_end = 1 << 30; f_c = 1 << 29; return; }
        const Item it = item_of<BM, BN>(ta, item);
        f_m0 = it.m0; f_n0 = it.n0; f_c = it.c0; f_end = it.c1;
        if (f_c < whole) {
            pA = uniform(a.A + it.m0 * a.lda + it.c0 * 128);
            pW = uniform(a.W + it.n0 * a.ldw + it.c0 * 128);
            maxA = (unsigned)min(a.M - 1 - it.m0, BM - 1) * lda + piece;
            maxW = (unsigned)min(a.N - 1 - it.n0, BN - 1) * ldw + piece;
        } else indirect();
        if (ta.split == 1) {
            const unsigned to = lds0 + NS * SLOT + f_scales * (SCALES * 4) + wave * 256;
            if (wave * 64 < SM) load_dwords_to_lds(uniform(a.sa), (unsigned)min(it.m0 + wave * 64 + lane, a.M - 1) * 4u, to);
            if (wave * 64 < SN) load_dwords_to_lds(uniform(a.sw), (unsigned)min(it.n0 + wave * 64 + lane, a.N - 1) * 4u, to + SM * 4);
            if (a.bias && wave * 64 < SN) load_dwords_to_lds(uniform(a.bias), (unsigned)min(it.n0 + wave * 64 + lane, a.N - 1) * 4u, to + (SM + SN) * 4);
            f_scales = f_scales == NS + 1 ? 0 : f_scales + 1;
        }
    };
    auto fetch = [&](int i) {
        const unsigned to = lds0 + wr + wave * 1024 + i * 4096;
        if (i == 0) { runA = offA; runW = offW; }
        if (i < LA) { load_to_lds<0>(pA, min(runA, maxA), to); runA += 32 * lda; }
        else { load_to_lds<0>(pW, min(runW, maxW), to); runW += 32 * ldw; }
    };
    auto next_chunk = [&]() {
        if (f_c == whole) {                                 // ragged: over what the loads above left there, once they have landed
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            constexpr int AT_ONCE = L % 4 == 0 ? 4 : L % 3 == 0 ? 3 : L % 2 == 0 ? 2 : L % 5 == 0 ? 5 : 1;
            const int k = whole * 128 + piece;
#pragma unroll 1
            for (int i0 = 0; i0 < L; i0 += AT_ONCE) {
                u32x4 v[AT_ONCE];
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j) {
                    const int i = i0 + j, row = (wave + 4 * (i < LA ? i : i - LA)) * 8 + lr;
                    const int8_t* p = i < LA ? a.A + min(f_m0 + row, a.M - 1) * a.lda : a.W + min(f_n0 + row, a.N - 1) * a.ldw;
                    v[j] = load16(p, k, a.K);
                }
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j) *reinterpret_cast<u32x4*>(lds + wr + (wave + 4 * (i0 + j)) * 1024 + lane * 16) = v[j];
            }
        }
        ++f_c; pA += 128; pW += 128;
        bump(wr);
        if (f_c == f_end) { f_base += gridDim.x; open_item(); }
        else if (f_c >= whole) indirect();
    };
    open_item();
    for (int s = 0; s < NS; ++s) {
#pragma unroll
        for (int i = 0; i < L; ++i) fetch(i);
        next_chunk();
    }

    i32x4 acc[R][T], w[2][T], b[2][R];
    // (where piece g of a fragment's row c16 lies: in A's tiles; in the two kinds of W's, see column_of; the piece of the second half is 64 bytes away)
    auto place = [&](int row) { return (unsigned)(row * 128 + ((g ^ (row & 7) ^ (row >> 3 & 1) * 4) * 16)); };
    const unsigned fragA = place(c16), frag0 = place(column_of<T>(0, c16)), frag1 = place(column_of<T>(T > 1 ? 1 : 0, c16));
    const char *rA = lds + wm * R * 2048, *rW = lds + (FA + wn * T) * 2048;
    auto read = [&](auto H, int j) {                        // fragment j of half H of the chunk at rd: W's, then A's
        constexpr int h = decltype(H)::value;
        const bool pair = j < T / 2 * 2;
        const unsigned f = j >= T || !pair ? fragA : j & 1 ? frag1 : frag0, o = (h ? f ^ 64u : f) + rd;
        if (j < T) w[h][j] = *reinterpret_cast<const i32x4*>(rW + o + (pair ? j / 2 * 4096 : j * 2048));
        else b[h][j - T] = *reinterpret_cast<const i32x4*>(rA + o + (j - T) * 2048);
    };
    // all but the latest Later loads of this wave have landed and its reads are done; after the barrier so are the others'
    auto landed = [&](auto Later) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(Later)::value) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    landed(IC((NS - 1) * L));
    // Half a chunk: R slots of T MFMAs; the next half's fragments are asked for in the first of them.  Once all waves have those of a chunk's second half
    // (a barrier half way through its first half) its place is free and the chunk NS ahead is asked for, spread over the slots that are left until the
    // chunk's end: as soon and as evenly as can be, since what the L2s deliver sets the time (us, 128 x 128 and 256 x 192 tiles, 8192 x 4096 x 12288: 401 and
    // 365 when it was asked for in the second half only, 361 and 337 so).
    constexpr int READ_SLOTS = R > 2 ? R / 2 : R, FREE = R - READ_SLOTS, FETCH_SLOTS = FREE + R, EARLY = L * FREE / FETCH_SLOTS;
    auto half = [&](auto H, auto First) {
        constexpr int h = decltype(H)::value;
        unroll<R>([&](auto Rr) {
            constexpr int r = decltype(Rr)::value;
#pragma unroll
            for (int t = 0; t < T; ++t) acc[r][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[h][t], b[h][r], decltype(First)::value ? i32x4{0, 0, 0, 0} : acc[r][t], 0, 0, 0);
            if constexpr (r < READ_SLOTS)
                unroll<(R + T) * (r + 1) / READ_SLOTS - (R + T) * r / READ_SLOTS>([&](auto J) { read(IC(1 - h), (R + T) * r / READ_SLOTS + decltype(J)::value); });
            if constexpr (h == 0 && FREE > 0 && r == READ_SLOTS) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
            }
            if constexpr (h == 1 || r >= READ_SLOTS) {
                constexpr int f = h == 0 ? r - READ_SLOTS : FREE + r;
                unroll<L * (f + 1) / FETCH_SLOTS - L * f / FETCH_SLOTS>([&](auto I) { fetch(L * f / FETCH_SLOTS + decltype(I)::value); });
            }
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    int now_scales = 0;
    for (int base = 0; base < items; base += gridDim.x) {
        const int item = item_at(base);
        if (item < 0) break;
        const Item it = item_of<BM, BN>(ta, item);
        // (read here although the last half before has them too: held through the storing of a tile they cost spills)
#pragma unroll
        for (int j = 0; j < R + T; ++j) read(IC(0), j);
        auto chunk = [&](auto First) {
            half(IC(0), First);
            bump(rd);
            landed(IC((NS - 2) * L + EARLY));
            half(IC(1), std::false_type{});
            next_chunk();
        };
        chunk(std::true_type{});
        for (int c = it.c0 + 1; c < it.c1; ++c) chunk(std::false_type{});
        if (ta.part) {          // partial sums as they lie in the registers: [split][tile][wave][r][t][lane]
            i32x4* P = ta.part + ((size_t)item * 4 + wave) * (T * R * 64) + lane;
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int t = 0; t < T; ++t) P[(r * T + t) * 64] = acc[r][t];
        } else {
            const float *rows = scales + now_scales * SCALES, *sw = rows + SM + wn * T * 16;
            float sa[R];
#pragma unroll
            for (int r = 0; r < R; ++r) sa[r] = rows[(wm * R + r) * 16 + c16];
            store_tile<T, R>(a, it.m0 + wm * R * 16, it.n0 + wn * T * 16, acc, sa, sw, sw + SN);
            now_scales = now_scales == NS + 1 ? 0 : now_scales + 1;
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // (no direct-to-LDS load may outlive the workgroup)
}

// Sum of the partial tiles of a split k range, a wave per 16 rows x 16 T columns.
template <int R, int T, int WM>
__global__ __launch_bounds__(256) void gemm_int8_join_kernel(TiledArgs ta) {
    constexpr int WN = 4 / WM;
    __shared__ __attribute__((aligned(16))) float scales[4][2][16 * T];
    only_live(ta, 16 * R * WM);
    const GemmInt8Args& a = ta.g;
    const int sub = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), idx = blockIdx.x * 4 + sub, lane = threadIdx.x & 63;
    const int tiles = ta.tiles_m * ta.tiles_n, wave = idx / R % 4, r = idx % R;
    if (idx >= tiles * 4 * R) return;
    const Item it = item_of<16 * R * WM, 16 * T * WN>(ta, idx / (4 * R));
    const int m = it.m0 + (wave % WM * R + r) * 16, n = it.n0 + wave / WM * T * 16;
    if (m >= a.M || n >= a.N) return;                       // (whole waves, and no barrier below)
    const size_t stride = (size_t)tiles * (4 * R * T * 64);
    const i32x4* P = ta.part + (size_t)idx * (T * 64) + lane;
    const float sa[1] = {a.sa[min(m + (lane & 15), a.M - 1)]};
    for (int i = lane; i < 16 * T; i += 64) {
        scales[sub][0][i] = a.sw[min(n + i, a.N - 1)];
        if (a.bias) scales[sub][1][i] = a.bias[min(n + i, a.N - 1)];
    }
    i32x4 acc[1][T];
#pragma unroll
    for (int t = 0; t < T; ++t) acc[0][t] = i32x4{0, 0, 0, 0};
    for (int s = 0; s < ta.split; s += 4) {
        i32x4 p[4][T];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int t = 0; t < T; ++t) p[u][t] = s + u < ta.split ? P[(s + u) * stride + t * 64] : i32x4{0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int t = 0; t < T; ++t) acc[0][t] += p[u][t];
    }
    wave_lds_order();
    store_tile<T, 1>(a, m, n, acc, sa, scales[sub][0], scales[sub][1]);
}

template <int R, int T, int WM, int NS, int PER_CU> static void launch_tiled(const GemmInt8Args& g, int split, void* ws, hipStream_t s) {
    constexpr int BM = 16 * R * WM, BN = 16 * T * (4 / WM);
    TiledArgs ta{g, (g.M + BM - 1) / BM, (g.N + BN - 1) / BN, (g.K + 127) / 128, split, split > 1 ? (i32x4*)ws : nullptr};
    const int tiles = ta.tiles_m * ta.tiles_n;
    gemm_int8_tiled_kernel<R, T, WM, NS, PER_CU><<<std::min(tiles * split, 256 * PER_CU), 256, 0, s>>>(ta);
    if (split > 1) gemm_int8_join_kernel<R, T, WM><<<tiles * R, 256, 0, s>>>(ta);
}

// The bodies of the tiled kernel and what they cost, in us: start + per round of items the most loaded CU takes (round), per chunk of
// those (chunk), per chunk and workgroup that shares a CU (shared); per join (join) and MB of partial sums (per_mb).  Fitted to launches of
// 18 row counts from 1 to 8192 x 11 matrices from 256 x 688 to 37888 x 3584 x k splits; there the choice is on average 1 % slower than the best
// of these bodies and splits, at worst 26 %, and where all weights come from memory (640 MB of them in turn, 13 row counts up to 1024) 1 and
// 16 %.  (What it chooses by, not a forecast: inside a forward, where weights and rows are cold, QKV and gate/up of 120 rows take 22 and 36 us where
// it says 14 and 22.)  The second 128 x 128, one workgroup a CU and a chunk more in flight than the first's two each, is for such weights when no CU has a
// second tile: bf16 results of 192 rows by 12288 x 4096 23.4 us (30.9 with the first, 27.8 the best without it), 120 by 24576 x 4096 30.1
// (34.6); with more tiles two workgroups that overlap win: 1024 by 37888 x 3584 166 (182).
struct Int8Body { int bm, bn, per_cu; float start, round, chunk, shared, join, per_mb; };
static const Int8Body i8_bodies[] = {
    {256, 256, 1, 0.64f, 11.92f, 1.328f, 0.043f, 0.0f, 0.239f},
    {256, 192, 1, 0.77f, 8.02f, 0.994f, 0.006f, 1.89f, 0.197f},
    {128, 128, 2, 2.03f, 2.69f, 0.369f, 0.485f, 2.62f, 0.238f},
    {128, 128, 1, 4.20f, 1.25f, 0.484f, 0.0f, 3.19f, 0.262f},
    {128, 64, 2, 3.89f, 0.95f, 0.028f, 0.529f, 2.54f, 0.248f},
    {64, 64, 2, 3.95f, 0.49f, 0.073f, 0.305f, 2.25f, 0.328f},
    {32, 32, 3, 4.06f, 0.11f, 0.100f, 0.184f, 1.85f, 0.770f},
};
#define I8_MAX_PARTIAL ((size_t)1 << 28)
struct Int8Plan { int body, split; size_t partial_bytes; };
static Int8Plan int8_plan(int M, int N, int K, size_t most = I8_MAX_PARTIAL) {
    Int8Plan best{0, 1, 0};
    float best_cost = INFINITY;
    const int chunks = (K + 127) / 128;
    // us that the memory takes, at a fitted rate: of the fitted launches' weights a part lay in the cache behind the L2s, and a copy reaches 5.1
    const float stream = ((float)N * K + (float)M * K + 2.0f * (float)M * N) / 7.1e6f;
    for (int i = 0; i < (int)(sizeof(i8_bodies) / sizeof(i8_bodies[0])); ++i) {
        const Int8Body& b = i8_bodies[i];
        const size_t tiles = ((size_t)M + b.bm - 1) / b.bm * (((size_t)N + b.bn - 1) / b.bn);
        for (int split : {1, 2, 3, 4, 6, 8, 12, 16}) {
            const size_t items = tiles * split, partial = split > 1 ? items * b.bm * b.bn * 4 : 0;
            if (split > 1 && (split > chunks || partial > most)) break;
            const float per = (float)((items + 255) / 256), rounds = ceilf(per / b.per_cu), c = (float)((chunks + split - 1) / split);
            const float main = b.start + rounds * b.round + rounds * c * b.chunk + per / b.per_cu * c * b.shared;
            float cost = sqrtf(sqrtf(main * main * main * main + stream * stream * stream * stream));
            if (split > 1) cost += b.join + b.per_mb * 1e-6f * (float)partial;
            if (cost < best_cost) { best_cost = cost; best = Int8Plan{i, split, partial}; }
        }
    }
    return best;
}

static void launch_plan(const GemmInt8Args& a, const Int8Plan& p, void* workspace_dev, hipStream_t s) {
    switch (p.body) {
        case 0: launch_tiled<8, 8, 2, 2, 1>(a, p.split, workspace_dev, s); break;
        case 1: launch_tiled<8, 6, 2, 2, 1>(a, p.split, workspace_dev, s); break;
        case 2: launch_tiled<4, 4, 2, 2, 2>(a, p.split, workspace_dev, s); break;
        case 3: launch_tiled<4, 4, 2, 3, 1>(a, p.split, workspace_dev, s); break;
        case 4: launch_tiled<4, 2, 2, 3, 2>(a, p.split, workspace_dev, s); break;
        case 5: launch_tiled<2, 2, 2, 4, 2>(a, p.split, workspace_dev, s); break;
        default: launch_tiled<1, 1, 2, 4, 3>(a, p.split, workspace_dev, s); break;
    }
}

// The layers of a forward: aligned operands, fp32 out, as many splits as the workspace has room for.
void launch_gemm_int8(const int8_t* A, long lda, const float* sa, const int8_t* W, long ldw, const float* sw, float* C, long ldc, int M, int N, int K,
                      void* ws, size_t ws_bytes, const int* live, hipStream_t s) {
    GemmInt8Args a{A, W, sa, sw, nullptr, C, lda, ldw, ldc, M, N, K, BB_F32, live};
    launch_plan(a, int8_plan(M, N, K, std::min(ws_bytes, I8_MAX_PARTIAL)), ws, s);
}
size_t gemm_int8_partial_bytes(int M, int N, int K) { return int8_plan(M, N, K).partial_bytes; }

// Rows that are not 16-byte aligned go through copies that are, in the workspace.  (A kernel that took any alignment through registers was slower
// at every size: us, 64 x 24576 x 4097 79 against 65 with the copies, 64 x 4096 x 4097 64 against 26.)
static size_t copy_bytes(int rows, int K) { return align_up((size_t)rows * align_up(K, 16), 256); }
static bool sizes_ok(int M, int N, int K) { return M >= 0 && N >= 0 && M <= BB_GEMM_INT8_MAX_ROWS && N <= BB_GEMM_INT8_MAX_ROWS && K >= 1 && K <= BB_GEMM_INT8_MAX_K; }

extern "C" size_t bb_gemm_int8_workspace_bytes(int M, int N, int K, int aligned) {
    if (!sizes_ok(M, N, K) || M == 0 || N == 0 || K < 16) return 0;
    return align_up(int8_plan(M, N, K).partial_bytes, 256) + (aligned ? 0 : copy_bytes(M, K) + copy_bytes(N, K));
}

extern "C" int bb_gemm_int8(const int8_t* A_dev, long lda, const float* a_scale_dev, const int8_t* W_dev, long ldw, const float* w_scale_dev,
                            const float* bias_dev, void* C_dev, long ldc, int c_type, int M, int N, int K, void* workspace_dev,
                            size_t workspace_bytes, void* hip_stream) {
    if (!sizes_ok(M, N, K) || (c_type != BB_F32 && c_type != BB_BF16 && c_type != BB_F16)) return BB_EINVAL;
    if (M == 0 || N == 0) return BB_OK;
    if (!A_dev || !a_scale_dev || !W_dev || !w_scale_dev || !C_dev || (M > 1 && (lda < 0 || ldc < N)) || (N > 1 && ldw < 0)) return BB_EINVAL;
    if ((uintptr_t)a_scale_dev % 4 || (uintptr_t)w_scale_dev % 4 || (uintptr_t)bias_dev % 4 || (uintptr_t)C_dev % (c_type == BB_F32 ? 4 : 2)) return BB_EINVAL;
    if (M == 1) lda = ldc = 0;                              // (a single row has no next)
    if (N == 1) ldw = 0;
    hipStream_t s = (hipStream_t)hip_stream;
    // the tiled kernel's offsets within a tile are of 32 bits
    const long far = 1 << 23;
    auto aligned = [&](const int8_t* p, long ld) { return (uintptr_t)p % 16 == 0 && ld % 16 == 0 && ld <= far; };
    const bool a_aligned = aligned(A_dev, lda), w_aligned = aligned(W_dev, ldw);
    const size_t need = bb_gemm_int8_workspace_bytes(M, N, K, a_aligned && w_aligned);
    if (need > 0 && (!workspace_dev || (uintptr_t)workspace_dev % 16)) return workspace_bytes < need ? BB_ENOMEM : BB_EINVAL;
    if (workspace_bytes < need) return BB_ENOMEM;
    GemmInt8Args a{A_dev, W_dev, a_scale_dev, w_scale_dev, bias_dev, C_dev, lda, ldw, ldc, M, N, K, c_type, nullptr};
    if (K < 16) {
        gemm_int8_short_kernel<<<(unsigned)std::min<size_t>(((size_t)M * N + 255) / 256, 8192), 256, 0, s>>>(a);
        return hipGetLastError() == hipSuccess ? BB_OK : BB_EHIP;
    }
    const Int8Plan p = int8_plan(M, N, K);
    const int per_row = (K + 15) / 16;
    char* at = (char*)workspace_dev + align_up(p.partial_bytes, 256);
    auto copy = [&](const int8_t* src, long ld, int rows) {
        const size_t pieces = (size_t)rows * per_row;
        align_rows_kernel<<<(unsigned)std::min<size_t>((pieces + 255) / 256, 8192), 256, 0, s>>>(src, ld, (u32x4*)at, pieces, per_row, K);
        const int8_t* to = (const int8_t*)at;
        at += copy_bytes(rows, K);
        return to;
    };
    if (!a_aligned) { a.A = copy(A_dev, lda, M); a.lda = per_row * 16L; }
    if (!w_aligned) { a.W = copy(W_dev, ldw, N); a.ldw = per_row * 16L; }
    launch_plan(a, p, workspace_dev, s);
    return hipGetLastError() == hipSuccess ? BB_OK : BB_EHIP;
}

// ---- tests ------------------------------------------------------------------------------------------------------------------------------------
extern "C" int bb_debug_gemm_int8_plan(int M, int N, int K, int out[5]) {
    if (!out || !sizes_ok(M, N, K) || M == 0 || N == 0 || K < 16) return BB_EINVAL;
    const Int8Plan p = int8_plan(M, N, K);
    const Int8Body& b = i8_bodies[p.body];
    out[0] = p.body; out[1] = b.bm; out[2] = b.bn; out[3] = b.per_cu; out[4] = p.split;
    return BB_OK;
}

extern "C" int bb_debug_gemm_int8(const int8_t* A_dev, const float* a_scale_dev, const int8_t* W_dev, const float* w_scale_dev, long ld, float* C_dev, int M, int N, int K,
                                  int body, int split, const int* live_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    const int n_bodies = (int)(sizeof(i8_bodies) / sizeof(i8_bodies[0]));
    if (!A_dev || !a_scale_dev || !W_dev || !w_scale_dev || !C_dev || !sizes_ok(M, N, K) || M == 0 || N == 0 || K < 16 || (uintptr_t)A_dev % 16 || (uintptr_t)W_dev % 16 ||
        ld % 16 || ld < K || ld > 1 << 23 || body < 0 || body >= n_bodies || split < 1 || split > 16 || split > (K + 127) / 128) return BB_EINVAL;
    const Int8Body& b = i8_bodies[body];
    const size_t tiles = ((size_t)M + b.bm - 1) / b.bm * (((size_t)N + b.bn - 1) / b.bn), partial = split > 1 ? tiles * split * b.bm * b.bn * 4 : 0;
    if (partial > workspace_bytes || tiles * split > 1u << 30) return BB_ENOMEM;
    if (partial > 0 && (!workspace_dev || (uintptr_t)workspace_dev % 16)) return BB_EINVAL;
    GemmInt8Args a{A_dev, W_dev, a_scale_dev, w_scale_dev, nullptr, C_dev, ld, ld, N, M, N, K, BB_F32, live_dev};
    launch_plan(a, Int8Plan{body, split, partial}, workspace_dev, (hipStream_t)hip_stream);
    return hipGetLastError() == hipSuccess ? BB_OK : BB_EHIP;
}
