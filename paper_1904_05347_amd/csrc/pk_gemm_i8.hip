// pk_gemm_i8.hip -- products of 8-bit integers with a scale for each row of
// either operand: C[m][n] = sa[m] sb[n] sum_k A[m][k] B[n][k] + bias[n].
#include "pk_i8.hpp"
#include "pk_i8_checks.hpp"
#include "pk_partition.hpp"

namespace {

using pk::bf16;
using pk::f16;
using pk::Pack;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_u __attribute__((aligned(1)));

struct Args {
    const int8_t *A, *B;
    const float *sa, *sb, *bias;
    void *C;
    int64_t lda, ldb, ldc;
    int M, N, K;
};

// Four neighbouring elements of a row of C from n on.
template <typename T>
__device__ __forceinline__ void store4(const Args &p, int m, int n, const i32x4 &acc)
{
    if (m >= p.M || n >= p.N) return;
    const float sa = p.sa[m];
    T *c = (T *)p.C + (int64_t)m * p.ldc + n;
    typename Pack<T, 4>::V v;
    if (n + 4 <= p.N) {
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = (T)((float)acc[r] * (sa * p.sb[n + r]) + (p.bias ? p.bias[n + r] : 0.f));
        *reinterpret_cast<typename Pack<T, 4>::U *>(c) = v;
        return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (n + r < p.N) c[r] = (T)((float)acc[r] * (sa * p.sb[n + r]) + (p.bias ? p.bias[n + r] : 0.f));
}

// ------------------------------------------------------------ few rows of A
//
// A work-group makes 16 MT rows x 16 NT columns of C; its waves share K in
// blocks of 128 and add their sums through LDS.  Operands go from memory to the
// registers the matrix instruction reads: nothing is staged.
// v_mfma_i32_16x16x64_i8 takes 16 bytes a lane from row lane % 16 of each
// operand; which k they are does not matter as long as both operands agree, so
// lane / 16 takes 32 neighbouring bytes of a block for two instructions, and a
// row's 128 bytes are read whole.

// 16 bytes of a row from k on.  At the row's end the last 16 are read instead
// (both operands do, so the k still agree); the first `drop` of them belong to
// the chunk before.  A row shorter than 16 is read byte by byte.
__device__ __forceinline__ i32x4 chunk(const int8_t *row, int k, int K)
{
    if (K >= 16) return *reinterpret_cast<const i32x4_u *>(row + (k + 16 <= K ? k : K - 16));
    i32x4 v = {0, 0, 0, 0};
    if (k == 0)
        for (int j = 0; j < K; ++j) v[j / 4] |= (row[j] & 255) << (j % 4 * 8);
    return v;
}

// Zeroes the bytes of chunk(row, k, K) that are not its own.
__device__ __forceinline__ i32x4 own_bytes(i32x4 v, int k, int K)
{
    if (K < 16) return v;
    const int drop = k + 16 <= K ? 0 : k + 16 - K;  // of this chunk, 16 or more: all
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int d = drop - 4 * w;
        v[w] &= d <= 0 ? -1 : d >= 4 ? 0 : (int)(0xffffffffu << (8 * d));
    }
    return v;
}

template <typename T, int MT, int NT, int WAVES>
__global__ void __launch_bounds__(WAVES * 64) gemm_i8_rows_kernel(Args p)
{
    __shared__ i32x4 part[WAVES][MT * NT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * (16 * NT), m0 = blockIdx.y * (16 * MT);
    const int8_t *pa[MT], *pb[NT];  // rows beyond the last are the last: their sums are not stored
#pragma unroll
    for (int t = 0; t < MT; ++t) pa[t] = p.A + (int64_t)min(m0 + t * 16 + i, p.M - 1) * p.lda;
#pragma unroll
    for (int t = 0; t < NT; ++t) pb[t] = p.B + (int64_t)min(n0 + t * 16 + i, p.N - 1) * p.ldb;
    i32x4 acc[MT][NT] = {};
    for (int k0 = wave * 128; k0 < p.K; k0 += WAVES * 128) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = k0 + g * 32 + h * 16;
            i32x4 a[MT], b[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) b[t] = chunk(pb[t], k, p.K);
#pragma unroll
            for (int t = 0; t < MT; ++t) a[t] = own_bytes(chunk(pa[t], k, p.K), k, p.K);
#pragma unroll
            for (int u = 0; u < MT; ++u)
#pragma unroll
                for (int t = 0; t < NT; ++t)
                    acc[u][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[t], a[u], acc[u][t], 0, 0, 0);
        }
    }
#pragma unroll
    for (int u = 0; u < MT; ++u)
#pragma unroll
        for (int t = 0; t < NT; ++t) part[wave][u * NT + t][lane] = acc[u][t];
    __syncthreads();
    for (int q = wave; q < MT * NT; q += WAVES) {
        i32x4 s = part[0][q][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) s += part[w][q][lane];
        store4<T>(p, m0 + q / NT * 16 + i, n0 + q % NT * 16 + g * 4, s);
    }
}

// ------------------------------------------------------------- many rows of A
//
// A work-group makes a BM x BN tile of C, its WM x WN waves a part each.  Both
// operands pass through LDS in K-blocks of 128 bytes, two stages of it: while
// one is multiplied the next is copied straight from memory into the other
// (DMA; operands whose rows start at multiples of four bytes), or is in flight
// to registers and written there afterwards (any other alignment).
// A row's eight 16-byte chunks lie in LDS with their position's low bits
// exchanged by the row's, so that the sixteen rows a wave reads at once, 128
// bytes apart, lie in different banks.

// Which row of the wave's 16 TN rows of B element `i` of its tile `t` is: a
// lane's accumulators of all tiles are then neighbours in a row of C.
template <int TN>
__device__ __forceinline__ int b_row(int t, int i) { return (i >> 2) * (4 * TN) + t * 4 + (i & 3); }

__device__ __forceinline__ int swizzle_a(int row) { return row & 7; }
// of the rows that b_row gives to neighbouring lanes
template <int TN>
__device__ __forceinline__ int swizzle_b(int row) { return (row & 3) | (row / (4 * TN) & 1) << 2; }

// A tile's rows of an operand for copies from memory straight into LDS.  They
// stop at the operand's last element (its four-byte word, which lies in memory
// whole): the last row's last chunk may reach past it.
struct Source {
    __amdgpu_buffer_rsrc_t rs;
    __device__ __forceinline__ Source(const int8_t *at, int64_t rows, int64_t ld, int K)
    {
        const int64_t bytes = ((rows - 1) * ld + K + 3) & ~(int64_t)3;
        rs = __builtin_amdgcn_make_buffer_rsrc((void *)at, 0, bytes < 0x7fffffff ? (int)bytes : 0x7fffffff, 0x00020000);
    }
    // the wave's 64 lanes' 16 bytes at off + k, one after the other to `to`; zeros for off < 0
    __device__ __forceinline__ void copy16(int8_t *to, int off, int k) const
    {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void *)to, 16, off, k, 0, 0);
    }
};

template <typename T, int BM, int BN, int WM, int WN, bool DMA>
__global__ void __launch_bounds__(WM * WN * 64) gemm_i8_tile_kernel(Args p, int tiles_m, int tiles_n, int group_m)
{
    constexpr int BK = 128, NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16, STAGE = (BM + BN) * BK;
    constexpr int LA = BM / (8 * NW), LB = BN / (8 * NW);  // copies of 16 bytes a lane, for A and for B
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && TM * WM * 16 == BM && TN * WN * 16 == BN, "whole copies");
    __shared__ __attribute__((aligned(16))) int8_t lds[2 * STAGE];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    const int wm = wave / WN, wn = wave % WN;
    int tm, tn;
    pk::tile_of_ints(tiles_m, tiles_n, group_m, pk::xcd_tile(blockIdx.x, tiles_m * tiles_n, 8), tm, tn);
    const int m0 = tm * BM, n0 = tn * BN, K = p.K;
    const int8_t *A = p.A + (int64_t)m0 * p.lda, *B = p.B + (int64_t)n0 * p.ldb;
    const int rows_a = p.M - m0, rows_b = p.N - n0;

    // copy slot u of this lane: row (u NW + wave) 8 + lane / 8 of the tile, chunk position lane % 8
    int off_a[LA], off_b[LB], k_a[LA], k_b[LB];
#pragma unroll
    for (int u = 0; u < LA; ++u) {
        const int r = (u * NW + wave) * 8 + lane / 8;
        k_a[u] = ((lane & 7) ^ swizzle_a(r)) * 16;
        off_a[u] = r < rows_a ? r * (int)p.lda + k_a[u] : (int)0x80000000;
    }
#pragma unroll
    for (int u = 0; u < LB; ++u) {
        const int r = (u * NW + wave) * 8 + lane / 8;
        k_b[u] = ((lane & 7) ^ swizzle_b<TN>(r)) * 16;
        off_b[u] = r < rows_b ? r * (int)p.ldb + k_b[u] : (int)0x80000000;
    }
    const Source src_a(A, rows_a, p.lda, K), src_b(B, rows_b, p.ldb, K);
    auto copy = [&](int k0, int8_t *stage) {
        const bool whole = k0 + BK <= K;
#pragma unroll
        for (int u = 0; u < LA; ++u)
            src_a.copy16(stage + (u * NW + wave) * 1024, whole || k0 + k_a[u] < K ? off_a[u] : (int)0x80000000, k0);
#pragma unroll
        for (int u = 0; u < LB; ++u)
            src_b.copy16(stage + BM * BK + (u * NW + wave) * 1024, whole || k0 + k_b[u] < K ? off_b[u] : (int)0x80000000,
                         k0);
    };
    i32x4 in_a[DMA ? 1 : LA], in_b[DMA ? 1 : LB];
    auto load = [&](int k0) {
        const bool whole = k0 + BK <= K;
#pragma unroll
        for (int u = 0; u < LA; ++u) {
            in_a[u] = i32x4{0, 0, 0, 0};
            if (off_a[u] >= 0 && (whole || k0 + k_a[u] < K)) {
                const int8_t *row = A + (off_a[u] - k_a[u]);
                in_a[u] = whole ? *reinterpret_cast<const i32x4_u *>(row + k0 + k_a[u])
                                : own_bytes(chunk(row, k0 + k_a[u], K), k0 + k_a[u], K);
            }
        }
#pragma unroll
        for (int u = 0; u < LB; ++u) {
            in_b[u] = i32x4{0, 0, 0, 0};
            if (off_b[u] >= 0 && (whole || k0 + k_b[u] < K)) {
                const int8_t *row = B + (off_b[u] - k_b[u]);
                in_b[u] = whole ? *reinterpret_cast<const i32x4_u *>(row + k0 + k_b[u]) : chunk(row, k0 + k_b[u], K);
            }
        }
    };
    auto put = [&](int8_t *stage) {
#pragma unroll
        for (int u = 0; u < LA; ++u)
            *reinterpret_cast<i32x4 *>(stage + (u * NW + wave) * 1024 + lane * 16) = in_a[u];
#pragma unroll
        for (int u = 0; u < LB; ++u)
            *reinterpret_cast<i32x4 *>(stage + BM * BK + (u * NW + wave) * 1024 + lane * 16) = in_b[u];
    };
    auto barrier = [] {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    i32x4 acc[TM][TN] = {};
    auto multiply = [&](const int8_t *stage) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            i32x4 a[TM], b[TN];
#pragma unroll
            for (int u = 0; u < TM; ++u) {
                const int r = (wm * TM + u) * 16 + i;
                a[u] = *reinterpret_cast<const i32x4 *>(stage + r * BK + ((h * 4 + g) ^ swizzle_a(r)) * 16);
            }
#pragma unroll
            for (int t = 0; t < TN; ++t) {
                const int r = wn * TN * 16 + b_row<TN>(t, i);
                b[t] = *reinterpret_cast<const i32x4 *>(stage + BM * BK + r * BK + ((h * 4 + g) ^ swizzle_b<TN>(r)) * 16);
            }
#pragma unroll
            for (int u = 0; u < TM; ++u)
#pragma unroll
                for (int t = 0; t < TN; ++t)
                    acc[u][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[t], a[u], acc[u][t], 0, 0, 0);
        }
    };

    const int blocks = (K + BK - 1) / BK;
    if constexpr (DMA) {
        copy(0, lds);
    } else {
        load(0);
        put(lds);
    }
    for (int kb = 0; kb < blocks; ++kb) {
        int8_t *now = lds + (kb & 1) * STAGE, *next = lds + (~kb & 1) * STAGE;
        barrier();
        if (DMA && kb + 1 == blocks && K % 16 != 0) {
            // the bytes of A's rows past K, copied with the last chunk, are
            // zeroed: what the same bytes of B hold then has no part
            for (int r = threadIdx.x; r < BM; r += NW * 64) {
                const int k = K - kb * BK;
                int8_t *c = now + r * BK + (k / 16 ^ swizzle_a(r)) * 16;
                for (int j = k % 16; j < 16; ++j) c[j] = 0;
            }
            barrier();
        }
        if (kb + 1 < blocks) {
            if constexpr (DMA)
                copy((kb + 1) * BK, next);
            else
                load((kb + 1) * BK);
        }
        multiply(now);
        if (!DMA && kb + 1 < blocks) put(next);
    }

    // lane: row u 16 + i of the wave's part, 4 TN columns from g 4 TN on
#pragma unroll
    for (int u = 0; u < TM; ++u)
#pragma unroll
        for (int t = 0; t < TN; ++t)
            store4<T>(p, m0 + (wm * TM + u) * 16 + i, n0 + wn * TN * 16 + g * (4 * TN) + t * 4, acc[u][t]);
}

// K == 0: the bias, or zeros.
template <typename T>
__global__ void __launch_bounds__(256) gemm_i8_empty_kernel(Args p)
{
    const int64_t total = (int64_t)p.M * p.N;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * 256) {
        const int64_t m = e / p.N, n = e - m * p.N;
        ((T *)p.C)[m * p.ldc + n] = (T)(p.bias ? p.bias[n] : 0.f);
    }
}

// ---------------------------------------------------------------- launches

template <typename T, int BM, int BN, int WM, int WN>
void launch_tile(const Args &a, bool dma, hipStream_t s)
{
    const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN;
    const dim3 grid((unsigned)(tiles_m * tiles_n)), block(WM * WN * 64);
    if (dma)
        hipLaunchKernelGGL((gemm_i8_tile_kernel<T, BM, BN, WM, WN, true>), grid, block, 0, s, a, tiles_m, tiles_n, 4);
    else
        hipLaunchKernelGGL((gemm_i8_tile_kernel<T, BM, BN, WM, WN, false>), grid, block, 0, s, a, tiles_m, tiles_n, 4);
}

template <typename T>
int launch(const Args &a, hipStream_t s)
{
    if (a.K == 0) {
        const int64_t blocks = ((int64_t)a.M * a.N + 255) / 256;
        hipLaunchKernelGGL((gemm_i8_empty_kernel<T>), dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, s, a);
        if (hipGetLastError() != hipSuccess) return PK_ERR_LAUNCH;
        pk::api_ran("gemm_i8_empty");
        return PK_OK;
    }
    const bool dma = ((uintptr_t)a.A | (uintptr_t)a.B | (uintptr_t)a.lda | (uintptr_t)a.ldb) % 4 == 0;
    if (a.M > 64 && a.lda <= 1 << 22 && a.ldb <= 1 << 22) {
        if ((int64_t)a.M * a.N >= 256 * 256 * 128) {
            launch_tile<T, 256, 256, 2, 4>(a, dma, s);
            pk::api_ran(dma ? "gemm_i8_256x256" : "gemm_i8_256x256_unaligned");
        } else {
            launch_tile<T, 128, 128, 2, 2>(a, dma, s);
            pk::api_ran(dma ? "gemm_i8_128x128" : "gemm_i8_128x128_unaligned");
        }
        return hipGetLastError() == hipSuccess ? PK_OK : PK_ERR_LAUNCH;
    }
    hipLaunchKernelGGL((gemm_i8_rows_kernel<T, 1, 1, 8>), dim3((unsigned)((a.N + 15) / 16), (unsigned)((a.M + 15) / 16)),
                       dim3(512), 0, s, a);
    if (hipGetLastError() != hipSuccess) return PK_ERR_LAUNCH;
    pk::api_ran("gemm_i8_16x16");
    return PK_OK;
}

}  // namespace

extern "C" int pk_gemm_i8(int64_t M, int64_t N, int64_t K, const int8_t *A, int64_t lda, const float *a_scale,
                          const int8_t *B, int64_t ldb, const float *b_scale, const float *bias, void *C, int dtype,
                          int64_t ldc, void *stream)
{
    using namespace pk;
    using namespace pk::checks;
    api_begin();
    const int size = dtype_size(dtype);
    if (M < 0) return api_invalid(1);
    if (N < 0) return api_invalid(2);
    if (K < 0) return api_invalid(3);
    if (short_ld(lda, K)) return api_invalid(5);
    if (short_ld(ldb, K)) return api_invalid(8);
    if (!size) return api_invalid(12);
    if (short_ld(ldc, N)) return api_invalid(13);
    if (M == 0 || N == 0) return PK_OK;
    if (too_large({M, N, lda, ldb, ldc}) || K > 131071) return PK_ERR_NOT_SUPPORTED;
    if (misaligned(bias, 4)) return api_invalid(10);
    if (!C || misaligned(C, size)) return api_invalid(11);
    const Span sc = span(C, M, N, ldc, size);
    if (K) {
        if (!A) return api_invalid(4);
        if (!a_scale || misaligned(a_scale, 4)) return api_invalid(6);
        if (!B) return api_invalid(7);
        if (!b_scale || misaligned(b_scale, 4)) return api_invalid(9);
        if (overlap(sc, span(A, M, K, lda, 1)) || overlap(sc, span(a_scale, 1, M, M, 4)) ||
            overlap(sc, span(B, N, K, ldb, 1)) || overlap(sc, span(b_scale, 1, N, N, 4)))
            return api_invalid(11);
    }
    if (bias && overlap(sc, span(bias, 1, N, N, 4))) return api_invalid(11);
    const Args a = {A, B, a_scale, b_scale, bias, C, lda, ldb, ldc, (int)M, (int)N, (int)K};
    hipStream_t s = (hipStream_t)stream;
    return dtype == PK_F32 ? launch<float>(a, s) : dtype == PK_BF16 ? launch<bf16>(a, s) : launch<f16>(a, s);
}
