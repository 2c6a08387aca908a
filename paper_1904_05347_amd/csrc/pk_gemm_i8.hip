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
// operands pass through LDS in K-blocks of 128 bytes, STAGES of them: while one
// is multiplied the next ones are copied straight from memory (DMA; operands
// whose rows start at multiples of four bytes), or the next one is in flight to
// registers and written there afterwards (any other alignment; two stages).
//
// A block is multiplied in two halves of 64, and the operands of a half are read
// from LDS while the half before it is multiplied.  So the work-group's only
// barrier of a block stands where every wave has a half's operands in registers
// and its products ahead of it: nobody waits for LDS after a barrier.
//
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

// A tile's rows of an operand for copies from memory straight into LDS.  What
// lies past the operand's last element (its four-byte word, which lies in memory
// whole) is not read and arrives as zeros: rows past the last, and what the last
// row's last chunk has past its end.
struct Source {
    __amdgpu_buffer_rsrc_t rs;
    __device__ __forceinline__ Source(const int8_t *at, int64_t rows, int64_t ld, int K)
    {
        const int64_t bytes = ((rows - 1) * ld + K + 3) & ~(int64_t)3;
        rs = __builtin_amdgcn_make_buffer_rsrc((void *)at, 0, bytes < 0x7fffffff ? (int)bytes : 0x7fffffff, 0x00020000);
    }
    // the wave's 64 lanes' 16 bytes at off + k (k < K), one after the other to
    // `to`; zeros for off < 0.  Written out, because the compiler would wait for
    // every such copy before the next read of LDS, whichever stage that reads;
    // the kernel's own waits are at its barriers.  A copy's use of m0 comes one
    // wait state after it is set.
    __device__ __forceinline__ void copy16(int8_t *to, int off, int k) const
    {
        const unsigned at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void *)to;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                     :
                     : "s"(at), "v"(off), "s"(rs), "s"(k)
                     : "memory", "m0");
    }
};

template <typename T, int BM, int BN, int WM, int WN, int STAGES, bool DMA>
__global__ void __launch_bounds__(WM * WN * 64, 2) gemm_i8_tile_kernel(Args p, int tiles_m, int tiles_n, int group_m)
{
    constexpr int BK = 128, NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16, STAGE = (BM + BN) * BK;
    constexpr int LA = BM / (8 * NW), LB = BN / (8 * NW), L = LA + LB;  // copies of 16 bytes a lane and block
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && TM * WM * 16 == BM && TN * WN * 16 == BN, "whole copies");
    static_assert(DMA ? (STAGES - 2) * L < 64 : STAGES == 2, "copies in flight are counted in six bits");
    static_assert(BM <= 256 && BN <= 256, "offsets in a tile are 32-bit for leading dimensions up to kMostLd");
    __shared__ __attribute__((aligned(16))) int8_t lds[STAGES * STAGE];
    __shared__ __attribute__((aligned(16))) float factors[BM + 2 * BN];  // the scales of the tile's rows and columns, the bias
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15,
              g = lane >> 4;
    const int wm = wave / WN, wn = wave % WN;
    int tm, tn;
    pk::tile_of_ints(tiles_m, tiles_n, group_m, pk::xcd_tile(blockIdx.x, tiles_m * tiles_n, 8), tm, tn);
    const int m0 = tm * BM, n0 = tn * BN, K = p.K, blocks = (K + BK - 1) / BK;
    const int lda = (int)p.lda, ldb = (int)p.ldb;
    const int8_t *A = p.A + (int64_t)m0 * p.lda, *B = p.B + (int64_t)n0 * p.ldb;
    const int rows_a = p.M - m0, rows_b = p.N - n0;

    // copy u of this lane: row (u NW + wave) 8 + lane / 8 of the tile, chunk position lane % 8;
    // the swizzles do not depend on u
    const int row = wave * 8 + lane / 8;
    const int k_a = ((lane & 7) ^ swizzle_a(row)) * 16, k_b = ((lane & 7) ^ swizzle_b<TN>(row)) * 16;
    static_assert(8 * NW % (8 * TN) == 0, "swizzle_b");
    const Source src_a(A, rows_a, lda, K), src_b(B, rows_b, ldb, K);
    auto copy = [&]<bool WHOLE>(int kb, int stage) {
        const int k0 = kb * BK;
        const bool whole = WHOLE || k0 + BK <= K;
        const int oa = whole || k0 + k_a < K ? row * lda + k_a : (int)0x80000000;
        const int ob = whole || k0 + k_b < K ? row * ldb + k_b : (int)0x80000000;
        int8_t *to = lds + stage * STAGE + wave * 1024;
#pragma unroll
        for (int u = 0; u < LA; ++u) src_a.copy16(to + u * NW * 1024, oa + u * NW * 8 * lda, k0);
#pragma unroll
        for (int u = 0; u < LB; ++u) src_b.copy16(to + BM * BK + u * NW * 1024, ob + u * NW * 8 * ldb, k0);
    };
    i32x4 in_a[DMA ? 1 : LA], in_b[DMA ? 1 : LB];
    auto load = [&]<bool WHOLE>(int kb) {
        const int k0 = kb * BK;
        const bool whole = WHOLE || k0 + BK <= K;
        auto from = [&](const int8_t *base, int r, int rows, int ld, int k, bool left) {
            i32x4 v = {0, 0, 0, 0};
            if (r < rows && (whole || k < K)) {
                const int8_t *at = base + (int64_t)r * ld;
                v = whole ? *reinterpret_cast<const i32x4_u *>(at + k) : chunk(at, k, K);
                if (left && !whole) v = own_bytes(v, k, K);
            }
            return v;
        };
#pragma unroll
        for (int u = 0; u < LA; ++u) in_a[u] = from(A, row + u * NW * 8, rows_a, lda, k0 + k_a, true);
#pragma unroll
        for (int u = 0; u < LB; ++u) in_b[u] = from(B, row + u * NW * 8, rows_b, ldb, k0 + k_b, false);
    };
    auto put = [&](int stage) {
        int8_t *to = lds + stage * STAGE + wave * 1024 + lane * 16;
#pragma unroll
        for (int u = 0; u < LA; ++u) *reinterpret_cast<i32x4 *>(to + u * NW * 1024) = in_a[u];
#pragma unroll
        for (int u = 0; u < LB; ++u) *reinterpret_cast<i32x4 *>(to + BM * BK + u * NW * 1024) = in_b[u];
    };
    // this wave's reads of LDS are done, and its copies of all but the newest
    // `later` blocks have landed: the barrier then says so of every wave's
    auto barrier = [&](int later) {
        if (STAGES > 3 && later >= 2)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(STAGES > 3 ? 2 * L : 0) : "memory");
        else if (STAGES > 2 && later >= 1)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(STAGES > 2 ? L : 0) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // The bytes of A's rows past K that were copied with the last chunk are
    // zeroed: what the same bytes of B hold then has no part.
    auto cut = [&](int kb, int stage) {
        if (DMA && K % 16 != 0 && kb == blocks - 1) {
            for (int r = threadIdx.x; r < BM; r += NW * 64) {
                const int k = K - kb * BK;
                int8_t *c = lds + stage * STAGE + r * BK + (k / 16 ^ swizzle_a(r)) * 16;
                for (int j = k % 16; j < 16; ++j) c[j] = 0;
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        }
    };

    struct Half {
        i32x4 a[TM], b[TN];
    };
    const int at_a = (wm * TM * 16 + i) * BK, at_b = BM * BK + (wn * TN * 16 + b_row<TN>(0, i)) * BK;
    const int c_a = swizzle_a(i), c_b = swizzle_b<TN>(b_row<TN>(0, i));
    auto read = [&](Half &f, int stage, int h) {
        const int8_t *pa = lds + stage * STAGE + at_a + ((h * 4 + g) ^ c_a) * 16;
        const int8_t *pb = lds + stage * STAGE + at_b + ((h * 4 + g) ^ c_b) * 16;
#pragma unroll
        for (int t = 0; t < TN; ++t) f.b[t] = *reinterpret_cast<const i32x4 *>(pb + t * 4 * BK);
#pragma unroll
        for (int u = 0; u < TM; ++u) f.a[u] = *reinterpret_cast<const i32x4 *>(pa + u * 16 * BK);
    };
    i32x4 acc[TM][TN] = {};
    auto multiply = [&](const Half &f) {
#pragma unroll
        for (int u = 0; u < TM; ++u)
#pragma unroll
            for (int t = 0; t < TN; ++t)
                acc[u][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f.b[t], f.a[u], acc[u][t], 0, 0, 0);
    };

    float factor[(BM + 2 * BN + NW * 64 - 1) / (NW * 64)];
#pragma unroll
    for (int j = 0; j < (BM + 2 * BN + NW * 64 - 1) / (NW * 64); ++j) {
        const int e = threadIdx.x + j * NW * 64;
        const float *from = e < BM ? p.sa + min(m0 + e, p.M - 1) : e < BM + BN ? p.sb + min(n0 + e - BM, p.N - 1)
                            : p.bias && e < BM + 2 * BN ? p.bias + min(n0 + e - BM - BN, p.N - 1) : nullptr;
        factor[j] = from ? *from : 0.f;
    }
    auto keep_factors = [&] {
#pragma unroll
        for (int j = 0; j < (BM + 2 * BN + NW * 64 - 1) / (NW * 64); ++j)
            if ((BM + 2 * BN) % (NW * 64) == 0 || threadIdx.x + j * NW * 64 < BM + 2 * BN)
                factors[threadIdx.x + j * NW * 64] = factor[j];
    };

    Half f0, f1;
    if constexpr (DMA) {
#pragma unroll
        for (int s = 0; s < STAGES; ++s)
            if (s < blocks) copy.template operator()<false>(s, s);
        keep_factors();
        barrier(blocks - 1 < STAGES - 1 ? blocks - 1 : STAGES - 1);
    } else {
        load.template operator()<false>(0);
        put(0);
        keep_factors();
        barrier(0);
        if (blocks > 1) load.template operator()<false>(1);
    }
    cut(0, 0);
    read(f0, 0, 0);
    int now = 0;
    // a half's reads of LDS go between the products of the half before
    auto interleave = [] {
#pragma unroll
        for (int j = 0; j < TM + TN; ++j) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, TM * TN / (TM + TN), 0);
        }
    };
    // One block; MIDDLE: blocks up to kb + STAGES exist, and are whole.
    auto step = [&]<bool MIDDLE>(int kb) {
        const int next = now + 1 == STAGES ? 0 : now + 1;
        read(f1, now, 1);
        multiply(f0);
        interleave();
        if (MIDDLE || kb + 1 < blocks) {
            if constexpr (!DMA) put(next);
            // blocks kb + 2 .. kb + STAGES - 1 may still be on their way
            const int later = blocks - kb - 2;
            barrier(MIDDLE || later >= STAGES - 2 ? STAGES - 2 : later);
            if (!MIDDLE) cut(kb + 1, next);
            if constexpr (DMA) {
                if (MIDDLE || kb + STAGES < blocks) copy.template operator()<MIDDLE>(kb + STAGES, now);
            } else {
                if (MIDDLE || kb + 2 < blocks) load.template operator()<MIDDLE>(kb + 2);
            }
            read(f0, next, 0);
        }
        multiply(f1);
        interleave();
        now = next;
    };
    int kb = 0;
    for (; (kb + STAGES + 1) * BK <= K; ++kb) step.template operator()<true>(kb);
    for (; kb < blocks; ++kb) step.template operator()<false>(kb);

    // lane: row u 16 + i of the wave's part, 4 TN columns from g 4 TN on
    const int ml = wm * TM * 16 + i, nl = wn * TN * 16 + g * (4 * TN);
    float sb[4 * TN], bias[4 * TN];
#pragma unroll
    for (int j = 0; j < 4 * TN; ++j) {
        sb[j] = factors[BM + nl + j];
        bias[j] = factors[BM + BN + nl + j];
    }
#pragma unroll
    for (int u = 0; u < TM; ++u) {
        const float sa = factors[ml + u * 16];
        const int m = m0 + ml + u * 16, n = n0 + nl;
        T *c = (T *)p.C + (int64_t)m * p.ldc + n;
        if (m >= p.M) continue;
        constexpr int E = 4 * TN < 16 / (int)sizeof(T) ? 4 * TN : 16 / (int)sizeof(T);
#pragma unroll
        for (int j = 0; j < 4 * TN; j += E) {
            typename Pack<T, E>::V v;
#pragma unroll
            for (int e = 0; e < E; ++e)
                v[e] = (T)fmaf((float)acc[u][(j + e) / 4][(j + e) % 4], sa * sb[j + e], bias[j + e]);
            if (n + j + E <= p.N) {
                *reinterpret_cast<typename Pack<T, E>::U *>(c + j) = v;
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (n + j + e < p.N) c[j + e] = v[e];
            }
        }
    }
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

constexpr int64_t kMostLd = 1 << 22;  // of gemm_i8_tile_kernel

template <typename T, int BM, int BN, int WM, int WN, int STAGES>
void launch_tile(const Args &a, bool dma, hipStream_t s)
{
    const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN;
    const dim3 grid((unsigned)(tiles_m * tiles_n)), block(WM * WN * 64);
    if (dma)
        hipLaunchKernelGGL((gemm_i8_tile_kernel<T, BM, BN, WM, WN, STAGES, true>), grid, block, 0, s, a, tiles_m, tiles_n, 4);
    else
        hipLaunchKernelGGL((gemm_i8_tile_kernel<T, BM, BN, WM, WN, 2, false>), grid, block, 0, s, a, tiles_m, tiles_n, 4);
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
    if (a.M > 64 && a.lda <= kMostLd && a.ldb <= kMostLd) {
        if ((int64_t)a.M * a.N >= 256 * 256 * 128) {
            launch_tile<T, 256, 256, 2, 4, 2>(a, dma, s);
            pk::api_ran(dma ? "gemm_i8_256x256" : "gemm_i8_256x256_unaligned");
        } else {
            launch_tile<T, 128, 128, 2, 2, 4>(a, dma, s);
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
