// pk_gemm_i8.hip -- products of 8-bit integers with a scale for each row of
// either operand: C[m][n] = sa[m] sb[n] sum_k A[m][k] B[n][k] + bias[n].
#include "pk_i8.hpp"
#include "pk_i8_checks.hpp"
#include "pk_partition.hpp"

namespace {

using pk::bf16;
using pk::f16;
using pk::Pack;
using pk::rounded;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_u __attribute__((aligned(1)));

struct Args {
    const int8_t *A, *B;
    const float *sa, *sb, *bias;
    void *C;
    int64_t lda, ldb, ldc;
    int M, N, K;
    bool beyond_cache;  // C is written past the last-level cache
};

// ------------------------------------------------------------ few rows of A
//
// A work-group makes 8 rows x 8 columns of C; its waves share K in blocks of
// 128 and add their sums through LDS.  Operands go from memory to the registers
// the matrix instruction reads: nothing is staged.
// v_mfma_i32_16x16x64_i8 multiplies 16 rows of each operand, 64 bytes of each; a
// load that follows it touches half of 16 memory lines, which runs at half the
// rate of 8 whole ones.  So its 16 rows are the two halves of the 128 bytes of 8
// rows, of either operand: of its 16 x 16 sums those count whose halves are the
// same, and the two 8 x 8 parts are added at the end.
// Bound by the latency of a launch and of memory while B is small, by reading B
// beyond that: one row, 4096 x 4096 4.9 us (a launch 2 to 3; reading B at a large
// copy's rate 3.3), 8192 x 8192 12.3 us (5.5 TB/s).  Each eight rows read B again.

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

template <typename T, int WAVES, int U>
__global__ void __launch_bounds__(WAVES * 64) gemm_i8_rows_kernel(Args p)
{
    __shared__ i32x4 part[WAVES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4, K = p.K;
    const int n0 = blockIdx.x * 8, m0 = blockIdx.y * 8;
    // rows beyond the last are the last: their sums are not stored
    const int8_t *pa = p.A + (int64_t)min(m0 + i % 8, p.M - 1) * p.lda, *pb = p.B + (int64_t)min(n0 + i % 8, p.N - 1) * p.ldb;
    // the scales of this lane's row and columns, before they are needed
    const int m = min(m0 + i % 8, p.M - 1), n = n0 + g % 2 * 4;
    const float sa = p.sa[m];
    float sb[4], bias[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        sb[r] = p.sb[min(n + r, p.N - 1)];
        bias[r] = p.bias ? p.bias[min(n + r, p.N - 1)] : 0.f;
    }
    i32x4 acc = {0, 0, 0, 0};
    auto blocks = [&]<int V, bool WHOLE>(int k0) {
        i32x4 a[V], b[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int k = k0 + v * (WAVES * 128) + (i / 8 * 4 + g) * 16;
            b[v] = WHOLE ? *reinterpret_cast<const i32x4_u *>(pb + k) : chunk(pb, k, K);
            a[v] = WHOLE ? *reinterpret_cast<const i32x4_u *>(pa + k) : own_bytes(chunk(pa, k, K), k, K);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[v], a[v], acc, 0, 0, 0);
    };
    int k0 = wave * 128;
    for (; k0 + (U - 1) * (WAVES * 128) + 128 <= K; k0 += U * WAVES * 128) blocks.template operator()<U, true>(k0);
    for (; k0 + 128 <= K; k0 += WAVES * 128) blocks.template operator()<1, true>(k0);
    if (k0 < K) blocks.template operator()<1, false>(k0);
    part[wave][lane] = acc;
    __syncthreads();
    // lane: row i % 8, columns g 4 to g 4 + 3 of the first half's sums (g < 2, i < 8)
    if (wave > 0 || g >= 2 || i >= 8 || m0 + i >= p.M || n >= p.N) return;
    i32x4 s = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += part[w][lane] + part[w][lane + 2 * 16 + 8];
    typename Pack<T, 4>::V v;
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = rounded<T>(fmaf((float)s[r], sa * sb[r], bias[r]));
    T *c = (T *)p.C + (int64_t)m * p.ldc + n;
    if (n + 4 <= p.N) {
        *reinterpret_cast<typename Pack<T, 4>::U *>(c) = v;
        return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (n + r < p.N) c[r] = v[r];
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
// bytes apart, lie in different banks (no conflicts counted).
//
// Where there are few tiles, KG groups of waves share K, each with stages of its
// own, and add their sums through LDS: half the steps that follow one another
// (32 x 4096 x 4096 in tiles of 32 x 32: 7.2 us in two groups, 8.0 in one; in tiles
// of 16 x 16, four groups, 5.9).
//
// What bounds it.  256 x 256, 8192^3: 417 to 435 us from run to run, 2530 to 2640
// TOP/s: the matrix cores are busy for two thirds of the time at the 1.9 GHz that the
// power leaves; the same loop without the copies takes 330 us, with copies that stay
// in L2 377.  128 x 128 and less (4096 x 4096 weights: 1024 rows 19.7 us, 512 13.4,
// 256 9.5): the copies' arrival.  A CU reads 70 to 85 GB/s while it goes through K,
// four fifths of it from L2, from which alone it reads 152 (105 to 110 from the
// last-level cache); half of the waves' cycles are waits, and the matrix cores are
// busy for 10 to 26 % of the time.  Fewer rows: the latency of a launch, the first
// block and the stores (32 rows 5.9 us).  128 bytes of a row that start inside a
// memory line are two lines: operands whose rows start at multiples of 16 bytes but
// not of 128 take up to 1.3 times as long, those at odd addresses twice (4096^3 114
// us, 53): with a workspace larger products copy such rows to whole lines first.

// Which row of the wave's 16 TN rows of B element `i` of its tile `t` is: the
// accumulators of P tiles, 4 P in a lane, are neighbours in a row of C (P such
// that they are one store of 16 bytes), and so are those of four lanes.
template <int P>
__device__ __forceinline__ int b_row(int t, int i) { return t / P * (16 * P) + (i >> 2) * (4 * P) + t % P * 4 + (i & 3); }

__device__ __forceinline__ int swizzle_a(int row) { return row & 7; }
// of the rows that b_row gives to neighbouring lanes
template <int P>
__device__ __forceinline__ int swizzle_b(int row) { return (row & 3) | (row / (4 * P) & 1) << 2; }

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
    // the kernel's own waits are at its barriers.  The compiler does not see what
    // the copy has to keep from the instructions before it either: m0, where `to` is
    // passed, is read one wait state after it is set, scalar operands five after a
    // vector instruction that may have made them.
    __device__ __forceinline__ void copy16(int8_t *to, int off, int k) const
    {
        const unsigned at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void *)to;
        asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                     :
                     : "{m0}"(at), "v"(off), "s"(rs), "s"(k)
                     : "memory");
    }
};

template <typename T, int BM, int BN, int WM, int WN, int KG, int STAGES, bool DMA>
__global__ void __launch_bounds__(KG * WM * WN * 64, 2)
    gemm_i8_tile_kernel(Args p, int tiles_m, int tiles_n, int group_m)
{
    constexpr int BK = 128, NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16, STAGE = (BM + BN) * BK;
    constexpr int LA = BM / (8 * NW), LB = BN / (8 * NW), L = LA + LB;  // copies of 16 bytes a lane and block
    constexpr int THREADS = KG * NW * 64;
    constexpr int P = TN * (int)sizeof(T) < 4 ? TN : 4 / (int)sizeof(T);  // tiles of a 16-byte store
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && TM * WM * 16 == BM && TN * WN * 16 == BN, "whole copies");
    static_assert(DMA ? STAGES <= 4 && (STAGES - 2) * L < 64 : STAGES == 2, "copies in flight are counted in six bits");
    static_assert(BM <= 256 && BN <= 256, "offsets in a tile are 32-bit for leading dimensions up to kMostLd");
    static_assert((KG - 1) * BM * BN * 4 <= KG * STAGES * STAGE, "sums of the other groups fit the stages");
    __shared__ __attribute__((aligned(16))) int8_t lds_all[KG * STAGES * STAGE];
    __shared__ __attribute__((aligned(16))) float factors[BM + 2 * BN];  // the scales of the tile's rows and columns, the bias
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave_all / NW, wave = wave_all % NW;
    const int wm = wave / WN, wn = wave % WN;
    int tm, tn;
    pk::tile_of_ints(tiles_m, tiles_n, group_m, pk::xcd_tile(blockIdx.x, tiles_m * tiles_n, 8), tm, tn);
    const int m0 = tm * BM, n0 = tn * BN, K = p.K;
    const int lda = (int)p.lda, ldb = (int)p.ldb;
    const int8_t *A = p.A + (int64_t)m0 * p.lda, *B = p.B + (int64_t)n0 * p.ldb;
    const int rows_a = p.M - m0, rows_b = p.N - n0;
    // this group's blocks: `count` from `first` on, at most `per`, the number of steps of every group
    const int blocks = (K + BK - 1) / BK, per = (blocks + KG - 1) / KG, first = group * per;
    const int count = KG == 1 ? blocks : max(0, min(per, blocks - first));
    int8_t *const lds = lds_all + group * (STAGES * STAGE);

    // copy u of this lane: row (u NW + wave) 8 + lane / 8 of the tile, chunk position lane % 8;
    // the swizzles do not depend on u
    const int row = wave * 8 + lane / 8;
    const int k_a = ((lane & 7) ^ swizzle_a(row)) * 16, k_b = ((lane & 7) ^ swizzle_b<P>(row)) * 16;
    static_assert(NW % P == 0 && TN % P == 0, "swizzle_b");
    const Source src_a(A, rows_a, lda, K), src_b(B, rows_b, ldb, K);
    auto copy = [&]<bool WHOLE>(int j, int stage) {
        const int k0 = (first + j) * BK;
        const bool whole = WHOLE || k0 + BK <= K;
        const int oa = whole || k0 + k_a < K ? row * lda + k_a : (int)0x80000000;
        const int ob = whole || k0 + k_b < K ? row * ldb + k_b : (int)0x80000000;
        int8_t *to = lds + stage * STAGE + wave * 1024;
#pragma unroll
        for (int u = 0; u < LA; ++u) src_a.copy16(to + u * NW * 1024, oa + u * NW * 8 * lda, k0);
#pragma unroll
        for (int u = 0; u < LB; ++u) src_b.copy16(to + BM * BK + u * NW * 1024, ob + u * NW * 8 * ldb, k0);
    };
    // The bytes of A's rows past K that were copied with the last chunk are
    // zeroed: what the same bytes of B hold then has no part.
    auto cut = [&](int j, int stage) {
        const int left = K - (first + j) * BK - k_a;  // of this lane's chunks
        if (left > 0 && left < 16) {
            int8_t *c = lds + stage * STAGE + wave * 1024 + lane * 16;
#pragma unroll
            for (int u = 0; u < LA; ++u)
                for (int e = left; e < 16; ++e) c[u * NW * 1024 + e] = 0;
        }
    };
    i32x4 in_a[DMA ? 1 : LA], in_b[DMA ? 1 : LB];
    auto load = [&]<bool WHOLE>(int j) {
        const int k0 = (first + j) * BK;
        const bool whole = WHOLE || k0 + BK <= K;
        auto from = [&](i32x4 &in, const int8_t *base, int r, int rows, int ld, int k, bool left) {
            const int8_t *at = base + (int64_t)min(r, rows - 1) * ld;  // rows beyond the last: their sums are not stored
            if (whole) {
                in = *reinterpret_cast<const i32x4_u *>(at + k);
            } else {
                in = k < K ? chunk(at, k, K) : i32x4{0, 0, 0, 0};
                if (left) in = own_bytes(in, k, K);
            }
        };
#pragma unroll
        for (int u = 0; u < LA; ++u) from(in_a[u], A, row + u * NW * 8, rows_a, lda, k0 + k_a, true);
#pragma unroll
        for (int u = 0; u < LB; ++u) from(in_b[u], B, row + u * NW * 8, rows_b, ldb, k0 + k_b, false);
    };
    auto put = [&](int stage) {
        int8_t *to = lds + stage * STAGE + wave * 1024 + lane * 16;
#pragma unroll
        for (int u = 0; u < LA; ++u) *reinterpret_cast<i32x4 *>(to + u * NW * 1024) = in_a[u];
#pragma unroll
        for (int u = 0; u < LB; ++u) *reinterpret_cast<i32x4 *>(to + BM * BK + u * NW * 1024) = in_b[u];
    };
    // this wave's copies of all but the newest `later` blocks have landed
    auto landed = [&](int later) {
        if (STAGES > 3 && later >= 2)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(STAGES > 3 ? 2 * L : 0) : "memory");
        else if (STAGES > 2 && later >= 1)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(STAGES > 2 ? L : 0) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    // this wave's accesses of LDS are done: the barrier then says so of every wave's
    auto barrier = [] {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    struct Half {
        i32x4 a[TM], b[TN];
    };
    const int at_a = (wm * TM * 16 + i) * BK, at_b = BM * BK + (wn * TN * 16 + b_row<P>(0, i)) * BK;
    const int c_a = swizzle_a(i), c_b = swizzle_b<P>(b_row<P>(0, i));
    auto read = [&](Half &f, int stage, int h) {
        const int8_t *pa = lds + stage * STAGE + at_a + ((h * 4 + g) ^ c_a) * 16;
        const int8_t *pb = lds + stage * STAGE + at_b + ((h * 4 + g) ^ c_b) * 16;
#pragma unroll
        for (int t = 0; t < TN; ++t) f.b[t] = *reinterpret_cast<const i32x4 *>(pb + b_row<P>(t, 0) * BK);
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
    // a half's reads of LDS go between the products of the half before
    auto interleave = [] {
#pragma unroll
        for (int j = 0; j < TM + TN; ++j) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, TM * TN > TM + TN ? TM * TN / (TM + TN) : 1, 0);
        }
    };

    constexpr int FACTORS = (BM + 2 * BN + THREADS - 1) / THREADS;
    float factor[FACTORS];
#pragma unroll
    for (int j = 0; j < FACTORS; ++j) {
        const int e = threadIdx.x + j * THREADS;
        const float *from = e < BM ? p.sa + min(m0 + e, p.M - 1) : e < BM + BN ? p.sb + min(n0 + e - BM, p.N - 1)
                            : p.bias && e < BM + 2 * BN ? p.bias + min(n0 + e - BM - BN, p.N - 1) : nullptr;
        factor[j] = from ? *from : 0.f;
    }

    Half f0, f1;
    if constexpr (DMA) {
#pragma unroll
        for (int s = 0; s < STAGES; ++s)
            if (s < count) copy.template operator()<false>(s, s);
    } else if (count > 0) {
        load.template operator()<false>(0);
        put(0);
    }
#pragma unroll
    for (int j = 0; j < FACTORS; ++j)
        if ((BM + 2 * BN) % THREADS == 0 || threadIdx.x + j * THREADS < BM + 2 * BN)
            factors[threadIdx.x + j * THREADS] = factor[j];
    if constexpr (DMA) {
        landed(count - 1 < STAGES - 1 ? count - 1 : STAGES - 1);
        cut(0, 0);
    }
    barrier();
    if (!DMA && count > 1) load.template operator()<false>(1);
    if (count > 0) read(f0, 0, 0);
    int now = 0;
    // a large tile's copies are issued after the reads that its products wait for
    // (4096^3 60.3 us, 62.7 before them; the smaller tiles the other way round)
    constexpr bool LATE = BM * BN > 128 * 128;
    // One block; MIDDLE: the group's blocks up to j + STAGES exist, and are whole.
    auto step = [&]<bool MIDDLE>(int j) {
        const int next = now + 1 == STAGES ? 0 : now + 1;
        if (MIDDLE || j < count) {
            read(f1, now, 1);
            multiply(f0);
            interleave();
        }
        if (MIDDLE || j + 1 < per) {
            if constexpr (DMA) {
                // blocks j + 2 .. j + STAGES - 1 may still be on their way
                const int later = count - j - 2;
                landed(MIDDLE || later >= STAGES - 2 ? STAGES - 2 : later);
                if (!MIDDLE) cut(j + 1, next);
            } else {
                if (MIDDLE || j + 1 < count) put(next);
            }
            barrier();
            if (LATE && (MIDDLE || j + 1 < count)) read(f0, next, 0);
            if constexpr (DMA) {
                if (MIDDLE || j + STAGES < count) copy.template operator()<MIDDLE>(j + STAGES, now);
            } else {
                if (MIDDLE || j + 2 < count) load.template operator()<MIDDLE>(j + 2);
            }
            if (!LATE && (MIDDLE || j + 1 < count)) read(f0, next, 0);
        }
        if (MIDDLE || j < count) {
            multiply(f1);
            interleave();
        }
        now = next;
    };
    int j = 0;
    for (const int whole = min(count, K / BK - first) - STAGES; j < whole; ++j) step.template operator()<true>(j);
    for (; j < per; ++j) step.template operator()<false>(j);

    if constexpr (KG > 1) {
        // the groups' sums are added in the first one's registers
        i32x4 *const sums = (i32x4 *)lds_all;
        barrier();
        if (group > 0) {
#pragma unroll
            for (int u = 0; u < TM; ++u)
#pragma unroll
                for (int t = 0; t < TN; ++t) sums[(((group - 1) * NW + wave) * (TM * TN) + u * TN + t) * 64 + lane] = acc[u][t];
        }
        barrier();
        if (group > 0) return;
#pragma unroll
        for (int o = 0; o < KG - 1; ++o)
#pragma unroll
            for (int u = 0; u < TM; ++u)
#pragma unroll
                for (int t = 0; t < TN; ++t) acc[u][t] += sums[((o * NW + wave) * (TM * TN) + u * TN + t) * 64 + lane];
    }

    // lane: row u 16 + i of the wave's part, E columns from q 16 P + g E on
    constexpr int E = 4 * P;
    const int ml = wm * TM * 16 + i, nl = wn * TN * 16 + g * E;
    float sb[TN / P][E], bias[TN / P][E];
#pragma unroll
    for (int q = 0; q < TN / P; ++q)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            sb[q][e] = factors[BM + nl + q * 16 * P + e];
            bias[q][e] = factors[BM + BN + nl + q * 16 * P + e];
        }
    typedef typename Pack<T, E>::V V;
    // all of the part's results, by stores of one kind
    auto store_all = [&]<bool BEYOND_CACHE>() {
        // the compiler would make one plain store of both kinds' branches
        if (BEYOND_CACHE) asm volatile("");
        auto store = [&](int m, int n, const V &v) {
            if (m >= p.M) return;
            T *c = (T *)p.C + (int64_t)m * p.ldc + n;
            if (n + E <= p.N) {
                if constexpr (BEYOND_CACHE)
                    __builtin_nontemporal_store(v, reinterpret_cast<typename Pack<T, E>::U *>(c));
                else
                    *reinterpret_cast<typename Pack<T, E>::U *>(c) = v;
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (n + e < p.N) c[e] = v[e];
            }
        };
#pragma unroll
        for (int u = 0; u < TM; ++u) {
            const float sa = factors[ml + u * 16];
            const int m = m0 + ml + u * 16, n = n0 + nl;
            auto value = [&](int q) {
                V v;
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = rounded<T>(fmaf((float)acc[u][q * P + e / 4][e % 4], sa * sb[q][e], bias[q][e]));
                return v;
            };
            if constexpr (TN / P % 2 == 0 && sizeof(V) == 16) {
                // Four lanes' stores are 64 neighbouring bytes.  Neighbouring lanes
                // exchange halves, so that a store has eight lanes' 128 bytes, a
                // memory line, of every other row.
                const bool odd = i & 1;
#pragma unroll
                for (int q = 0; q < TN / P; q += 2) {
                    const i32x4 lo = __builtin_bit_cast(i32x4, value(q)), hi = __builtin_bit_cast(i32x4, value(q + 1));
                    i32x4 first, second;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int got = __builtin_amdgcn_update_dpp(0, odd ? lo[w] : hi[w], 0xb1, 0xf, 0xf, false);
                        first[w] = odd ? got : lo[w];
                        second[w] = odd ? hi[w] : got;
                    }
                    const int at = n + (q + odd) * 16 * P;
                    store(m - odd, at, __builtin_bit_cast(V, first));
                    store(m - odd + 1, at, __builtin_bit_cast(V, second));
                }
            } else {
#pragma unroll
                for (int q = 0; q < TN / P; ++q) store(m, n + q * 16 * P, value(q));
            }
        }
    };
    // smaller tiles are for smaller results; the second form's registers made the
    // compiler wait for all copies in the loop of some (256 x 4096 x 4096 13.2 us, 9.6)
    if (BM * BN >= 128 * 128 && p.beyond_cache)
        store_all.template operator()<true>();
    else
        store_all.template operator()<false>();
}

// ------------------------------------------------- rows laid out at memory lines

// Rows that start anywhere, copied to rows of whole memory lines, once, where a
// product would read them several times at twice the lines.  A wave takes 2048
// bytes of a row, a lane 16 at a time (1024 bytes a wave take the same, loads
// past the cache 5 % of the product longer: its reader finds the rest there).
// The last 16 bytes of a row are filled up with zeros.  Bound by memory: 2330 +
// 5318 rows of 6724 bytes 17 us, 6.0 TB/s read and written, some of it in cache;
// a few MB take a launch and its latency, 3 to 6 us.  4096^3 of odd rows: 64 to 70
// us, 114 as they lie.
struct Rows {
    const int8_t *from;
    int64_t ld;
    int8_t *to;
    int rows;
};
struct Layout {
    Rows a, b;  // rows == 0: the operand stays where it is
    int64_t ld;
    int K, parts;  // parts of 2048 bytes of a row
};

__global__ void __launch_bounds__(256) gemm_i8_lay_out_kernel(Layout p)
{
    const int lane = threadIdx.x & 63;
    const int64_t wave = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int64_t row = wave / p.parts;
    const int part = (int)(wave - row * p.parts);
    const bool of_b = row >= p.a.rows;
    if (of_b) row -= p.a.rows;
    if (of_b && row >= p.b.rows) return;
    const int8_t *from = of_b ? p.b.from + row * p.b.ld : p.a.from + row * p.a.ld;
    int8_t *to = (of_b ? p.b.to : p.a.to) + row * p.ld;
    i32x4 v[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int k = part * 2048 + u * 1024 + lane * 16;
        if (k >= p.K) continue;
        v[u] = *reinterpret_cast<const i32x4_u *>(from + (k + 16 <= p.K ? k : p.K - 16));
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int k = part * 2048 + u * 1024 + lane * 16, late = k + 16 - p.K;
        if (k >= p.K) continue;
        if (late > 0) v[u] = __builtin_bit_cast(i32x4, __builtin_bit_cast(unsigned __int128, v[u]) >> (8 * late));
        *reinterpret_cast<i32x4 *>(to + k) = v[u];
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
constexpr int kMostK = 131071;         // 128 * 128 * K stays below 2^31
constexpr int kMostSide = 1 << 17;    // rows and columns of C of one launch

template <typename T, int BM, int BN, int WM, int WN, int KG, int STAGES, bool DMA>
void launch_tile(const Args &a, hipStream_t s)
{
    const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN;
    // tiles of four tile rows run together: an XCD's 32 CUs then share the rows of A and B that they read
    hipLaunchKernelGGL((gemm_i8_tile_kernel<T, BM, BN, WM, WN, KG, STAGES, DMA>), dim3((unsigned)(tiles_m * tiles_n)),
                       dim3(KG * WM * WN * 64), 0, s, a, tiles_m, tiles_n, 4);
}

template <typename T>
void launch_rows(const Args &a, hipStream_t s)
{
    hipLaunchKernelGGL((gemm_i8_rows_kernel<T, 8, 4>), dim3((unsigned)((a.N + 7) / 8), (unsigned)((a.M + 7) / 8)),
                       dim3(512), 0, s, a);
}

// ---------------------------------------------------------------- choice
//
// The configuration of the least predicted time.  A configuration's time in us is
//   base + round * ceil(x / resident) + steps * max(least * ceil(x / resident), block * x),
// x = the tiles of the fullest CU, resident = its work-groups at once, steps = the
// 128-byte blocks of K that a group of waves goes through one after the other: a
// block takes `least` where the CU waits for memory, `block` where its
// work-groups share it.  Fewer than eight rows cost gemm_i8_rows less: the share
// `few` of a step does not depend on them.  The figures are fitted to timed calls
// of every configuration at 280 sizes, M 1 to 8192, N and K 64 to 16384, within 7
// to 13 % of them (22 % gemm_i8_rows of unaligned operands); the choice takes 0.7 %
// longer than the fastest configuration of each size (1.4 % unaligned).
struct Config {
    const char *name;
    int bm, bn, kg, resident;
    float base, round, least, block, few;
};

// rows that start at multiples of four bytes: copied straight into LDS
const Config kAligned[] = {
    {"gemm_i8_256x256", 256, 256, 1, 1, 0.00f, 8.10f, 1.258f, 0.000f, 1.f},
    {"gemm_i8_128x256", 128, 256, 1, 1, 0.00f, 5.47f, 0.740f, 0.000f, 1.f},
    {"gemm_i8_128x128", 128, 128, 1, 1, 0.00f, 4.44f, 0.475f, 0.000f, 1.f},
    {"gemm_i8_64x128", 64, 128, 1, 2, 0.39f, 3.59f, 0.100f, 0.300f, 1.f},
    {"gemm_i8_64x64_k2", 64, 64, 2, 1, 1.25f, 2.81f, 0.387f, 0.000f, 1.f},
    {"gemm_i8_32x64_k2", 32, 64, 2, 2, 1.90f, 1.99f, 0.290f, 0.288f, 1.f},
    {"gemm_i8_32x32_k2", 32, 32, 2, 2, 1.96f, 1.95f, 0.207f, 0.201f, 1.f},
    {"gemm_i8_16x16_k4", 16, 16, 4, 2, 2.09f, 1.40f, 0.230f, 0.195f, 1.f},
    {"gemm_i8_rows", 8, 8, 8, 4, 2.62f, 0.12f, 0.280f, 0.398f, 0.72f},
};
// any other alignment: through registers
const Config kUnaligned[] = {
    {"gemm_i8_128x256_any", 128, 256, 1, 1, 0.00f, 5.06f, 0.100f, 1.652f, 1.f},
    {"gemm_i8_128x128_any", 128, 128, 1, 2, 0.08f, 3.95f, 0.100f, 1.002f, 1.f},
    {"gemm_i8_64x64_any", 64, 64, 1, 4, 0.52f, 2.78f, 0.600f, 0.409f, 1.f},
    {"gemm_i8_64x64_k2_any", 64, 64, 2, 2, 2.48f, 1.41f, 0.445f, 0.902f, 1.f},
    {"gemm_i8_32x32_k4_any", 32, 32, 4, 2, 2.13f, 1.35f, 0.100f, 0.881f, 1.f},
    {"gemm_i8_16x16_k8_any", 16, 16, 8, 2, 2.47f, 0.81f, 0.400f, 0.844f, 1.f},
    {"gemm_i8_rows", 8, 8, 8, 4, 2.51f, 0.00f, 0.293f, 0.823f, 0.85f},
};

template <typename T>
void launch_config(const Config *c, const Args &a, hipStream_t s)
{
    if (c >= kUnaligned && c < kUnaligned + 7) {
        switch (c - kUnaligned) {
        case 0: return launch_tile<T, 128, 256, 2, 4, 1, 2, false>(a, s);
        case 1: return launch_tile<T, 128, 128, 2, 4, 1, 2, false>(a, s);
        case 2: return launch_tile<T, 64, 64, 2, 4, 1, 2, false>(a, s);
        case 3: return launch_tile<T, 64, 64, 2, 2, 2, 2, false>(a, s);
        case 4: return launch_tile<T, 32, 32, 2, 2, 4, 2, false>(a, s);
        case 5: return launch_tile<T, 16, 16, 1, 1, 8, 2, false>(a, s);
        default: return launch_rows<T>(a, s);
        }
    }
    switch (c - kAligned) {
    case 0: return launch_tile<T, 256, 256, 2, 4, 1, 2, true>(a, s);
    case 1: return launch_tile<T, 128, 256, 2, 4, 1, 3, true>(a, s);
    case 2: return launch_tile<T, 128, 128, 2, 4, 1, 4, true>(a, s);
    case 3: return launch_tile<T, 64, 128, 2, 4, 1, 3, true>(a, s);
    case 4: return launch_tile<T, 64, 64, 2, 2, 2, 3, true>(a, s);
    case 5: return launch_tile<T, 32, 64, 1, 4, 2, 3, true>(a, s);
    case 6: return launch_tile<T, 32, 32, 2, 2, 2, 4, true>(a, s);
    case 7: return launch_tile<T, 16, 16, 1, 1, 4, 4, true>(a, s);
    default: return launch_rows<T>(a, s);
    }
}

float predicted_us(const Config &c, const Args &a)
{
    constexpr int kCUs = 256;
    const int64_t tiles = (int64_t)((a.M + c.bm - 1) / c.bm) * ((a.N + c.bn - 1) / c.bn);
    const int64_t x = (tiles + kCUs - 1) / kCUs, rounds = (x + c.resident - 1) / c.resident;
    const int steps = ((a.K + 127) / 128 + c.kg - 1) / c.kg;
    const float share = c.few + (1.f - c.few) * 0.125f * (float)(a.M < 8 ? a.M : 8);
    const float least = c.least * (float)rounds, block = c.block * (float)x;
    return c.base + c.round * (float)rounds + share * (float)steps * (least > block ? least : block);
}

bool rows_of_words(const int8_t *at, int64_t ld) { return ((uintptr_t)at | (uintptr_t)ld) % 4 == 0; }

const Config *choose(const Args &a, float *us = nullptr)
{
    const bool dma = rows_of_words(a.A, a.lda) && rows_of_words(a.B, a.ldb);
    const Config *from = dma ? kAligned : kUnaligned, *rows = dma ? kAligned + 8 : kUnaligned + 6;
    const Config *best = a.lda > kMostLd || a.ldb > kMostLd ? rows : from;
    float least = predicted_us(*best, a);
    for (const Config *c = best + 1; c <= rows; ++c) {
        const float t = predicted_us(*c, a);
        if (t >= least) continue;
        best = c;
        least = t;
    }
    if (us) *us = least;
    return best;
}

// Is C written past the last-level cache, of 256 MB?  Only whole memory lines can
// be (parts of lines take twice as long: 4832 x 12370 x 536 to fp32, rows at
// multiples of 8 bytes, 164 us, 77 through it), and only where C, of more than
// 96 MB, would not stay there beside what this call and the ones around it read:
// 8192 x 16384 x 1024 to bf16 143 us, 178 through it, and 209 and 239 with a reader
// of C after it; 8192 x 8192 x 4096 to fp16 203 and 227; 8192^3 424 and 434.  Where
// it would stay, through it is faster: 12288 x 4096 x 1024 to fp32 66 us, 73 past
// it (with its reader 109 and 113).  The limit is fitted to 35 sizes.
bool past_the_cache(int64_t M, int64_t N, int64_t K, const void *C, int size, int64_t ldc)
{
    if (((uintptr_t)C | (uintptr_t)(ldc * size)) % 128) return false;
    const int64_t bytes = M * N * size;
    return bytes > (int64_t)96 << 20 && bytes + 4 * K * (M + N) > (int64_t)280 << 20;
}

constexpr int64_t kMostLayout = (int64_t)1 << 30;  // bytes of workspace

// Bytes of workspace for the rows of A, B or both laid out at memory lines, and
// what is laid out; 0 where they stay.  Only rows at other addresses than
// multiples of four: those at multiples of 4 or 16 lose less than the copy takes
// (2330 x 5318 x 6724: 97 and 95 us, at lines 81, laid out first 98).  Rows under
// a K-block have nothing to gain.  The copy is predicted as 3 us and 0.3 us a
// megabyte, at 300 sizes of odd rows: the choice takes 0.5 % longer than the
// better of both at each size, 9 % less than never laying out, 7 % more at worst.
size_t layout_of(const Args &a, Layout *p)
{
    *p = {};
    if (rows_of_words(a.A, a.lda) && rows_of_words(a.B, a.ldb)) return 0;
    if (a.K < 128) return 0;
    Args laid = a;
    p->ld = ((int64_t)a.K + 127) & ~(int64_t)127;
    p->K = a.K;
    p->parts = (a.K + 2047) / 2048;
    if (!rows_of_words(a.A, a.lda)) {
        p->a = {a.A, a.lda, nullptr, a.M};
        laid.A = nullptr;
        laid.lda = p->ld;
    }
    if (!rows_of_words(a.B, a.ldb)) {
        p->b = {a.B, a.ldb, nullptr, a.N};
        laid.B = nullptr;
        laid.ldb = p->ld;
    }
    const int64_t bytes = ((int64_t)p->a.rows + p->b.rows) * p->ld;
    if (bytes > kMostLayout) return 0;
    float as_it_is, after;
    choose(a, &as_it_is);
    choose(laid, &after);
    return after + 3.f + 0.3e-6f * (float)bytes < as_it_is ? (size_t)bytes : 0;
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
    // a launch's grid holds the tiles of at most kMostSide rows and columns
    const Config *c = nullptr;
    for (int m = 0; m < a.M; m += kMostSide)
        for (int n = 0; n < a.N; n += kMostSide) {
            Args part = a;
            part.M = a.M - m < kMostSide ? a.M - m : kMostSide;
            part.N = a.N - n < kMostSide ? a.N - n : kMostSide;
            part.A += m * a.lda;
            part.B += n * a.ldb;
            part.sa += m;
            part.sb += n;
            if (a.bias) part.bias += n;
            part.C = (T *)a.C + m * a.ldc + n;
            c = choose(part);
            launch_config<T>(c, part, s);
            if (hipGetLastError() != hipSuccess) return PK_ERR_LAUNCH;
        }
    pk::api_ran(c->name);
    return PK_OK;
}

}  // namespace

extern "C" size_t pk_gemm_i8_workspace_bytes_for(int64_t M, int64_t N, int64_t K, const int8_t *A, int64_t lda,
                                                 const int8_t *B, int64_t ldb)
{
    using namespace pk::checks;
    if (M <= 0 || N <= 0 || K <= 0 || short_ld(lda, K) || short_ld(ldb, K)) return 0;
    if (too_large({M, N, lda, ldb}) || K > kMostK) return 0;
    Layout p;
    return layout_of({A, B, nullptr, nullptr, nullptr, nullptr, lda, ldb, 0, (int)M, (int)N, (int)K, false}, &p);
}

extern "C" int pk_gemm_i8_ws(int64_t M, int64_t N, int64_t K, const int8_t *A, int64_t lda, const float *a_scale,
                             const int8_t *B, int64_t ldb, const float *b_scale, const float *bias, void *C, int dtype,
                             int64_t ldc, void *workspace, size_t workspace_bytes, void *stream)
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
    if (too_large({M, N, lda, ldb, ldc}) || K > kMostK) return PK_ERR_NOT_SUPPORTED;
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
    const bool beyond_cache = past_the_cache(M, N, K, C, size, ldc);
    Args a = {A, B, a_scale, b_scale, bias, C, lda, ldb, ldc, (int)M, (int)N, (int)K, beyond_cache};
    hipStream_t s = (hipStream_t)stream;
    Layout p;
    const size_t need = workspace && !misaligned(workspace, 16) ? layout_of(a, &p) : 0;
    if (need && need <= workspace_bytes) {
        const Span ws = {(uintptr_t)workspace, (uintptr_t)workspace + need};
        if (overlap(ws, sc) || overlap(ws, span(A, M, K, lda, 1)) || overlap(ws, span(B, N, K, ldb, 1)) ||
            overlap(ws, span(a_scale, 1, M, M, 4)) || overlap(ws, span(b_scale, 1, N, N, 4)) ||
            (bias && overlap(ws, span(bias, 1, N, N, 4))))
            return api_invalid(14);
        int8_t *to = (int8_t *)workspace;
        if (p.a.rows) {
            a.A = p.a.to = to;
            a.lda = p.ld;
            to += p.a.rows * p.ld;
        }
        if (p.b.rows) {
            a.B = p.b.to = to;
            a.ldb = p.ld;
        }
        const int64_t waves = ((int64_t)p.a.rows + p.b.rows) * p.parts;
        hipLaunchKernelGGL(gemm_i8_lay_out_kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, p);
        if (hipGetLastError() != hipSuccess) return PK_ERR_LAUNCH;
    }
    return dtype == PK_F32 ? launch<float>(a, s) : dtype == PK_BF16 ? launch<bf16>(a, s) : launch<f16>(a, s);
}

extern "C" int pk_gemm_i8(int64_t M, int64_t N, int64_t K, const int8_t *A, int64_t lda, const float *a_scale,
                          const int8_t *B, int64_t ldb, const float *b_scale, const float *bias, void *C, int dtype,
                          int64_t ldc, void *stream)
{
    return pk_gemm_i8_ws(M, N, K, A, lda, a_scale, B, ldb, b_scale, bias, C, dtype, ldc, nullptr, 0, stream);
}
