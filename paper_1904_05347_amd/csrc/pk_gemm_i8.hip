// pk_gemm_i8.hip -- products of 8-bit integers with a scale for each row of
// either operand: C[m][n] = sa[m] sb[n] sum_k A[m][k] B[n][k] + bias[n].
#include "pk_i8.hpp"
#include "pk_i8_checks.hpp"

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
