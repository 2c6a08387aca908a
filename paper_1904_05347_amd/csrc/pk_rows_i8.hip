// pk_rows_i8.hip -- rows of a matrix to 8-bit integers with one scale a row,
// alone or as the end of the operator that makes the row, and back.
//
// Row z becomes q = rint(z * (127 * (1 / a))) and scale = a / 127 with a = max |z|.
// What z is:
//   PLAIN   the input;
//   NORM    h * w, h = x (+ residual, rounded to its type: what is stored), and
//           the scale takes the norm's 1 / sqrt(mean h^2 + eps): a factor common
//           to the row cancels in q, so both reductions (sum of squares, largest
//           magnitude) are made in one pass over the data;
//   GATED   act(gate) * up.
// The row's values stay in registers between the reduction and the rounding, so
// every input is read once and every output written once; a row too long for
// that has what is beyond read (and computed) twice.  Bound by memory: the norm of
// 8192 x 4096 bf16 with a residual moves 235 MB in 39 us (6.0 TB/s; a plain copy
// reaches 5.0), the gated activation of 8192 x 8192 336 MB in 54 us, fp32 rows of
// that 336 MB in 57 us; a few rows by the latency of a launch and of memory (one
// row of 4096: 2.6 us).  Gated rows that the registers do not hold are computed
// twice: 2048 x 53248 bf16, 545 MB in 141 us (3.9 TB/s).
#include "pk_i8.hpp"
#include "pk_i8_checks.hpp"
#include "pk_rows_i8_launch.hpp"

#pragma clang fp contract(off)  // z times that factor is rounded before it is rounded to an integer

namespace {

using pk::bf16;
using pk::f16;
using pk::kMostRows;
using pk::Pack;
using pk::rounded;
using pk::rows_group;
using pk::rows_groups;

enum { PLAIN, NORM, GATED };

struct RowArgs {
    const void *x, *y;  // the input (gate); the residual (up), or NULL
    const void *w;      // NORM: the weight
    void *sum;          // NORM: x + residual, or NULL
    int8_t *q;
    float *scale;
    int64_t ldx, ldy, lds, ldq;
    int M, N, act;
    float eps;
};

// act(g) = g q / (1 + q): q = exp(g) (silu) or exp of twice the argument of gelu's
// tanh, 2 sqrt(2 / pi) (g + 0.044715 g^3): 1 / 2 (1 + tanh u) is
// exp(2 u) / (1 + exp(2 u)).  q is made as h^2, h = 2^s, and the factors are
// multiplied one by one, so that nothing before the result leaves the 32 bits'
// range: the activation falls to the least subnormal as its formula does.  Where
// q / (1 + q) is 1, q is held at a power of two, so that the factors change no bit
// of g: 2^60, and 2^28 (silu: at 28 ln(2) s is 14 and nothing is left).  The
// exponential and the reciprocal are the hardware's, within a unit in the last
// place each.
//   silu: s = g log2(e) / 2 is rounded, by up to |s| / 2 units of exp's result
// (65 half units of the activation at -83); what the rounding left out goes into
// one of the factors, exp(g - 2 ln(2) s) = 1 + that (6 half units of the activation).
//   gelu: the polynomial's own rounding is of that size and stays: fp32 has the
// cube to three roundings, whatever is done with it.
template <int ACT>
__device__ __forceinline__ float activate(float g)
{
    if constexpr (ACT == PK_ACT_SILU) {
        const float most = fminf(g, 0x1.3687aap+4f), s = 0.72134752f * most;
        // 2 ln(2) in two parts, the first rounded to fp32
        constexpr double two_ln2 = 1.3862943611198906;
        constexpr float hi = (float)two_ln2, lo = (float)(two_ln2 - (double)hi);
        const float left = fmaf(s, -lo, fmaf(s, -hi, most));
        const float h = __builtin_amdgcn_exp2f(s), k = fmaf(h, left, h);
        return g * __builtin_amdgcn_rcpf(fmaf(h, k, 1.f)) * h * k;
    } else {
        // log2(e) / 2 is in the constants
        constexpr float c = 0.5f * 1.5957691216057308f * 1.4426950408889634f;
        const float h = __builtin_amdgcn_exp2f(fminf(g * fmaf(0.044715f * c, g * g, c), 30.f));
        return g * __builtin_amdgcn_rcpf(fmaf(h, h, 1.f)) * h * h;
    }
}

// v of every lane combined by op, in every lane; `none` leaves v as it is.
template <typename Op>
__device__ __forceinline__ int across_wave(int v, int none, Op op)
{
    v = op(v, __builtin_amdgcn_update_dpp(none, v, 0xb1, 0xf, 0xf, false));   // lane ^ 1
    v = op(v, __builtin_amdgcn_update_dpp(none, v, 0x4e, 0xf, 0xf, false));   // lane ^ 2
    v = op(v, __builtin_amdgcn_update_dpp(none, v, 0x141, 0xf, 0xf, false));  // mirrored in 8
    v = op(v, __builtin_amdgcn_update_dpp(none, v, 0x140, 0xf, 0xf, false));  // mirrored in 16
    v = op(v, __builtin_amdgcn_update_dpp(none, v, 0x142, 0xa, 0xf, false));  // lane 15 and 47 to the next 16
    v = op(v, __builtin_amdgcn_update_dpp(none, v, 0x143, 0xc, 0xf, false));  // lane 31 to the upper half
    return __builtin_amdgcn_readlane(v, 63);
}

// What one work-item reads of E neighbouring elements.
template <typename T, typename W, int MODE>
struct Chunk {
    static constexpr int E = 16 / (int)sizeof(T);
    typedef typename Pack<T>::U U;
    typedef typename Pack<W, E>::U UW;
    typename Pack<T>::V x, y;
    typename Pack<W, E>::V w;

    // elements e .. e + E - 1 of the row; those at N and beyond are 0
    __device__ __forceinline__ void load(const T *px, const T *py, const W *pw, int e, int N)
    {
        if (e + E <= N) {
            // read once: the caches keep what is written here for the reader of it
            // (8192 x 8192 fp32 to 8 bits and back: 105.9 us, 141.7 without)
            x = __builtin_nontemporal_load(reinterpret_cast<const U *>(px + e));
            if (MODE == GATED || (MODE == NORM && py)) y = __builtin_nontemporal_load(reinterpret_cast<const U *>(py + e));
            if (MODE == NORM) w = *reinterpret_cast<const UW *>(pw + e);
            return;
        }
        x = y = (typename Pack<T>::V)(T)0.f;
        w = (typename Pack<W, E>::V)(W)0.f;
        if (e >= N) return;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const bool in = e + j < N;
            x[j] = in ? px[e + j] : (T)0.f;
            if (MODE == GATED || (MODE == NORM && py)) y[j] = in ? py[e + j] : (T)0.f;
            if (MODE == NORM) w[j] = in ? pw[e + j] : (W)0.f;
        }
    }
    // z of these elements; NORM: h replaces x
    __device__ __forceinline__ void values(bool added, int act, float *z)
    {
        if (MODE == GATED && act == PK_ACT_SILU) {
#pragma unroll
            for (int j = 0; j < E; ++j) z[j] = activate<PK_ACT_SILU>((float)x[j]) * (float)y[j];
        } else if (MODE == GATED) {
#pragma unroll
            for (int j = 0; j < E; ++j) z[j] = activate<PK_ACT_GELU>((float)x[j]) * (float)y[j];
        }
#pragma unroll
        for (int j = 0; j < E; ++j) {
            if (MODE == PLAIN) z[j] = (float)x[j];
            if (MODE == NORM) {
                if (added) x[j] = (T)((float)x[j] + (float)y[j]);
                z[j] = (float)x[j] * (float)w[j];
            }
        }
    }
};

template <typename T>
__device__ __forceinline__ void put(T *p, int e, int N, const typename Pack<T>::V &v)
{
    constexpr int E = 16 / (int)sizeof(T);
    if (e + E <= N) {
        *reinterpret_cast<typename Pack<T>::U *>(p + e) = v;
        return;
    }
#pragma unroll
    for (int j = 0; j < E; ++j)
        if (e + j < N) p[e + j] = v[j];
}

// Magnitudes as integers: ordered as the floats are, infinity above every
// number and NaN above infinity, so a NaN is not lost in the maximum.
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// q as the lowest byte of z * inv + 1.5 2^23, whose units are integers: the
// addition rounds to the nearest, ties to even.
template <int E>
__device__ __forceinline__ void quantized(int8_t *q, int e, int N, const float *z, float inv)
{
    typename Pack<int8_t, E>::V v = (typename Pack<int8_t, E>::V)(int8_t)0;
    if (inv != 0.f) {
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = (int8_t)__float_as_uint(z[j] * inv + 0x1.8p23f);
    }
    if (e + E <= N) {
        *reinterpret_cast<typename Pack<int8_t, E>::U *>(q + e) = v;
        return;
    }
#pragma unroll
    for (int j = 0; j < E; ++j)
        if (e + j < N) q[e + j] = v[j];
}

// TPR work-items a row, VPT 16-byte chunks of it in each one's registers.
template <typename T, typename W, int MODE, int TPR, int VPT>
__global__ void __launch_bounds__(rows_group(TPR)) rows_i8_kernel(RowArgs p)
{
    constexpr int E = 16 / (int)sizeof(T), WAVES = TPR / 64, STEP = TPR * E;
    const int t = threadIdx.x % TPR;
    // NORM: the same in a wave, as the compiler cannot see; addresses in scalar
    // registers leave more of the others (16384 x 2048 fp16 39.1 us, 40.7).  GATED
    // then has fewer loads in flight (16384 x 1000 bf16 20.4 us, 17.1).
    const int of_group = threadIdx.x / TPR;
    const int64_t row = (int64_t)blockIdx.x * (rows_group(TPR) / TPR) +
                        (MODE == NORM ? __builtin_amdgcn_readfirstlane(of_group) : of_group);
    if (row >= p.M) return;  // TPR < 256: whole waves, and no barrier below
    const T *px = (const T *)p.x + row * p.ldx;
    const T *py = p.y ? (const T *)p.y + row * p.ldy : nullptr;
    const W *pw = (const W *)p.w;
    T *ps = MODE == NORM && p.sum ? (T *)p.sum + row * p.lds : nullptr;
    int8_t *pq = p.q + row * p.ldq;
    const int N = p.N;

    Chunk<T, W, MODE> c[VPT];
    float z[VPT][E], ss = 0.f;
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) c[i].load(px, py, pw, i * STEP + t * E, N);
    auto reduce = [&](const Chunk<T, W, MODE> &k, const float *v) {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            if (MODE == NORM) ss = fmaf((float)k.x[j], (float)k.x[j], ss);
            most = __builtin_elementwise_maximum(most, fabsf(v[j]));  // keeps a NaN
        }
    };
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        c[i].values(py != nullptr, p.act, z[i]);
        if (ps) put(ps, i * STEP + t * E, N, c[i].x);
        reduce(c[i], z[i]);
    }
    for (int e = VPT * STEP + t * E; e < N; e += STEP) {
        Chunk<T, W, MODE> k;
        float v[E];
        k.load(px, py, pw, e, N);
        k.values(py != nullptr, p.act, v);
        if (ps) put(ps, e, N, k.x);
        reduce(k, v);
    }

    // v of the row's work-items added, in each of them
    auto total = [&](float v) {
        v = __int_as_float(across_wave(__float_as_int(v), 0, [](int a, int b) {
            return __float_as_int(__int_as_float(a) + __int_as_float(b));
        }));
        if constexpr (TPR > 64) {
            __shared__ float s_v[WAVES];
            if (t % 64 == 0) s_v[t / 64] = v;
            __syncthreads();
            v = s_v[0];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) v += s_v[i];
        }
        return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
    };
    unsigned am = (unsigned)across_wave((int)magnitude(most), 0, [](int a, int b) { return (int)max((unsigned)a, (unsigned)b); });
    __shared__ unsigned s_am[WAVES];
    if (TPR > 64 && t % 64 == 0) s_am[t / 64] = am;
    if constexpr (MODE == NORM)
        ss = total(ss);  // its barrier is s_am's as well
    else if constexpr (TPR > 64)
        __syncthreads();
    if constexpr (TPR > 64) {
        am = s_am[0];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) am = max(am, s_am[i]);
    }

    // A row whose scale would fall below the normal numbers is a row of zeros;
    // one that holds an infinity or a NaN keeps it in its scale, so that it
    // reads back as NaN.
    am = __builtin_amdgcn_readfirstlane(am);
    const float a = __uint_as_float(am);
    const bool live = a >= 127.f * 0x1p-126f && a < __builtin_inff();
    const float inv = live ? 127.f * (1.f / a) : 0.f;
    // NORM: squares that leave the 32 bits' range below, where eps does not cover them
    const bool small = MODE == NORM && live && ss < 0x1p-80f && p.eps < 0x1p-100f;
    if (t == 0 && !small) {
        float s = a;
        if (live && MODE == NORM) s = a * (1.f / sqrtf(ss / (float)N + p.eps));
        if (am > 0x7f800000u) s = __uint_as_float(0x7fc00000u);
        p.scale[row] = live ? s / 127.f : am < 0x7f800000u ? 0.f : s;
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) quantized<E>(pq, i * STEP + t * E, N, z[i], inv);
    for (int e = VPT * STEP + t * E; e < N; e += STEP) {
        Chunk<T, W, MODE> k;
        float v[E];
        k.load(ps ? ps : px, ps ? nullptr : py, pw, e, N);  // ps may be the memory of px or py
        k.values(!ps && py, p.act, v);
        quantized<E>(pq, e, N, v, inv);
    }
    if constexpr (MODE == NORM) {
        if (!small) return;
        // They are added once more, of h times 2^100: of the least h, 2^-149, that is
        // 2^-98, and the sum stays below 2^120.  Here, where no value of the row is
        // held any more: further up it took registers from every call (fp32 4096 x
        // 12000 115 us, 100).
        constexpr float UP = 0x1p100f;
        ss = 0.f;
        for (int e = t * E; e < N; e += STEP) {
            Chunk<T, W, MODE> k;
            float v[E];
            k.load(ps ? ps : px, ps ? nullptr : py, pw, e, N);
            k.values(!ps && py, p.act, v);
#pragma unroll
            for (int j = 0; j < E; ++j) ss = fmaf((float)k.x[j] * UP, (float)k.x[j] * UP, ss);
        }
        if constexpr (TPR > 64) __syncthreads();  // the first sum has been read
        ss = total(ss);
        const float root = 1.f / sqrtf(ss / (float)N + p.eps * UP * UP);
        // the factors in the order that stays in range where the result does
        if (t == 0) p.scale[row] = (a < 1.f ? a * UP * root : a * root * UP) / 127.f;
    }
}

// x = q * scale: one team of TPR work-items a row, blockIdx.y cuts long rows.
// Bound by memory: 8192 x 8192 to bf16 201 MB in 30 us, the 8-bit values from the
// last-level cache where they were just written.
template <typename T, int TPR>
__global__ void __launch_bounds__(256) dequantize_i8_kernel(const int8_t *q, int64_t ldq, const float *scale, T *x,
                                                            int64_t ldx, int M, int N, int span)
{
    constexpr int E = 16 / (int)sizeof(T);
    const int64_t row = (int64_t)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    if (row >= M) return;
    const int8_t *pq = q + row * ldq;
    T *px = x + row * ldx;
    const float s = scale[row];
    const int e0 = blockIdx.y * span, e1 = N - e0 < span ? N : e0 + span;
#pragma unroll 4
    for (int e = e0 + (threadIdx.x % TPR) * E; e < e1; e += TPR * E) {
        typename Pack<T>::V v;
        if (e + E <= N) {
            const typename Pack<int8_t, E>::V b = *reinterpret_cast<const typename Pack<int8_t, E>::U *>(pq + e);
#pragma unroll
            for (int j = 0; j < E; ++j) v[j] = rounded<T>((float)b[j] * s);
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) v[j] = e + j < N ? rounded<T>((float)pq[e + j] * s) : (T)0.f;
        }
        put(px, e, N, v);
    }
}

// ---------------------------------------------------------------- launches

template <typename T, typename W, int MODE>
int launch_rows(const RowArgs &a, hipStream_t s)
{
    constexpr int E = 16 / (int)sizeof(T);
    const int chunks = (a.N + E - 1) / E;
#define PK_ROWS(TPR, VPT)                                                                                           \
    hipLaunchKernelGGL((rows_i8_kernel<T, W, MODE, TPR, VPT>), dim3((unsigned)rows_groups(a.M, TPR)),                  \
                       dim3(rows_group(TPR)), 0, s, a)
    // The fewest registers that hold a row.  Many rows: the fewest work-items that
    // do, a wave for a short row (bf16 norm, 16384 x 2048: one wave 39.5 us, four
    // 41.7; 8192 x 4096: four waves 39.0, eight 40.9), until the values of a row
    // leave too few of them on a CU (8192 x 8192 gated: eight waves 64.1, four
    // 67.2; fp32 rows of it: sixteen waves 57.6, four 66.0).  Few rows: more
    // work-items, for the latency (1024 x 4096: eight waves 8.5 us, four 8.9).
    const bool few = a.M <= 1024;
    if (chunks <= 64)
        PK_ROWS(64, 1);
    else if (chunks <= 128)
        PK_ROWS(64, 2);
    else if (chunks <= 256 && few)
        PK_ROWS(256, 1);
    else if (chunks <= 256)
        PK_ROWS(64, 4);
    else if (chunks <= 512 && few)
        PK_ROWS(512, 1);
    else if (chunks <= 512)
        PK_ROWS(256, 2);
    else if (chunks <= 1024)
        PK_ROWS(512, 2);
    else if (chunks <= 1536)
        PK_ROWS(512, 3);
    else if (chunks <= 2048)
        PK_ROWS(1024, 2);
    else
        PK_ROWS(1024, 4);
#undef PK_ROWS
    return hipGetLastError() == hipSuccess ? PK_OK : PK_ERR_LAUNCH;
}

template <int MODE>
int launch_rows(int dtype, int wtype, RowArgs a, int64_t M, hipStream_t s)
{
    const int64_t size = pk::dtype_size(dtype);
    for (; M > kMostRows; M -= kMostRows) {
        a.M = (int)kMostRows;
        const int st = launch_rows<MODE>(dtype, wtype, a, kMostRows, s);
        if (st != PK_OK) return st;
        a.x = (const char *)a.x + kMostRows * a.ldx * size;
        if (a.y) a.y = (const char *)a.y + kMostRows * a.ldy * size;
        if (a.sum) a.sum = (char *)a.sum + kMostRows * a.lds * size;
        a.q += kMostRows * a.ldq;
        a.scale += kMostRows;
    }
    a.M = (int)M;
    if (dtype == PK_F32) return launch_rows<float, float, MODE>(a, s);
    if constexpr (MODE == NORM) {
        if (wtype == PK_F32)
            return dtype == PK_BF16 ? launch_rows<bf16, float, MODE>(a, s) : launch_rows<f16, float, MODE>(a, s);
    }
    return dtype == PK_BF16 ? launch_rows<bf16, bf16, MODE>(a, s) : launch_rows<f16, f16, MODE>(a, s);
}

template <typename T>
int launch_dequantize(const int8_t *q, int64_t ldq, const float *scale, void *x, int64_t ldx, int64_t rows, int N,
                      hipStream_t s)
{
    constexpr int E = 16 / (int)sizeof(T);
    if (rows > kMostRows) {
        for (int64_t r = 0; r < rows; r += kMostRows) {
            const int st = launch_dequantize<T>(q + r * ldq, ldq, scale + r, (T *)x + r * ldx, ldx,
                                                rows - r < kMostRows ? rows - r : kMostRows, N, s);
            if (st != PK_OK) return st;
        }
        return PK_OK;
    }
    const int M = (int)rows;
    if (N <= 64 * E) {
        hipLaunchKernelGGL((dequantize_i8_kernel<T, 64>), dim3((unsigned)rows_groups(M, 64)), dim3(256), 0, s, q, ldq,
                           scale, (T *)x, ldx, M, N, N);
    } else {
        // a work-item's share is four chunks, so that their loads are in flight
        // together (more where the grid's second dimension would not hold them)
        constexpr int SHARE = 4 * 256 * E;
        const int span = (N / SHARE / 32768 + 1) * SHARE;
        hipLaunchKernelGGL((dequantize_i8_kernel<T, 256>),
                           dim3((unsigned)rows_groups(M, 256), (unsigned)((N - 1) / span + 1)), dim3(256), 0, s, q, ldq,
                           scale, (T *)x, ldx, M, N, span);
    }
    return hipGetLastError() == hipSuccess ? PK_OK : PK_ERR_LAUNCH;
}

}  // namespace

extern "C" {

int pk_quantize_i8(const void *x, int dtype, int64_t M, int64_t N, int64_t ldx, int8_t *q, int64_t ldq, float *scale,
                   void *stream)
{
    using namespace pk;
    using namespace pk::checks;
    api_begin();
    const int size = dtype_size(dtype);
    if (!size) return api_invalid(2);
    if (M < 0) return api_invalid(3);
    if (N < 0) return api_invalid(4);
    if (short_ld(ldx, N)) return api_invalid(5);
    if (short_ld(ldq, N)) return api_invalid(7);
    if (M == 0) return PK_OK;
    if (too_large({M, N, ldx, ldq})) return PK_ERR_NOT_SUPPORTED;
    if ((!x && N) || misaligned(x, size)) return api_invalid(1);
    if (!q && N) return api_invalid(6);
    if (!scale || misaligned(scale, 4)) return api_invalid(8);
    const Span sx = span(x, M, N, ldx, size), sq = span(q, M, N, ldq, 1), ss = span(scale, 1, M, M, 4);
    if (N && overlap(sq, sx)) return api_invalid(6);
    if (N && (overlap(ss, sx) || overlap(ss, sq))) return api_invalid(8);
    const RowArgs a = {x, nullptr, nullptr, nullptr, q, scale, ldx, 0, 0, ldq, 0, (int)N, 0, 0.f};
    const int st = launch_rows<PLAIN>(dtype, 0, a, M, (hipStream_t)stream);
    if (st == PK_OK) api_ran("quantize_i8");
    return st;
}

int pk_rmsnorm_i8(const void *x, int dtype, int64_t M, int64_t N, int64_t ldx, const void *residual, int64_t ldr,
                  const void *weight, int weight_dtype, float eps, void *sum, int64_t lds, int8_t *q, int64_t ldq,
                  float *scale, void *stream)
{
    using namespace pk;
    using namespace pk::checks;
    api_begin();
    const int size = dtype_size(dtype), wsize = dtype_size(weight_dtype);
    if (!size) return api_invalid(2);
    if (M < 0) return api_invalid(3);
    if (N < 0) return api_invalid(4);
    if (short_ld(ldx, N)) return api_invalid(5);
    if (residual && short_ld(ldr, N)) return api_invalid(7);
    if (weight_dtype != PK_F32 && weight_dtype != dtype) return api_invalid(9);
    if (!(eps >= 0.f)) return api_invalid(10);
    if (sum && !residual) return api_invalid(11);
    if (sum && short_ld(lds, N)) return api_invalid(12);
    if (short_ld(ldq, N)) return api_invalid(14);
    if (M == 0) return PK_OK;
    if (too_large({M, N, ldx, residual ? ldr : 0, sum ? lds : 0, ldq})) return PK_ERR_NOT_SUPPORTED;
    if ((!x && N) || misaligned(x, size)) return api_invalid(1);
    if (misaligned(residual, size)) return api_invalid(6);
    if ((!weight && N) || misaligned(weight, wsize)) return api_invalid(8);
    if (misaligned(sum, size)) return api_invalid(11);
    if (!q && N) return api_invalid(13);
    if (!scale || misaligned(scale, 4)) return api_invalid(15);
    if (N) {
        const Span sx = span(x, M, N, ldx, size), sr = residual ? span(residual, M, N, ldr, size) : sx,
                   sw = span(weight, 1, N, N, wsize), sq = span(q, M, N, ldq, 1), ss = span(scale, 1, M, M, 4);
        if (sum) {
            // the sum may be written over either of its terms, element for element
            const Span sh = span(sum, M, N, lds, size);
            if (overlap(sh, sx) && !(sum == x && lds == ldx)) return api_invalid(11);
            if (overlap(sh, sr) && !(sum == residual && lds == ldr)) return api_invalid(11);
            if (overlap(sh, sw)) return api_invalid(11);
            if (overlap(sq, sh)) return api_invalid(13);
            if (overlap(ss, sh)) return api_invalid(15);
        }
        if (overlap(sq, sx) || overlap(sq, sr) || overlap(sq, sw)) return api_invalid(13);
        if (overlap(ss, sx) || overlap(ss, sr) || overlap(ss, sw) || overlap(ss, sq)) return api_invalid(15);
    }
    const RowArgs a = {x, residual, weight, sum, q, scale, ldx, ldr, lds, ldq, 0, (int)N, 0, eps};
    const int st = launch_rows<NORM>(dtype, weight_dtype, a, M, (hipStream_t)stream);
    if (st == PK_OK) api_ran("rmsnorm_i8");
    return st;
}

int pk_gated_i8(const void *gate, int64_t ldg, const void *up, int64_t ldu, int dtype, int act, int64_t M, int64_t N,
                int8_t *q, int64_t ldq, float *scale, void *stream)
{
    using namespace pk;
    using namespace pk::checks;
    api_begin();
    const int size = dtype_size(dtype);
    if (!size) return api_invalid(5);
    if (act != PK_ACT_SILU && act != PK_ACT_GELU) return api_invalid(6);
    if (M < 0) return api_invalid(7);
    if (N < 0) return api_invalid(8);
    if (short_ld(ldg, N)) return api_invalid(2);
    if (short_ld(ldu, N)) return api_invalid(4);
    if (short_ld(ldq, N)) return api_invalid(10);
    if (M == 0) return PK_OK;
    if (too_large({M, N, ldg, ldu, ldq})) return PK_ERR_NOT_SUPPORTED;
    if ((!gate && N) || misaligned(gate, size)) return api_invalid(1);
    if ((!up && N) || misaligned(up, size)) return api_invalid(3);
    if (!q && N) return api_invalid(9);
    if (!scale || misaligned(scale, 4)) return api_invalid(11);
    if (N) {
        const Span sg = span(gate, M, N, ldg, size), su = span(up, M, N, ldu, size), sq = span(q, M, N, ldq, 1),
                   ss = span(scale, 1, M, M, 4);
        if (overlap(sq, sg) || overlap(sq, su)) return api_invalid(9);
        if (overlap(ss, sg) || overlap(ss, su) || overlap(ss, sq)) return api_invalid(11);
    }
    const RowArgs a = {gate, up, nullptr, nullptr, q, scale, ldg, ldu, 0, ldq, 0, (int)N, act, 0.f};
    const int st = launch_rows<GATED>(dtype, 0, a, M, (hipStream_t)stream);
    if (st == PK_OK) api_ran("gated_i8");
    return st;
}

int pk_dequantize_i8(const int8_t *q, int64_t ldq, const float *scale, int64_t M, int64_t N, void *x, int dtype,
                     int64_t ldx, void *stream)
{
    using namespace pk;
    using namespace pk::checks;
    api_begin();
    const int size = dtype_size(dtype);
    if (M < 0) return api_invalid(4);
    if (N < 0) return api_invalid(5);
    if (!size) return api_invalid(7);
    if (short_ld(ldq, N)) return api_invalid(2);
    if (short_ld(ldx, N)) return api_invalid(8);
    if (M == 0 || N == 0) return PK_OK;
    if (too_large({M, N, ldq, ldx})) return PK_ERR_NOT_SUPPORTED;
    if (!q) return api_invalid(1);
    if (!scale || misaligned(scale, 4)) return api_invalid(3);
    if (!x || misaligned(x, size)) return api_invalid(6);
    const Span sx = span(x, M, N, ldx, size);
    if (overlap(sx, span(q, M, N, ldq, 1)) || overlap(sx, span(scale, 1, M, M, 4))) return api_invalid(6);
    hipStream_t s = (hipStream_t)stream;
    const int st = dtype == PK_F32    ? launch_dequantize<float>(q, ldq, scale, x, ldx, M, (int)N, s)
                   : dtype == PK_BF16 ? launch_dequantize<bf16>(q, ldq, scale, x, ldx, M, (int)N, s)
                                      : launch_dequantize<f16>(q, ldq, scale, x, ldx, M, (int)N, s);
    if (st == PK_OK) api_ran("dequantize_i8");
    return st;
}

}  // extern "C"
