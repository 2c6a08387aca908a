// pk_attention.hip -- attention of drafted tokens over a paged cache.
//
//   o_i = sum_j p_ij v_j,  p_i the softmax over the j that row i sees of
//   x_ij = c tanh(scale (q_i . k_j) / c)   (scale (q_i . k_j) without a cap c).
//
// One pass over the cache: each wave takes 32 positions at a time and keeps, for
// each of its rows, the largest x so far, the sum of exponentials and the sum of
// values weighted by them.  All rows that read one head of the cache (its tokens
// times the query heads that share it) are columns of one product, so that K and V
// are read once for them.
//
// Lanes.  x^T = K q^T and o^T = V^T p^T on the 16 x 16 matrix instruction, whose
// operands hold 8 neighbours along the sum a lane: K's and q's rows are read as
// they lie, 16 bytes a lane.  In x^T a lane has one row's (lane % 16) x of four
// neighbouring positions, from two products of eight: the second product's operand,
// without any exchange, where V^T takes its positions in the same order.  V^T comes
// out of LDS transposed.
#include "pk_attention_plan.hpp"
#include "pk_heads_checks.hpp"
#include "pk_i8.hpp"
#include "pk_i8_checks.hpp"

namespace {

using namespace pk::attention;
using pk::bf16;
using pk::f16;
using pk::Pack;
using pk::rounded;

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;       // of a work-group
constexpr int kTile = 32;       // positions that a wave has in work
constexpr int kUnit = kWaves * kTile;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;

struct Args {
    const void *q;
    void *out;
    const void *key, *value;
    const int32_t *table, *lengths, *starts;
    const uint64_t *mask;
    float *lse, *parts;
    int64_t q_token, q_head, out_token, out_head, lse_token, table_row;
    int64_t key_page, key_place, key_head, value_page, value_place, value_head;
    int64_t pages;
    Shape shape;
    int B, d, page_size, page_shift;  // page_shift: of a power of two, else -1
    float scale, cap;  // scores are formed in powers of two: scale * log2(e), or scale / cap and cap * log2(e)
};

template <typename T>
struct Eight {
    typedef T V __attribute__((ext_vector_type(8)));
};

// Eight elements from p on, those from n on zero.
template <typename T>
__device__ __forceinline__ typename Eight<T>::V get8(const T *p, int n)
{
    typedef typename Eight<T>::V V;
    V v = (V)(T)0.f;
    if (n >= 8) {
        typedef V U __attribute__((aligned(sizeof(T))));
        return *reinterpret_cast<const U *>(p);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) v[j] = p[j];
    return v;
}

// c += a b^T for 16 x 32 operands: lane l holds row l % 16, elements 8 (l / 16) on.
__device__ __forceinline__ f32x4 product(Eight<bf16>::V a, Eight<bf16>::V b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 product(Eight<f16>::V a, Eight<f16>::V b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
// fp32 has products of 4: eight of them, one for each element of the lanes
__device__ __forceinline__ f32x4 product(Eight<float>::V a, Eight<float>::V b, f32x4 c)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
}

// A wave's 32 rows of V in LDS.  Rows are padded so that the lanes of one read of a
// column tile start at different banks: 8 apart in 16 bits, 4 in 32.
template <typename T, int D>
struct Staged {
    static constexpr int kPad = sizeof(T) == 2 ? 16 : 4;
    static constexpr int kRow = D + kPad;
    static constexpr int kBytes = kTile * kRow * (int)sizeof(T);

    // channels 16 n + lane % 16 of positions 4 (lane / 16) + 0..3 and those + 16
    static __device__ __forceinline__ typename Eight<T>::V column(const T *s, int n, int lane)
    {
        typename Eight<T>::V v;
        if constexpr (sizeof(T) == 2) {
            typedef short S4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) S4 *P;
            const T *p = s + (lane / 4) * kRow + n * 16 + (lane % 4) * 4;
            const S4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)p);
            const S4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p + 16 * kRow));
            const auto both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            v = __builtin_bit_cast(typename Eight<T>::V, both);
        } else {
            const T *p = s + (lane / 16) * 4 * kRow + n * 16 + lane % 16;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = p[j * kRow];
                v[4 + j] = p[(16 + j) * kRow];
            }
        }
        return v;
    }
};

// tanh, to 2 units in the last place.  The exponential's form would lose digits
// below 0.6: there x (1 + x^2 P(x^2)), P a least-squares fit whose error is 2^-30 of
// the result.
__device__ __forceinline__ float tanh_of(float x)
{
    const float y = fabsf(x), z = x * x;
    float p = fmaf(z, 0.00231141f, -0.00836057f);
    p = fmaf(z, p, 0.02177406f);
    p = fmaf(z, p, -0.0539599f);
    p = fmaf(z, p, 0.13333306f);
    p = fmaf(z, p, -0.33333333f);
    const float e = __builtin_amdgcn_exp2f(y * (2.f * kLog2e));  // infinite far out: 1 - 0
    const float far = copysignf(1.f - 2.f * __builtin_amdgcn_rcpf(1.f + e), x);
    return y < 0.6f ? fmaf(x * z, p, x) : far;
}

// ------------------------------------------------------------------ the line of units

constexpr int kThreads = kWaves * 64;

__device__ __forceinline__ Sequence sequence_of(const Args &p, int b)
{
    return sequence(p.shape, p.starts[b], p.starts[b + 1], p.lengths[b]);
}

__device__ __forceinline__ unsigned scan(unsigned v)
{
    const int lane = threadIdx.x % 64;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const unsigned w = __shfl_up(v, o);
        if (lane >= o) v += w;
    }
    return v;
}

// All sequences.  Up to 64 of them are a lane's each, and every wave knows them
// without waiting for another (a call of one token: two barriers and the reading of
// its sequence's indices less); of more, each work-item adds up its own run.
template <int THREADS>
struct Line {
    struct Shared {
        unsigned ends[THREADS], waves[THREADS / 64], base;
        int b;
    };
    const Args &p;
    Shared &s;
    const bool few;
    Sequence mine;
    unsigned end;  // of this lane's sequence
    unsigned total;

    __device__ __forceinline__ Line(const Args &args, Shared &shared) : p(args), s(shared), few(args.B <= 64)
    {
        const int t = threadIdx.x, lane = t % 64;
        if (few) {
            mine = sequence(p.shape, 0, 0, 0);
            if (lane < p.B) mine = sequence_of(p, lane);
            end = scan(mine.cost(p.shape.heads));
            total = __builtin_amdgcn_readlane(end, 63);
            return;
        }
        const int run = (p.B + THREADS - 1) / THREADS;
        unsigned sum = 0;
        for (int b = t * run; b < (t + 1) * run && b < p.B; ++b) sum += sequence_of(p, b).cost(p.shape.heads);
        end = scan(sum);
        if (lane == 63) s.waves[t / 64] = end;
        __syncthreads();
        total = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w < t / 64) end += s.waves[w];
            total += s.waves[w];
        }
        s.ends[t] = end;
        __syncthreads();
    }
    // sequence b's indices
    __device__ __forceinline__ Sequence get(int b) const
    {
        if (!few) return sequence_of(p, b);
        Sequence q;
        q.first = __builtin_amdgcn_readlane(mine.first, b);
        q.tokens = __builtin_amdgcn_readlane(mine.tokens, b);
        q.length = __builtin_amdgcn_readlane(mine.length, b);
        q.keys = __builtin_amdgcn_readlane(mine.keys, b);
        q.groups = __builtin_amdgcn_readlane(mine.groups, b);
        q.units = __builtin_amdgcn_readlane(mine.units, b);
        return q;
    }
    // the sequence that has unit u < total, and the units before it
    __device__ __forceinline__ void find(unsigned u, int &b, unsigned &base) const
    {
        const int t = threadIdx.x;
        if (few) {
            b = __builtin_ctzll(__ballot(u < end));
            base = b ? __builtin_amdgcn_readlane(end, b - 1) : 0;
            return;
        }
        const unsigned before = t ? s.ends[t - 1] : 0;
        if (u >= before && u < end) {
            unsigned at = before;
            int i = t * ((p.B + THREADS - 1) / THREADS);
            for (;; ++i) {
                const unsigned c = sequence_of(p, i).cost(p.shape.heads);
                if (u < at + c) break;
                at += c;
            }
            s.b = i;
            s.base = at;
        }
        __syncthreads();
        b = __builtin_amdgcn_readfirstlane(s.b);
        base = __builtin_amdgcn_readfirstlane(s.base);
    }
};

// The work-group's number on the line: neighbours on it share an XCD's L2.
__device__ __forceinline__ unsigned rank_of(unsigned block, unsigned active)
{
    const unsigned x = block % 8, extra = active % 8;
    return x * (active / 8) + (x < extra ? x : extra) + block / 8;
}

// A part's place in the workspace: `rows` x D sums, then maxima and sums of exponentials.
template <int D>
__device__ __forceinline__ float *part_of(const Args &p, unsigned group, int slot)
{
    return p.parts + (((uint64_t)group * 2 + slot) * (D + 2) << p.shape.rows_shift);
}

// Row r of an item's group: its token and query head.
struct RowAt {
    int64_t m;
    int h;
};
__device__ __forceinline__ RowAt row_at(const Args &p, const Sequence &q, int head, int r)
{
    const int t = r / p.shape.group;
    return {q.first + t, head * p.shape.group + (r - t * p.shape.group)};
}

// Four channels of a finished row, and its lse.
template <typename T>
__device__ __forceinline__ void finish(const Args &p, const Sequence &q, int head, int r, int c, f32x4 o, float l, float most)
{
    const RowAt at = row_at(p, q, head, r);
    const float inv = l == 0.f ? 0.f : 1.f / l;  // a row that saw nothing
    T *to = (T *)p.out + at.m * p.out_token + at.h * p.out_head + c;
    typename Pack<T, 4>::V v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = rounded<T>(o[j] * inv);
    if (c + 4 <= p.d) {
        *reinterpret_cast<typename Pack<T, 4>::U *>(to) = v;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < p.d) to[j] = v[j];
    }
    if (c == 0 && p.lse)
        p.lse[at.m * p.lse_token + at.h] = l == 0.f ? -__builtin_inff() : (most + __builtin_amdgcn_logf(l)) * kLn2;
}

// exp2(m - most), 0 for a part that saw nothing
__device__ __forceinline__ float weight_of(float m, float most)
{
    return m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m - most);
}

// ------------------------------------------------------------------ the attention

// NQ groups of 16 rows; the waves divide the positions.
template <typename T, int D, int NQ>
__global__ void __launch_bounds__(kThreads) attention_kernel(Args p)
{
    typedef typename Eight<T>::V V8;
    constexpr int C = D / 32, N = D / 16, ROWS = 16 * NQ;
    constexpr int kSum = ROWS * (D + 4) * 4;  // a wave's sums
    constexpr int kWave = Staged<T, D>::kBytes > kSum ? Staged<T, D>::kBytes : kSum;
    __shared__ __align__(16) char s_raw[kWaves * kWave];
    __shared__ Line<kThreads>::Shared s_line;
    __shared__ float s_m[kWaves][ROWS], s_l[kWaves][ROWS];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, col = lane % 16, g = lane / 16;
    T *s_v = reinterpret_cast<T *>(s_raw + wave * kWave);

    const Line<kThreads> line(p, s_line);
    const unsigned total = line.total, each = share(total, gridDim.x), active = (total + each - 1) / each;
    if (blockIdx.x >= active) return;
    const unsigned rank = rank_of(blockIdx.x, active), share_begin = rank * each;
    const unsigned share_end = share_begin + each < total ? share_begin + each : total;
    int b;
    unsigned base;
    line.find(share_begin, b, base);
    Sequence seq = line.get(b);

    for (unsigned u = share_begin; u < share_end;) {
        while (u >= base + seq.cost(p.shape.heads)) {
            base += seq.cost(p.shape.heads);
            seq = line.get(++b);
        }
        const unsigned item = (u - base) / (unsigned)seq.units, item_begin = base + item * seq.units, part_begin = u;
        const unsigned part_end = item_begin + seq.units < share_end ? item_begin + seq.units : share_end;
        const int head = (int)(item / (unsigned)seq.groups), row0 = (int)(item % (unsigned)seq.groups) * ROWS;
        const int rows = seq.tokens * p.shape.group - row0 < ROWS ? seq.tokens * p.shape.group - row0 : ROWS;
        const int begin = p.shape.unit_shift < 0 ? 0 : (int)(part_begin - item_begin) << p.shape.unit_shift;
        const int end = part_end == item_begin + seq.units ? seq.keys : (int)(part_end - item_begin) << p.shape.unit_shift;
        const int length = seq.length;
        const T *key = (const T *)p.key + head * p.key_head, *value = (const T *)p.value + head * p.value_head;
        const int32_t *table = p.table + b * p.table_row;

        // the rows, and which of the sequence's tokens each sees
        V8 q[NQ][C];
        uint64_t word[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int r = n * 16 + col;
            word[n] = 0;
            const T *at = (const T *)p.q;
            if (r < rows) {
                const RowAt row = row_at(p, seq, head, row0 + r);
                at += row.m * p.q_token + row.h * p.q_head;
                word[n] = p.mask ? p.mask[row.m] : ~0ull >> (63 - (int)(row.m - seq.first));
            }
#pragma unroll
            for (int c = 0; c < C; ++c) q[n][c] = get8(at + c * 32 + g * 8, r < rows ? p.d - c * 32 - g * 8 : 0);
        }

        f32x4 o[NQ][N];
        float m[NQ], l[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            m[n] = -__builtin_inff();
            l[n] = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) o[n][i] = (f32x4)0.f;
        }

        // where positions at + col and at + 16 + col lie: their pages' numbers
        auto page_at = [&](int j) {
            int page = -1;
            if (j < end) page = table[p.page_shift >= 0 ? j >> p.page_shift : (unsigned)j / (unsigned)p.page_size];
            return (unsigned)page < (uint64_t)p.pages ? page : -1;
        };
        auto place_in = [&](int j) {
            return p.page_shift >= 0 ? j & (p.page_size - 1) : (int)((unsigned)j % (unsigned)p.page_size);
        };
        V8 kk[2][C], vv[2][C];
        auto fetch = [&](int at, const int *page) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int place = place_in(at + h * 16 + col);
                const T *pk = key, *pv = value;
                if (page[h] >= 0) {
                    pk += page[h] * p.key_page + place * p.key_place;
                    pv += page[h] * p.value_page + place * p.value_place;
                }
#pragma unroll
                for (int c = 0; c < C; ++c) kk[h][c] = get8(pk + c * 32 + g * 8, page[h] >= 0 ? p.d - c * 32 - g * 8 : 0);
#pragma unroll
                for (int c = 0; c < C; ++c) vv[h][c] = get8(pv + c * 32 + g * 8, page[h] >= 0 ? p.d - c * 32 - g * 8 : 0);
            }
        };
        int at = begin + wave * kTile;
        int page[2] = {page_at(at + col), page_at(at + 16 + col)};
        if (at < end) fetch(at, page);
        int next[2] = {page_at(at + kUnit + col), page_at(at + kUnit + 16 + col)};

        for (; at < end; at += kUnit) {
            // positions that hold something
            const unsigned there = (unsigned)(__ballot(page[0] >= 0) & 0xffff) | (unsigned)(__ballot(page[1] >= 0) & 0xffff) << 16;
            f32x4 x[NQ][2];
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    x[n][h] = (f32x4)0.f;
#pragma unroll
                    for (int c = 0; c < C; ++c) x[n][h] = product(kk[h][c], q[n][c], x[n][h]);
                }
            // V to LDS; a token's NaN or infinity is told from here on
            bool odd = false;
            const bool drafted = at + kTile > length;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    *reinterpret_cast<V8 *>(s_v + (h * 16 + col) * Staged<T, D>::kRow + c * 32 + g * 8) = vv[h][c];
                    if (drafted) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) odd |= !(fabsf((float)vv[h][c][j]) < __builtin_inff());
                    }
                }
            odd = __any(odd);
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            // the next tile on its way
            page[0] = next[0];
            page[1] = next[1];
            if (at + kUnit < end) fetch(at + kUnit, page);
            next[0] = page_at(at + 2 * kUnit + col);
            next[1] = page_at(at + 2 * kUnit + 16 + col);

            V8 weight[NQ];
            unsigned seen[NQ];
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                seen[n] = there;
                if (drafted) {
                    const int off = length - at;  // the tile's first token
                    seen[n] &= off > 0 ? (unsigned)(word[n] << off) | ((1u << off) - 1) : -off < 64 ? (unsigned)(word[n] >> -off) : 0u;
                }
                float most = -__builtin_inff(), s[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s[e] = x[n][e / 4][e % 4] * p.scale;
                    if (p.cap != 0.f) s[e] = tanh_of(s[e]) * p.cap;
                }
                if (seen[n] != ~0u) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (!(seen[n] >> (e / 4 * 16 + g * 4 + e % 4) & 1)) s[e] = -__builtin_inff();
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) most = fmaxf(most, s[e]);
                most = fmaxf(most, __shfl_xor(most, 16));
                most = fmaxf(most, __shfl_xor(most, 32));
                most = fmaxf(most, m[n]);
                const float origin = most == -__builtin_inff() ? 0.f : most;
                const float shrink = __builtin_amdgcn_exp2f(m[n] - origin);
                m[n] = most;
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s[e] = __builtin_amdgcn_exp2f(s[e] - origin);
                    sum += s[e];
                    weight[n][e] = (T)s[e];
                }
                l[n] = fmaf(l[n], shrink, sum);
#pragma unroll
                for (int i = 0; i < N; ++i) o[n][i] *= shrink;
            }
            if (!odd) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const V8 v = Staged<T, D>::column(s_v, i, lane);
#pragma unroll
                    for (int n = 0; n < NQ; ++n) o[n][i] = product(v, weight[n], o[n][i]);
                }
            } else {
                // a NaN or an infinity reaches the rows that see it and no other: position by position
#pragma unroll
                for (int n = 0; n < NQ; ++n)
                    for (int from = 0; from < 4; ++from) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int j = e / 4 * 16 + from * 4 + e % 4;
                            const float w = __shfl((float)weight[n][e], from * 16 + col);
#pragma unroll 1
                            for (int c = 0; c < N * 4; ++c) {
                                const float v = (float)s_v[j * Staged<T, D>::kRow + (c / 4) * 16 + g * 4 + c % 4];
                                const float add = seen[n] >> j & 1 ? w * v : 0.f;
#pragma unroll
                                for (int i = 0; i < N * 4; ++i)
                                    if (i == c) o[n][i / 4][i % 4] += add;
                            }
                        }
                    }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }

        // the waves' sums together
        float *s_o = reinterpret_cast<float *>(s_raw + wave * kWave);
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            l[n] += __shfl_xor(l[n], 16);
            l[n] += __shfl_xor(l[n], 32);
            if (g == 0) {
                s_m[wave][n * 16 + col] = m[n];
                s_l[wave][n * 16 + col] = l[n];
            }
#pragma unroll
            for (int i = 0; i < N; ++i) *reinterpret_cast<f32x4 *>(s_o + (n * 16 + col) * (D + 4) + i * 16 + g * 4) = o[n][i];
        }
        __syncthreads();
        const bool whole = part_begin == item_begin && part_end == item_begin + seq.units;
        float *part = whole ? nullptr : part_of<D>(p, rank, slot_of(part_begin, share_begin));
        for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads) {
            const int r = i / (D / 4), c = i % (D / 4) * 4;
            float most = s_m[0][r];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) most = fmaxf(most, s_m[w][r]);
            f32x4 sum = (f32x4)0.f;
            float all = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float f = weight_of(s_m[w][r], most);
                sum += *reinterpret_cast<const f32x4 *>(s_raw + w * kWave + (r * (D + 4) + c) * 4) * f;
                all += s_l[w][r] * f;
            }
            if (whole) {
                if (c < p.d) finish<T>(p, seq, head, row0 + r, c, sum, all, most);
            } else {
                *reinterpret_cast<f32x4 *>(part + r * D + c) = sum;
                if (c == 0) {
                    part[ROWS * D + r] = most;
                    part[ROWS * (D + 1) + r] = all;
                }
            }
        }
        __syncthreads();
        u = part_end;
    }
}

// ------------------------------------------------------------------ the attention, copied to LDS

// A wave's 32 rows of K or V in LDS as copies leave them: 1 KiB an instruction, 16
// bytes a lane, so that a row's chunks of 16 bytes lie side by side.  Chunk c of row r
// is at place c ^ turn(r): sixteen rows' chunks of one column lie in all banks.
template <typename T, int D>
struct Copied {
    static constexpr int kChunks = D * (int)sizeof(T) / 16;  // of a row
    static constexpr int kRow = kChunks * 16;
    static constexpr int kBytes = kTile * kRow;
    static constexpr int kRows = 64 / kChunks;      // of a copy
    static constexpr int kCopies = kTile / kRows;   // of a tile
    static constexpr int kTurns = kRows >= 16 ? 1 : 16 / kRows < kCopies ? 16 / kRows : kCopies;  // copies until turn() repeats

    static __device__ __forceinline__ int turn(int r) { return kChunks >= 16 ? r & 15 : r >> 1 & 7; }

    // channels 8 i on of row r, for the product's operand
    static __device__ __forceinline__ typename Eight<T>::V row(const char *s, int r, int i)
    {
        if constexpr (sizeof(T) == 2) {
            return *reinterpret_cast<const typename Eight<T>::V *>(s + r * kRow + (i ^ turn(r)) * 16);
        } else {
            const f32x4 lo = *reinterpret_cast<const f32x4 *>(s + r * kRow + (2 * i ^ turn(r)) * 16);
            const f32x4 hi = *reinterpret_cast<const f32x4 *>(s + r * kRow + ((2 * i + 1) ^ turn(r)) * 16);
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }

    // channel 16 n + lane % 16 of positions 4 (lane / 16) + 0..3 and those + 16
    static __device__ __forceinline__ typename Eight<T>::V column(const char *s, int n, int lane)
    {
        typename Eight<T>::V v;
        if constexpr (sizeof(T) == 2) {
            typedef short S4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) S4 *P;
            const int r = lane / 4;
            const char *p = s + r * kRow + ((2 * n + lane / 2 % 2) ^ turn(r)) * 16 + lane % 2 * 8;
            const S4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)p);
            const S4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p + 16 * kRow));
            const auto both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            v = __builtin_bit_cast(typename Eight<T>::V, both);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = lane / 16 * 4 + j;
                const char *p = s + r * kRow + ((4 * n + lane / 4 % 4) ^ turn(r)) * 16 + lane % 4 * 4;
                v[j] = *reinterpret_cast<const float *>(p);
                v[4 + j] = *reinterpret_cast<const float *>(p + 16 * kRow);
            }
        }
        return v;
    }

    // element (r, channel)
    static __device__ __forceinline__ float at(const char *s, int r, int channel)
    {
        const int byte = channel * (int)sizeof(T);
        return (float)*reinterpret_cast<const T *>(s + r * kRow + (byte / 16 ^ turn(r)) * 16 + byte % 16);
    }
};

// Each lane's 16 bytes at base + off to the wave's 1 KiB from `to` on.  Written out,
// because the compiler would wait for every such copy before the next read of LDS; the
// wave waits for a tile's when it begins it.  m0, where `to` is passed, is read one wait
// state after it is set, scalar operands five after a vector instruction that may
// have made them.
__device__ __forceinline__ void copy16(char *to, const char *base, unsigned off)
{
    const unsigned at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void *)to;
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" : : "{m0}"(at), "v"(off), "s"(base) : "memory");
}

// The same attention where K's and V's rows are whole chunks of 16 bytes and a copy's
// rows lie in one page.  A wave's tiles go from memory straight to its own part of
// LDS, one on its way while the one before is worked on; nothing waits for another
// wave until their sums are joined.
template <typename T, int D, int NQ, int WAVES>
__global__ void __launch_bounds__(WAVES * 64) stream_kernel(Args p)
{
    typedef typename Eight<T>::V V8;
    typedef Copied<T, D> S;
    constexpr int C = D / 32, N = D / 16, ROWS = 16 * NQ, THREADS = WAVES * 64, STEP = WAVES * kTile;
    constexpr int kStage = 2 * S::kBytes, kWave = 2 * kStage;  // K and V, twice
    static_assert(ROWS * (D + 4) * 4 <= kWave, "a wave's sums fit its stages");
    __shared__ __align__(16) char s_raw[WAVES * kWave];
    __shared__ typename Line<THREADS>::Shared s_line;
    __shared__ float s_m[WAVES][ROWS], s_l[WAVES][ROWS];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, g = lane / 16;
    char *const s_own = s_raw + wave * kWave;

    const Line<THREADS> line(p, s_line);
    const unsigned total = line.total, each = share(total, gridDim.x), active = (total + each - 1) / each;
    if (blockIdx.x >= active) return;
    const unsigned rank = rank_of(blockIdx.x, active), share_begin = rank * each;
    const unsigned share_end = share_begin + each < total ? share_begin + each : total;
    int b;
    unsigned base;
    line.find(share_begin, b, base);
    Sequence seq = line.get(b);

    // what a lane copies: a row of each copy, and its chunk of it
    const int chunks = p.d * (int)sizeof(T) / 16;
    unsigned key_off[S::kTurns], value_off[S::kTurns];
    bool copies[S::kTurns];
#pragma unroll
    for (int t = 0; t < S::kTurns; ++t) {
        const int r = lane / S::kChunks, c = lane % S::kChunks ^ S::turn(t * S::kRows + r);
        key_off[t] = (unsigned)(r * (int)p.key_place * (int)sizeof(T) + c * 16);
        value_off[t] = (unsigned)(r * (int)p.value_place * (int)sizeof(T) + c * 16);
        copies[t] = c < chunks;
    }
    // chunks that no copy writes are multiplied by zeros
    if (p.d != D)
        for (int i = threadIdx.x; i < WAVES * kWave / 16; i += THREADS) reinterpret_cast<f32x4 *>(s_raw)[i] = (f32x4)0.f;
    bool zeroed = p.d != D;

    for (unsigned u = share_begin; u < share_end;) {
        while (u >= base + seq.cost(p.shape.heads)) {
            base += seq.cost(p.shape.heads);
            seq = line.get(++b);
        }
        const unsigned item = (u - base) / (unsigned)seq.units, item_begin = base + item * seq.units, part_begin = u;
        const unsigned part_end = item_begin + seq.units < share_end ? item_begin + seq.units : share_end;
        const int head = (int)(item / (unsigned)seq.groups), row0 = (int)(item % (unsigned)seq.groups) * ROWS;
        const int rows = seq.tokens * p.shape.group - row0 < ROWS ? seq.tokens * p.shape.group - row0 : ROWS;
        const int begin = p.shape.unit_shift < 0 ? 0 : (int)(part_begin - item_begin) << p.shape.unit_shift;
        const int end = part_end == item_begin + seq.units ? seq.keys : (int)(part_end - item_begin) << p.shape.unit_shift;
        const int length = seq.length;
        const char *key = (const char *)((const T *)p.key + head * p.key_head);
        const char *value = (const char *)((const T *)p.value + head * p.value_head);
        const int32_t *table = p.table + b * p.table_row;

        // lane r and r + 32 have row r of a tile: whether it holds something, and where it lies
        auto page_at = [&](int j) {
            int page = -1;
            if (j < end) page = table[p.page_shift >= 0 ? j >> p.page_shift : (unsigned)j / (unsigned)p.page_size];
            return (unsigned)page < (uint64_t)p.pages ? page : -1;
        };
        auto copy = [&](int at, int page, char *to) {
            const int j = at + lane % 32;
            const int place = p.page_shift >= 0 ? j & (p.page_size - 1) : (int)((unsigned)j % (unsigned)p.page_size);
            const int64_t k = (page * p.key_page + place * p.key_place) * (int)sizeof(T);
            const int64_t v = (page * p.value_page + place * p.value_place) * (int)sizeof(T);
            auto from = [&](const char *first, int64_t off, int r) {
                const unsigned lo = __builtin_amdgcn_readlane((int)off, r), hi = __builtin_amdgcn_readlane((int)(off >> 32), r);
                return first + (int64_t)((uint64_t)hi << 32 | lo);
            };
            const unsigned there = (unsigned)__ballot(page >= 0);
            // all of K, then all of V
#pragma unroll
            for (int i = 0; i < S::kCopies; ++i)
                if (there >> (i * S::kRows) & 1) {
                    const char *at = from(key, k, i * S::kRows);
                    if (copies[i % S::kTurns]) copy16(to + i * 1024, at, key_off[i % S::kTurns]);
                }
#pragma unroll
            for (int i = 0; i < S::kCopies; ++i)
                if (there >> (i * S::kRows) & 1) {
                    const char *at = from(value, v, i * S::kRows);
                    if (copies[i % S::kTurns]) copy16(to + S::kBytes + i * 1024, at, value_off[i % S::kTurns]);
                }
        };
        int at = begin + wave * kTile, stage = 0;
        int page = page_at(at + lane % 32);
        if (zeroed) {
            __syncthreads();  // the zeros are in place
            zeroed = false;
        }
        if (at < end) copy(at, page, s_own);
        int next = page_at(at + STEP + lane % 32);

        // the rows, and which of the sequence's tokens each sees
        V8 q[NQ][C];
        uint64_t word[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int r = n * 16 + col;
            word[n] = 0;
            const T *from = (const T *)p.q;
            if (r < rows) {
                const RowAt row = row_at(p, seq, head, row0 + r);
                from += row.m * p.q_token + row.h * p.q_head;
                word[n] = p.mask ? p.mask[row.m] : ~0ull >> (63 - (int)(row.m - seq.first));
            }
#pragma unroll
            for (int c = 0; c < C; ++c) q[n][c] = get8(from + c * 32 + g * 8, r < rows ? p.d - c * 32 - g * 8 : 0);
        }
        f32x4 o[NQ][N];
        float m[NQ], l[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            m[n] = -__builtin_inff();
            l[n] = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) o[n][i] = (f32x4)0.f;
        }

        for (; at < end; at += STEP, stage ^= 1) {
            char *const s_k = s_own + stage * kStage, *const s_v = s_k + S::kBytes;
            const unsigned there = (unsigned)__ballot(page >= 0);
            // this tile is here, and the other stage has been read
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            if (at + STEP < end) copy(at + STEP, next, s_own + (stage ^ 1) * kStage);
            page = next;
            next = page_at(at + 2 * STEP + lane % 32);

            if (there != ~0u) {
                // V's rows that hold nothing: zeros, whatever was copied with them
                for (int i = lane; i < S::kBytes / 16; i += 64)
                    if (!(there >> (i / S::kChunks) & 1)) reinterpret_cast<f32x4 *>(s_v)[i] = (f32x4)0.f;
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
            const bool drafted = at + kTile > length;
            bool odd = false;
            if (drafted) {
                // a token's NaN or infinity: some rows may not see it
                for (int i = lane; i < S::kBytes / 16; i += 64) {
                    typedef T V __attribute__((ext_vector_type(16 / sizeof(T))));
                    const V v = reinterpret_cast<const V *>(s_v)[i];
#pragma unroll
                    for (int j = 0; j < 16 / (int)sizeof(T); ++j) odd |= !(fabsf((float)v[j]) < __builtin_inff());
                }
                odd = __any(odd);
            }

            f32x4 x[NQ][2];
#pragma unroll
            for (int n = 0; n < NQ; ++n) x[n][0] = x[n][1] = (f32x4)0.f;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const V8 k = S::row(s_k, h * 16 + col, c * 4 + g);
#pragma unroll
                    for (int n = 0; n < NQ; ++n) x[n][h] = product(k, q[n][c], x[n][h]);
                }

            V8 weight[NQ];
            unsigned seen[NQ];
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                seen[n] = there;
                if (drafted) {
                    const int off = length - at;  // the tile's first token
                    seen[n] &= off > 0 ? (unsigned)(word[n] << off) | ((1u << off) - 1) : -off < 64 ? (unsigned)(word[n] >> -off) : 0u;
                }
                float most = -__builtin_inff(), s[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s[e] = x[n][e / 4][e % 4] * p.scale;
                    if (p.cap != 0.f) s[e] = tanh_of(s[e]) * p.cap;
                }
                if (drafted || there != ~0u) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (!(seen[n] >> (e / 4 * 16 + g * 4 + e % 4) & 1)) s[e] = -__builtin_inff();
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) most = fmaxf(most, s[e]);
                most = fmaxf(most, __shfl_xor(most, 16));
                most = fmaxf(most, __shfl_xor(most, 32));
                // the sums' origin moves only where a weight would pass 2^8: they stay in range,
                // and nearly no tile has them multiplied
                if (__any(most > m[n] + 8.f)) {
                    most = fmaxf(most, m[n]);
                    const float shrink = __builtin_amdgcn_exp2f(m[n] - (most == -__builtin_inff() ? 0.f : most));
                    m[n] = most;
                    l[n] *= shrink;
#pragma unroll
                    for (int i = 0; i < N; ++i) o[n][i] *= shrink;
                }
                const float origin = m[n] == -__builtin_inff() ? 0.f : m[n];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s[e] = __builtin_amdgcn_exp2f(s[e] - origin);
                    l[n] += s[e];
                    weight[n][e] = (T)s[e];
                }
            }
            if (!odd) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const V8 v = S::column(s_v, i, lane);
#pragma unroll
                    for (int n = 0; n < NQ; ++n) o[n][i] = product(v, weight[n], o[n][i]);
                }
            } else {
                // a NaN or an infinity reaches the rows that see it and no other: position by position
#pragma unroll
                for (int n = 0; n < NQ; ++n)
                    for (int from = 0; from < 4; ++from) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int j = e / 4 * 16 + from * 4 + e % 4;
                            const float w = __shfl((float)weight[n][e], from * 16 + col);
                            const bool sees = seen[n] >> j & 1;
#pragma unroll
                            for (int i = 0; i < N; ++i)
#pragma unroll
                                for (int c = 0; c < 4; ++c) {
                                    const float v = S::at(s_v, j, i * 16 + g * 4 + c);
                                    o[n][i][c] += sees ? w * v : 0.f;
                                }
                        }
                    }
            }
        }

        // the waves' sums together
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        float *s_o = reinterpret_cast<float *>(s_own);
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            l[n] += __shfl_xor(l[n], 16);
            l[n] += __shfl_xor(l[n], 32);
            if (g == 0) {
                s_m[wave][n * 16 + col] = m[n];
                s_l[wave][n * 16 + col] = l[n];
            }
#pragma unroll
            for (int i = 0; i < N; ++i) *reinterpret_cast<f32x4 *>(s_o + (n * 16 + col) * (D + 4) + i * 16 + g * 4) = o[n][i];
        }
        __syncthreads();
        const bool whole = part_begin == item_begin && part_end == item_begin + seq.units;
        float *part = whole ? nullptr : part_of<D>(p, rank, slot_of(part_begin, share_begin));
        for (int i = threadIdx.x; i < rows * (D / 4); i += THREADS) {
            const int r = i / (D / 4), c = i % (D / 4) * 4;
            float most = s_m[0][r];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) most = fmaxf(most, s_m[w][r]);
            f32x4 sum = (f32x4)0.f;
            float all = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = weight_of(s_m[w][r], most);
                sum += *reinterpret_cast<const f32x4 *>(s_raw + w * kWave + (r * (D + 4) + c) * 4) * f;
                all += s_l[w][r] * f;
            }
            if (whole) {
                if (c < p.d) finish<T>(p, seq, head, row0 + r, c, sum, all, most);
            } else {
                *reinterpret_cast<f32x4 *>(part + r * D + c) = sum;
                if (c == 0) {
                    part[ROWS * D + r] = most;
                    part[ROWS * (D + 1) + r] = all;
                }
            }
        }
        __syncthreads();
        if (p.d != D && part_end < share_end) {
            for (int i = threadIdx.x; i < WAVES * kWave / 16; i += THREADS) reinterpret_cast<f32x4 *>(s_raw)[i] = (f32x4)0.f;
            zeroed = true;
        }
        u = part_end;
    }
}

constexpr int kJoinThreads = 1024;

// Joins the parts of items that more than one work-group had.  A work-group for each
// border between shares; the first border in an item does it.  Its lanes take four
// channels of a row each, and where there are fewer of them than lanes, the parts in
// turn: many parts (a long sequence alone) would else be read one after the other.
// Sums are made in an order that the call's sizes alone decide.
template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(Args p, unsigned groups)
{
    __shared__ typename Line<kJoinThreads>::Shared s_line;
    __shared__ float s_sum[kJoinThreads][7];  // a maximum, a sum of exponentials, four of values; odd, for the banks
    const Line<kJoinThreads> line(p, s_line);
    const unsigned total = line.total, each = share(total, groups), border = (blockIdx.x + 1) * each;
    if (border >= total) return;
    int b;
    unsigned base;
    line.find(border, b, base);
    const Sequence seq = line.get(b);
    const unsigned item = (border - base) / (unsigned)seq.units, begin = base + item * seq.units, end = begin + seq.units;
    if (begin == border || begin + each < border) return;
    const int most_rows = 1 << p.shape.rows_shift, head = (int)(item / (unsigned)seq.groups);
    const int row0 = (int)(item % (unsigned)seq.groups) * most_rows;
    const int rows = seq.tokens * p.shape.group - row0 < most_rows ? seq.tokens * p.shape.group - row0 : most_rows;
    const unsigned first = blockIdx.x, parts = (end - 1) / each - first + 1;
    auto part = [&](unsigned i) {
        const unsigned from = (first + i) * each;
        return part_of<D>(p, first + i, slot_of(i ? from : begin, from));
    };
    // lanes to a part's sums: a power of two
    int lanes = D / 4;
    while (lanes < rows * (D / 4) && lanes < kJoinThreads) lanes *= 2;
    const int turns = kJoinThreads / lanes, turn = threadIdx.x / lanes;
    for (int i = threadIdx.x % lanes; i - (int)(threadIdx.x % lanes) < rows * (D / 4); i += lanes) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        const bool on = r < rows;
        float most = -__builtin_inff(), all = 0.f;
        f32x4 sum = (f32x4)0.f;
        if (on) {
#pragma unroll 8
            for (unsigned w = turn; w < parts; w += turns) most = fmaxf(most, part(w)[D * most_rows + r]);
#pragma unroll 8
            for (unsigned w = turn; w < parts; w += turns) {
                const float *from = part(w), f = weight_of(from[D * most_rows + r], most);
                sum += *reinterpret_cast<const f32x4 *>(from + r * D + c) * f;
                all += from[(D + 1) * most_rows + r] * f;
            }
        }
        // the turns' sums, two by two
        float *mine = s_sum[threadIdx.x];
        for (int o = turns / 2; o > 0; o /= 2) {
            __syncthreads();
            if (turn >= o && turn < 2 * o) {
                mine[0] = most;
                mine[1] = all;
#pragma unroll
                for (int j = 0; j < 4; ++j) mine[2 + j] = sum[j];
            }
            __syncthreads();
            if (turn < o) {
                const float *other = s_sum[threadIdx.x + o * lanes];
                const float top = fmaxf(most, other[0]), f = weight_of(most, top), h = weight_of(other[0], top);
                all = all * f + other[1] * h;
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] = sum[j] * f + other[2 + j] * h;
                most = top;
            }
        }
        if (turn == 0 && on && c < p.d) finish<T>(p, seq, head, row0 + r, c, sum, all, most);
    }
}

// ------------------------------------------------------------------ launches

int padded(int64_t d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

struct Form {
    int D, nq;
    int unit;        // positions that a work-group's waves have in work
    int64_t groups;  // work-groups
    size_t bytes;    // of the workspace
    int64_t items;
};

// Waves of stream_kernel: what a CU's LDS holds of their stages.
constexpr int stream_waves(int row_bytes) { return row_bytes >= 1024 ? 1 : row_bytes >= 512 ? 2 : 4; }

// The form of a call: the work-groups that the card holds at once.
Form form_of(int size, int64_t d, int64_t group, int64_t heads, int64_t B, int64_t capacity, int64_t most, bool copied)
{
    Form f;
    f.D = padded(d);
    const int waves = copied ? stream_waves(f.D * size) : kWaves;
    f.nq = most * group > 16 && f.D <= 128 ? 2 : 1;
    f.unit = waves * kTile;
    const int64_t items = B * heads * ((most * group + 16 * f.nq - 1) / (16 * f.nq));
    const int64_t units = capacity <= f.unit ? 1 : (capacity + f.unit - 1) / f.unit;
    const bool divided = items <= kMostLine / units;  // else an item is a unit
    const int64_t line = divided ? items * units : items;
    f.items = items;
    if (copied)
        f.groups = 256 * (f.D * size <= 128 ? 2 : 1);
    else
        f.groups = 256 * (f.D == 256 ? 1 : f.nq == 2 ? 2 : 3);
    if (f.groups > line) f.groups = line;
    f.bytes = units == 1 || !divided ? 0 : (size_t)f.groups * 2 * 16 * f.nq * (f.D + 2) * sizeof(float);
    return f;
}

template <typename T, int D>
int join(const Args &a, const Form &f, bool joined, hipStream_t s)
{
    if (hipGetLastError() != hipSuccess) return PK_ERR_LAUNCH;
    if (!joined || f.groups == 1) return PK_OK;
    hipLaunchKernelGGL((join_kernel<T, D>), dim3((unsigned)(f.groups - 1)), dim3(kJoinThreads), 0, s, a, (unsigned)f.groups);
    return hipGetLastError() == hipSuccess ? PK_OK : PK_ERR_LAUNCH;
}

template <typename T, int D, int NQ>
int launch(const Args &a, const Form &f, bool copied, bool joined, hipStream_t s)
{
    if (copied) {
        constexpr int WAVES = stream_waves(D * (int)sizeof(T));
        hipLaunchKernelGGL((stream_kernel<T, D, NQ, WAVES>), dim3((unsigned)f.groups), dim3(WAVES * 64), 0, s, a);
    } else {
        hipLaunchKernelGGL((attention_kernel<T, D, NQ>), dim3((unsigned)f.groups), dim3(kThreads), 0, s, a);
    }
    return join<T, D>(a, f, joined, s);
}

template <typename T>
int launch(const Args &a, const Form &f, bool copied, bool joined, hipStream_t s)
{
    if (f.D == 64) return f.nq == 1 ? launch<T, 64, 1>(a, f, copied, joined, s) : launch<T, 64, 2>(a, f, copied, joined, s);
    if (f.D == 128) return f.nq == 1 ? launch<T, 128, 1>(a, f, copied, joined, s) : launch<T, 128, 2>(a, f, copied, joined, s);
    return launch<T, 256, 1>(a, f, copied, joined, s);
}

// Whether K and V can be copied in whole chunks: 16-byte rows at 16-byte places, the
// rows of a copy (up to 8) in one page and within 32-bit offsets of each other.
bool can_copy(const pk_cache &c, int64_t d, int size)
{
    if (d * size % 16 || (uintptr_t)c.key % 16 || (uintptr_t)c.value % 16 || c.page_size % 8) return false;
    for (int i = 0; i < 3; ++i)
        if (c.key_stride[i] * size % 16 || c.value_stride[i] * size % 16) return false;
    return c.key_stride[1] < 1 << 24 && c.value_stride[1] < 1 << 24;
}

}  // namespace

extern "C" {

size_t pk_attention_tree_workspace_bytes(int dtype, int64_t d, int64_t q_heads, int64_t heads, int64_t B, int64_t P,
                                         int64_t page_size, int64_t most)
{
    using namespace pk::heads;
    if (!pk::dtype_size(dtype) || d < 1 || d > 256 || heads < 1 || q_heads < heads || q_heads % heads || q_heads > kMostHeads ||
        B < 1 || B > kMostSize || P < 1 || P > kMostSize || page_size < 1 || page_size > kMostSize || most < 1 ||
        most > kMostTokens || P * page_size > kMostSize)
        return 0;
    // either form
    const Form a = form_of(pk::dtype_size(dtype), d, q_heads / heads, heads, B, P * page_size, most, false);
    const Form b = form_of(pk::dtype_size(dtype), d, q_heads / heads, heads, B, P * page_size, most, true);
    return a.bytes > b.bytes ? a.bytes : b.bytes;
}

int pk_attention_tree(int dtype, int64_t M, int64_t d, const pk_heads *q, const pk_cache *cache, const int32_t *page_table,
                      int64_t B, int64_t P, int64_t ld_table, const int32_t *lengths, const int32_t *starts, int64_t most,
                      const uint64_t *mask, float scale, float cap, const pk_heads *out, float *lse, int64_t ld_lse,
                      void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace pk;
    using namespace pk::heads;
    api_begin();
    const int size = dtype_size(dtype);
    if (!size) return api_invalid(1);
    if (M < 0) return api_invalid(2);
    if (d < 1) return api_invalid(3);
    if (!q) return api_invalid(4);
    if (!cache) return api_invalid(5);
    if (B < 0) return api_invalid(7);
    if (P < 0) return api_invalid(8);
    if (ld_table < P) return api_invalid(9);
    if (most < 1) return api_invalid(12);
    if (!(cap >= 0.f) || cap > 3e38f) return api_invalid(15);
    if (!out || out->heads != q->heads) return api_invalid(16);
    if (lse && ld_lse < q->heads) return api_invalid(18);
    if ((uintptr_t)workspace % 16) return api_invalid(19);
    if (M > kMostSize || d > 256 || B > kMostSize || P > kMostSize || ld_table > kMostSize || most > kMostTokens ||
        (lse && ld_lse > kMostSize))
        return PK_ERR_NOT_SUPPORTED;
    int st;
    if ((st = check_heads(*q, M, size, false, d))) return st == PK_ERR_INVALID_VALUE ? api_invalid(4) : st;
    if ((st = check_cache(*cache, size, false, d))) return st == PK_ERR_INVALID_VALUE ? api_invalid(5) : st;
    if (cache->heads < 1 || q->heads % cache->heads) return api_invalid(5);
    if ((st = check_heads(*out, M, size, true, d))) return st == PK_ERR_INVALID_VALUE ? api_invalid(16) : st;
    if (P && cache->page_size > kMostSize / P) return PK_ERR_NOT_SUPPORTED;
    if (M == 0 || B == 0 || q->heads == 0) return PK_OK;
    if (P && (!page_table || (uintptr_t)page_table % 4)) return api_invalid(6);
    if (!lengths || (uintptr_t)lengths % 4) return api_invalid(10);
    if (!starts || (uintptr_t)starts % 4) return api_invalid(11);
    if ((uintptr_t)mask % 8) return api_invalid(13);
    if ((uintptr_t)lse % 4) return api_invalid(17);
    const int64_t heads = cache->heads, group = q->heads / heads;
    const bool copied = can_copy(*cache, d, size);
    const Form f = form_of(size, d, group, heads, B, P * cache->page_size, most, copied);
    if (f.items > kMostLine) return PK_ERR_NOT_SUPPORTED;
    const bool joined = f.bytes && workspace && workspace_bytes >= f.bytes;
    const Region in[7] = {of_heads(*q, M, d, size), of_cache(cache->key, cache->key_stride, *cache, d, size),
                          of_cache(cache->value, cache->value_stride, *cache, d, size),
                          matrix(page_table, P ? B : 0, ld_table * 4, P * 4), flat(lengths, 4 * B), flat(starts, 4 * B + 4),
                          flat(mask, mask ? 8 * M : 0)};
    const Region ro = of_heads(*out, M, d, size), rl = matrix(lse, lse ? M : 0, ld_lse * 4, q->heads * 4),
                 rw = flat(workspace, joined ? (int64_t)f.bytes : 0);
    for (int i = 0; i < 7; ++i) {
        if (shared(ro, in[i]) && !(i == 0 && same_place(*q, *out, M))) return api_invalid(16);
        if (shared(rl, in[i])) return api_invalid(17);
        if (shared(rw, in[i])) return api_invalid(19);
    }
    if (shared(rl, ro)) return api_invalid(17);
    if (shared(rw, ro) || shared(rw, rl)) return api_invalid(19);

    Args a = {};
    a.q = q->data;
    a.out = out->data;
    a.key = cache->key;
    a.value = cache->value;
    a.table = page_table;
    a.lengths = lengths;
    a.starts = starts;
    a.mask = mask;
    a.lse = lse;
    a.parts = (float *)workspace;
    a.q_token = q->token_stride;
    a.q_head = q->head_stride;
    a.out_token = out->token_stride;
    a.out_head = out->head_stride;
    a.lse_token = ld_lse;
    a.table_row = ld_table;
    a.key_page = cache->key_stride[0];
    a.key_place = cache->key_stride[1];
    a.key_head = cache->key_stride[2];
    a.value_page = cache->value_stride[0];
    a.value_place = cache->value_stride[1];
    a.value_head = cache->value_stride[2];
    a.pages = cache->pages;
    a.shape = {(int)M, (int)(P * cache->page_size), (int)heads, (int)group, (int)most, f.nq == 2 ? 5 : 4, -1};
    if (joined)
        for (a.shape.unit_shift = 0; 1 << a.shape.unit_shift < f.unit;) ++a.shape.unit_shift;
    a.B = (int)B;
    a.d = (int)d;
    a.page_size = (int)cache->page_size;
    a.page_shift = -1;
    for (int i = 0; i < 31; ++i)
        if ((int64_t)1 << i == cache->page_size) a.page_shift = i;
    a.scale = cap != 0.f ? scale / cap : scale * kLog2e;
    a.cap = cap * kLog2e;
    hipStream_t s = (hipStream_t)stream;
    st = dtype == PK_F32 ? launch<float>(a, f, copied, joined, s) : dtype == PK_BF16 ? launch<bf16>(a, f, copied, joined, s) : launch<f16>(a, f, copied, joined, s);
    if (st == PK_OK) api_ran(copied ? "attention_tree_copied" : "attention_tree_read");
    return st;
}

}  // extern "C"
