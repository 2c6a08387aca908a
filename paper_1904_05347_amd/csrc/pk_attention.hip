// pk_attention.hip -- attention of drafted tokens over a paged cache.
//
//   o_i = sum_j p_ij v_j,  p_i the softmax over the j that row i sees of
//   x_ij = c tanh(scale (q_i . k_j) / c)   (scale (q_i . k_j) without a cap c).
//
// One pass over the cache, 32 positions at a time: for each row the largest x so far,
// the sum of exponentials and the sum of values weighted by them.  All rows that
// read one head of the cache (its tokens times the query heads that share it) are
// columns of one product, so that K and V are read once for up to 128 of them.
//
// Lanes.  x^T = K q^T and o^T = V^T p^T on the 16 x 16 matrix instruction, whose
// operands hold 8 neighbours along the sum a lane: K's and q's rows are read as
// they lie, 16 bytes a lane.  In x^T a lane has one row's (lane % 16) x of four
// neighbouring positions, from two products of eight: the second product's operand,
// without any exchange, where V^T takes its positions in the same order.  V^T comes
// out of LDS transposed.
//
// Few rows: bound by reading the cache (32 sequences of up to 8192 positions, 8 heads of
// 128 bf16: 675 MB in 133 us, 5.1 TB/s, as a large copy).  Many: by the matrix cores,
// from about 400 rows a head (reached: 440 to 665 Tflop/s of a large product's 1234).
// Small calls: by what is waited for one after the other, instructions from a cold cache
// (about 30 ns for each 64 bytes), lengths, table, K, V, the joining launch.
#include "pk_attention_plan.hpp"
#include "pk_heads_checks.hpp"
#include "pk_i8.hpp"
#include "pk_i8_checks.hpp"

#include <cmath>

namespace {

using namespace pk::attention;
using pk::bf16;
using pk::f16;
using pk::Pack;
using pk::rounded;

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;  // positions of one step
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
    // scores are formed in powers of two: scale * log2(e), or scale / cap and cap * log2(e).
    // scale is positive: q is multiplied by its sign (by 0, and scale is 1, for a scale of 0).
    // All are held to what 32 bits hold: an infinite one would make NaN of scores of 0, a
    // subnormal one has too few bits.
    float scale, cap, sign;
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

// Softmax's weights for the matrix instruction.  One number of 16 bits would be off by as much as
// the result's own rounding (2^-8 in bf16, 2^-11 in fp16), so it is two: the weight cut off, and what
// is left, together within 2^-16 of it in bf16, 2^-20 in fp16 (or 2^-23, two of its least numbers).
// The products by V double for it.  Of calls over 4096 to 32768 positions the error against 64
// bits was 1.08 to 1.42 times that of the result's rounding alone, and now is that.  4 trees of 64
// tokens over up to 32768 positions, 64 heads over 8 of 128 bf16, took 199 us and take 223 (all of
// 32768 in fp16 348 and 439), small fp16 calls 19.7 for 18.4, what memory bounds up to 1.5 % more.
template <typename T>
struct Weights {
    typename Eight<T>::V first, second;
    // w[i / 4][i % 4] is weight i
    __device__ __forceinline__ void set(const f32x4 (&w)[2])
    {
        if constexpr (__is_same(T, bf16)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // the upper half of its bits; and 2^-21 more than is left, so that the second is above 0
                // as well (down to weights of 2^-112): an infinite value times 0 would be no number
                const unsigned upper = __float_as_uint(w[i / 4][i % 4]) & 0xffff0000u;
                first[i] = __builtin_bit_cast(bf16, (unsigned short)(upper >> 16));
                second[i] = (bf16)fmaf(w[i / 4][i % 4], 1.f + 0x1p-21f, -__uint_as_float(upper));
            }
        } else if constexpr (sizeof(T) == 2) {
            typedef T T2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                // (as many bits as fp16 has; infinite values: stray())
                float left[2];
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    left[j] = w[i / 4][i % 4 + j] - __uint_as_float(__float_as_uint(w[i / 4][i % 4 + j]) & 0xffffe000u);
                const T2 f = __builtin_bit_cast(T2, __builtin_amdgcn_cvt_pkrtz(w[i / 4][i % 4], w[i / 4][i % 4 + 1]));
                const T2 r = __builtin_bit_cast(T2, __builtin_amdgcn_cvt_pkrtz(left[0], left[1]));
                first[i] = f[0], first[i + 1] = f[1], second[i] = r[0], second[i + 1] = r[1];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) first[i] = w[i / 4][i % 4];
        }
    }
};

// tanh, to 1.7 units in the last place (the worst of all numbers from 1e-30 to 20, tried on
// an MI355X).  The exponential's form would lose digits below 0.6: there x (1 + x^2 P(x^2)), P a
// least-squares fit whose error is 2^-30 of the result.
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
    // sequence b's indices (of a share's first; those after it are read when it gets there: held
    // in lanes they would take registers from the whole of it)
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
    // the units before sequence b, of up to 64
    __device__ __forceinline__ unsigned before(int b) const { return b ? __builtin_amdgcn_readlane(end, b - 1) : 0; }
    // the sequence that has unit u < total, and the units before it
    __device__ __forceinline__ void find(unsigned u, int &b, unsigned &base) const
    {
        const int t = threadIdx.x;
        if (few) {
            b = __builtin_ctzll(__ballot(u < end));
            base = before(b);
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
    const float inv = l == 0.f ? 0.f : __builtin_amdgcn_rcpf(l);  // 0: a row that saw nothing
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

// ------------------------------------------------------------------ K and V in LDS

// The lane's number as the compiler cannot know it ahead: addresses made of it are made
// where they are used.  Left alone, they are made once before all loops and held in
// registers that the sums need.
__device__ __forceinline__ unsigned lane_here()
{
    unsigned lane = threadIdx.x % 64;
    asm volatile("" : "+v"(lane));
    return lane & 63;
}

// Rows of K or V in LDS as copies leave them: 1 KiB an instruction, 16 bytes a lane, so
// that a row's chunks of 16 bytes lie side by side.  Chunk c of row r is at place
// c ^ turn(r): sixteen rows' chunks of one column lie in all banks.
template <typename T, int D>
struct Lds {
    static constexpr int kElements = 16 / (int)sizeof(T);
    static constexpr int kChunks = D / kElements;  // of a row
    static constexpr int kRow = kChunks * 16;
    static constexpr int kRows = 64 / kChunks;  // of a copy

    static __device__ __forceinline__ unsigned turn(unsigned r) { return kChunks >= 16 ? r & 15 : r >> 1 & 7; }

    typedef __attribute__((address_space(3))) const char *At;
    static __device__ __forceinline__ unsigned address(const char *s) { return (unsigned)(uintptr_t)(At)s; }
    template <typename X>
    static __device__ __forceinline__ X load(unsigned at)
    {
        return *(__attribute__((address_space(3))) const X *)(uintptr_t)at;
    }

    // Operands for the product: channels 8 (4 c + lane / 16) on of rows lane % 16 and those + 16
    // of a tile at s.  A tile lies at a multiple of 1 KiB, so that another column's chunk is
    // another value of the address's bits within a row: one xor, one read.
    struct RowReader {
        unsigned base, g;
        __device__ __forceinline__ RowReader(const char *s, unsigned lane) : g(lane / 16)
        {
            const unsigned col = lane % 16;
            base = address(s) + col * kRow + (((sizeof(T) == 2 ? g : 2 * g) ^ turn(col)) << 4);
        }
        // chunks from `chunks` on are zero
        template <bool PART>
        __device__ __forceinline__ typename Eight<T>::V get(int h, int c, int chunks) const
        {
            typedef typename Eight<T>::V V;
            const unsigned i = 4 * c + g;
            if constexpr (sizeof(T) == 2) {
                const V v = load<V>((base ^ c << 6) + h * 16 * kRow);
                return PART && i >= (unsigned)chunks ? (V)(T)0.f : v;
            } else {
                const f32x4 lo = load<f32x4>((base ^ c << 7) + h * 16 * kRow), hi = load<f32x4>((base ^ c << 7 ^ 16) + h * 16 * kRow);
                return __builtin_shufflevector(PART && 2 * i >= (unsigned)chunks ? (f32x4)0.f : lo,
                                               PART && 2 * i + 1 >= (unsigned)chunks ? (f32x4)0.f : hi, 0, 1, 2, 3, 4, 5, 6, 7);
            }
        }
    };

    // channel 16 n + lane % 16 of rows 4 (lane / 16) + 0..3 and those + 16
    struct ColumnReader {
        unsigned base;
        __device__ __forceinline__ ColumnReader(const char *s, unsigned lane)
        {
            if constexpr (sizeof(T) == 2) {
                const unsigned r = lane / 4;
                base = address(s) + r * kRow + ((lane / 2 % 2 ^ turn(r)) << 4) + lane % 2 * 8;
            } else {
                const unsigned r = lane / 16 * 4;
                base = address(s) + r * kRow + ((lane / 4 % 4 ^ turn(r)) << 4) + lane % 4 * 4;
            }
        }
        // (of tile h)
        __device__ __forceinline__ typename Eight<T>::V get(int n, int h) const
        {
            typename Eight<T>::V v;
            if constexpr (sizeof(T) == 2) {
                typedef short S4 __attribute__((ext_vector_type(4)));
                typedef __attribute__((address_space(3))) S4 *P;
                const unsigned at = (base ^ n << 5) + h * kTile * kRow;
                const S4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)at);
                const S4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(at + 16 * kRow));
                const auto both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                v = __builtin_bit_cast(typename Eight<T>::V, both);
            } else {
                static_assert(kChunks >= 16, "turn(r + j) = turn(r) ^ j");
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned at = (base ^ n << 6 ^ j << 4) + j * kRow + h * kTile * kRow;
                    v[j] = load<float>(at);
                    v[4 + j] = load<float>(at + 16 * kRow);
                }
            }
            return v;
        }
    };

    static __device__ __forceinline__ float at(const char *s, int r, int channel)
    {
        const int byte = channel * (int)sizeof(T);
        return (float)*reinterpret_cast<const T *>(s + r * kRow + (byte / 16 ^ turn(r)) * 16 + byte % 16);
    }
};

// Each lane's 16 bytes at base + off to the wave's 1 KiB from `to` on.  Written out,
// because the compiler would wait for every such copy before the next read of LDS; the
// kernels wait for a tile's when they begin it.  m0, where `to` is passed, is read one
// wait state after it is set, scalar operands five after a vector instruction that
// may have made them.
__device__ __forceinline__ void copy16(char *to, const char *base, unsigned off)
{
    const unsigned at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void *)to;
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" : : "{m0}"(at), "v"(off), "s"(base) : "memory");
}

// fp16, whose least numbers are not far below 1.
template <typename T>
constexpr bool narrow = sizeof(T) == 2 && !__is_same(T, bf16);

// What one wave brings of an item's K and V into LDS: ROWS rows of a tile, from row
// `first` of it on (a multiple of 8).
//   COPIED   straight from memory: rows are whole chunks at multiples of 16 bytes, and a
//            copy's rows (up to 8) lie in one page;
//   else     through registers, chunk by chunk: any head size, alignment and page.
template <typename T, int D, int ROWS, bool COPIED>
struct Mover {
    typedef Lds<T, D> L;
    typedef typename Pack<T>::V V;
    static constexpr int kCopies = ROWS / L::kRows;
    static_assert(kCopies * L::kRows == ROWS, "whole copies");
    const Args &p;
    const char *key, *value;  // the head's
    const int32_t *table;
    int first, chunks;
    // COPIED: a lane's row in a copy, in bytes of K and of V, and its chunk in copies that turn nothing
    unsigned key_row, value_row, chunk;
    V in_k[COPIED ? 1 : kCopies], in_v[COPIED ? 1 : kCopies];

    __device__ __forceinline__ Mover(const Args &args, int first_row) : p(args), first(first_row)
    {
        const int lane = threadIdx.x % 64, r = lane / L::kChunks;
        chunks = (p.d + L::kElements - 1) / L::kElements;
        key_row = (unsigned)(r * (int)p.key_place * (int)sizeof(T));
        value_row = (unsigned)(r * (int)p.value_place * (int)sizeof(T));
        // turn(first + i kRows + r) = turn(first + r) ^ turn(i kRows): rows of a copy, of copies and
        // of the tile are different bits of what turn() takes
        chunk = lane % L::kChunks ^ L::turn(first + r);
    }
    __device__ __forceinline__ void head(int b, int h)
    {
        key = (const char *)((const T *)p.key + h * p.key_head);
        value = (const char *)((const T *)p.value + h * p.value_head);
        table = p.table + b * p.table_row;
    }
    // What the table has for position j < end, else -1.  It is looked at, by page(), a tile later:
    // here that would be waited for, and all copies that were begun before with it.
    __device__ __forceinline__ int entry_at(int j, int end) const
    {
        int entry = -1;
        if (j < end) entry = table[p.page_shift >= 0 ? j >> p.page_shift : (unsigned)j / (unsigned)p.page_size];
        return entry;
    }
    // the page, or -1
    __device__ __forceinline__ int page(int entry) const { return (unsigned)entry < (uint64_t)p.pages ? entry : -1; }
    // The rows of the tile at position `at`, whose pages are `page` (row lane % 32 of what
    // this wave moves, or lane % 64 of 64), on their way to s_k and s_v, both at the tile's row 0.
    __device__ __forceinline__ void begin(int at, int page, char *s_k, char *s_v)
    {
        const int lane = threadIdx.x % 64, j = at + first + lane % ROWS;
        const int place = p.page_shift >= 0 ? j & (p.page_size - 1) : (int)((unsigned)j % (unsigned)p.page_size);
        // (COPIED: strides in bytes have 32 bits, and so has the offset of a position in its page)
        const auto offset = [&](int64_t of_page, int64_t of_place) {
            if constexpr (COPIED)
                return (int64_t)((uint64_t)(unsigned)page * ((unsigned)of_page * (unsigned)sizeof(T)) +
                                 (unsigned)place * ((unsigned)of_place * (unsigned)sizeof(T)));
            else
                return (page * of_page + place * of_place) * (int)sizeof(T);
        };
        const int64_t k = offset(p.key_page, p.key_place), v = offset(p.value_page, p.value_place);
        if constexpr (COPIED) {
            auto from = [&](const char *start, int64_t off, int r) {
                const unsigned lo = __builtin_amdgcn_readlane((int)off, r), hi = __builtin_amdgcn_readlane((int)(off >> 32), r);
                return start + (int64_t)((uint64_t)hi << 32 | lo);
            };
            // (made here each time: a register for each copy's would be held through the loop)
            unsigned chunk_here = chunk;
            asm volatile("" : "+v"(chunk_here));
            const unsigned here = (unsigned)__ballot(page >= 0) & (unsigned)((1ull << ROWS) - 1);
            if (here == (unsigned)((1ull << ROWS) - 1) && p.d == D) {
                // all of K, then all of V
                auto side = [&](const char *head, int64_t off, unsigned row, unsigned step, char *to) {
                    const char *start = nullptr;
#pragma unroll
                    for (int i = 0; i < kCopies; ++i) {
                        // eight rows lie in one page
                        if (i * L::kRows % 8 == 0)
                            start = from(head, off, i * L::kRows);
                        else
                            start += step;
                        copy16(to + (first + i * L::kRows) * L::kRow, start, row + (chunk_here ^ L::turn(i * L::kRows)) * 16);
                    }
                };
                side(key, k, key_row, (unsigned)p.key_place * (unsigned)(L::kRows * sizeof(T)), s_k);
                side(value, v, value_row, (unsigned)p.value_place * (unsigned)(L::kRows * sizeof(T)), s_v);
            } else if (here) {
                // A sequence's end, or pages that are none: in the place of rows that hold nothing come
                // others that do, so that nothing but these is ever read: their weights are 0, and a
                // value that is no number is told by odd().  Chunks beyond the head's are left out.
                const int any = __builtin_ctz(here);
#pragma unroll 1
                for (int i = 0; i < 2 * kCopies; ++i) {
                    const bool is_key = i < kCopies;
                    const int r0 = (is_key ? i : i - kCopies) * L::kRows, from_row = here >> r0 & 1 ? r0 : any;
                    const unsigned c = chunk_here ^ L::turn(r0);
                    // rows of a copy lie in one page, those that hold something before the others
                    const bool holds = here >> (from_row + lane / L::kChunks) & 1;
                    const unsigned row = holds ? (is_key ? key_row : value_row) : 0;
                    const char *start = from(is_key ? key : value, is_key ? k : v, from_row);
                    if (c < (unsigned)chunks) copy16((is_key ? s_k : s_v) + (first + r0) * L::kRow, start, row + c * 16);
                }
            }
        } else {
            // A head's last chunk is read with the elements before it, which whole() shifts out when
            // they are there: element by element each load would be waited for (one sequence of
            // 30000 positions, 4 heads of 255 fp16: 57 us, 342 so).
            const auto each = [&](auto &&part) {
#pragma unroll
                for (int i = 0; i < kCopies; ++i) {
                    const int r = i * L::kRows + lane / L::kChunks, c = lane % L::kChunks;
                    const int64_t ok = (int64_t)((uint64_t)(unsigned)__shfl((int)(k >> 32), r) << 32 | (unsigned)__shfl((int)k, r));
                    const int64_t ov = (int64_t)((uint64_t)(unsigned)__shfl((int)(v >> 32), r) << 32 | (unsigned)__shfl((int)v, r));
                    const int n = __shfl(page, r) >= 0 ? p.d - c * L::kElements : 0;
                    in_k[i] = part((const T *)(key + ok) + c * L::kElements, n);
                    in_v[i] = part((const T *)(value + ov) + c * L::kElements, n);
                }
            };
            if (p.d >= L::kElements)
                each([&](const T *from, int n) {
                    V v = (V)(T)0.f;
                    if (n > 0) v = *reinterpret_cast<const typename Pack<T>::U *>(from - lack(n));
                    return v;
                });
            else
                each([](const T *from, int n) {
                    V v = (V)(T)0.f;
#pragma unroll
                    for (int j = 0; j < L::kElements; ++j)
                        if (j < n) v[j] = from[j];
                    return v;
                });
        }
    }
    // The elements that a head's last chunk lacks of a whole one (n are there), 0 for other chunks.
    __device__ __forceinline__ int lack(int n) const
    {
        return n > 0 && n < L::kElements && p.d >= L::kElements ? L::kElements - n : 0;
    }
    // zeros after a last chunk's elements
    static __device__ __forceinline__ V whole(V v, int lack)
    {
        typedef unsigned __int128 Bits;
        return __builtin_bit_cast(V, __builtin_bit_cast(Bits, v) >> (lack * 8 * (int)sizeof(T)));
    }
    // What begin() began is in LDS (of this wave); `there`: the rows that hold something.  Where
    // there are none nothing was begun, and V's become zeros: their weights are, but LDS may hold NaN.
    __device__ __forceinline__ void end(uint64_t there, char *s_k, char *s_v)
    {
        const int lane = threadIdx.x % 64;
        if constexpr (COPIED) {
            constexpr uint64_t all = (1ull << ROWS) - 1;
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            if (!(there & all)) {
                f32x4 *to = reinterpret_cast<f32x4 *>(s_v + first * L::kRow);
#pragma unroll 1
                for (unsigned i = lane_here(); i < ROWS * L::kChunks; i += 64) to[i] = (f32x4)0.f;
            }
        } else {
            if (p.d % L::kElements) {
                const int l = lack(p.d - lane % L::kChunks * L::kElements);
#pragma unroll
                for (int i = 0; i < kCopies; ++i) in_k[i] = whole(in_k[i], l), in_v[i] = whole(in_v[i], l);
            }
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                const int r = first + i * L::kRows + lane / L::kChunks, c = lane % L::kChunks ^ L::turn(r);
                *reinterpret_cast<V *>(s_k + r * L::kRow + c * 16) = in_k[i];
                *reinterpret_cast<V *>(s_v + r * L::kRow + c * 16) = in_v[i];
            }
        }
    }
    // whether its rows of V, from row `from` of them on, have a NaN or an infinity
    __device__ __forceinline__ bool odd(const char *s_v, int from) const
    {
        bool odd = false;
#pragma unroll 1
        for (unsigned i = (from < 0 ? 0 : from) * L::kChunks + lane_here(); i < ROWS * L::kChunks; i += 64) {
            const unsigned r = first + i / L::kChunks, c = i % L::kChunks ^ L::turn(r);
            const V v = *reinterpret_cast<const V *>(s_v + r * L::kRow + i % L::kChunks * 16);
#pragma unroll
            for (int j = 0; j < L::kElements; ++j) odd |= c < (unsigned)chunks && !(fabsf((float)v[j]) < __builtin_inff());
        }
        return __any(odd);
    }
};

// A wave's stores to LDS are seen by its loads after this
__device__ __forceinline__ void own_lds()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ------------------------------------------------------------------ the attention

__device__ __forceinline__ bool finite(float v) { return fabsf(v) < __builtin_inff(); }

// Whether a sum of values is infinite or no number.  An infinite value times a weight that fp16 does not
// hold makes that of what is infinite: where there are such sums a part is gone through again, carefully,
// with weights of 32 bits for all values that are no finite numbers.
__device__ __forceinline__ bool stray(f32x4 sum) { return !(sum[0] * 0.f + sum[1] * 0.f + sum[2] * 0.f + sum[3] * 0.f == 0.f); }

// The larger of v in lanes 16 and 32 apart, in all of them.
__device__ __forceinline__ float across(float v)
{
    // a swap of the odd rows of sixteen of the one with the even ones of the other, both v, leaves
    // each row beside its neighbour; then the same of halves
    const unsigned u = __float_as_uint(v);
    const auto rows = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = fmaxf(__uint_as_float(rows[0]), __uint_as_float(rows[1]));
    const unsigned w = __float_as_uint(v);
    const auto halves = __builtin_amdgcn_permlane32_swap(w, w, false, false);
    return fmaxf(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
}

// 16 NQ rows of an item, a wave's: lane l has row l % 16 of each sixteen.
template <typename T, int D, int NQ>
struct Rows {
    typedef typename Eight<T>::V V8;
    typedef Lds<T, D> L;
    static constexpr int C = D / 32, N = D / 16;
    static constexpr int kGroup = sizeof(T) == 2 ? 8 : 4;  // operands read from LDS at once: 32 registers
    // Weights are exp2(score - origin + kLift).  bf16 holds them however small they are.  fp16 ends at
    // 2^-24, and many positions that each have less than that beside one far above them may hold a
    // share of the row together (one 17.5 above 2^17 others: 0.3 %).  So in fp16 weights go up to
    // 2^15, and a tile whose largest would have less than 2^(kLift - kFall) moves the origin down to
    // it: the sums' 32 bits have room for what they then hold, for kSpan powers of two from the
    // highest origin on.
    static constexpr bool kNarrow = narrow<T>;
    static constexpr float kLift = kNarrow ? 8.f : 0.f, kRise = kNarrow ? 7.f : 8.f, kFall = 8.f, kSpan = 60.f;
    V8 q[NQ][C];
    uint64_t word[NQ];  // the sequence's tokens that a row sees
    f32x4 o[NQ][N];     // sums of values: channels 16 i + 4 (l / 16) + 0..3
    float l[NQ];        // sums of exponentials: of this lane's positions
    float m[NQ];        // their origin, in the products' units
    float highest[kNarrow ? NQ : 1];  // the highest that it had

    // Sixteens of rows from row0 on, `step` rows from one to the next; those from `rows` on are
    // the last one again, and are not stored.  WHOLE: rows are whole chunks of 16 bytes.
    template <bool WHOLE>
    __device__ __forceinline__ void load(const Args &p, const Sequence &seq, int head, int row0, int step, int rows, int chunks)
    {
        const int lane = threadIdx.x % 64, col = lane % 16, g = lane / 16;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int r = row0 + n * step + col;
            const RowAt row = row_at(p, seq, head, r < rows ? r : rows - 1);
            const T *from = (const T *)p.q + row.m * p.q_token + row.h * p.q_head;
            word[n] = p.mask ? p.mask[row.m] : ~0ull >> (63 - (int)(row.m - seq.first));
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if constexpr (!WHOLE) {
                    q[n][c] = get8(from + c * 32 + g * 8, p.d - c * 32 - g * 8);
                } else {
                    constexpr int E = L::kElements;
                    typename Pack<T>::V part[8 / E];
#pragma unroll
                    for (int h = 0; h < 8 / E; ++h) {
                        const int i = (c * 4 + g) * (8 / E) + h;
                        part[h] = *reinterpret_cast<const typename Pack<T>::U *>(from + (i < chunks ? i : 0) * E);
                        if (p.d != D && i >= chunks) part[h] = (typename Pack<T>::V)(T)0.f;
                    }
                    if constexpr (E == 8)
                        q[n][c] = part[0];
                    else
                        q[n][c] = __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
                }
            }
        }
        if (p.sign == 1.f) return;
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) q[n][c][j] = (T)((float)q[n][c][j] * p.sign);
    }

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            m[n] = -__builtin_inff();
            if constexpr (kNarrow) highest[n] = m[n];
            l[n] = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) o[n][i] = (f32x4)0.f;
        }
    }

    // What the sums of row n are relative to, in powers of two.
    __device__ __forceinline__ float origin(const Args &p, int n) const { return m[n] * (p.cap != 0.f ? 1.f : p.scale) - kLift; }

    // Whether a tile whose largest score is `most` moves the origin of row n down to it.
    __device__ __forceinline__ bool falls(int n, float most, float scale) const
    {
        if constexpr (kNarrow) return (m[n] - most) * scale > kFall && (highest[n] - most) * scale <= kSpan;
        return false;
    }

    // H tiles of 32 positions, from position `at` on; `there`: the positions that hold something;
    // `odd`: values among them that are no numbers, some of which a row may not see; `scratch`: 2 KiB
    // of LDS.
    template <int H>
    __device__ __forceinline__ void step(const Args &p, const char *s_k, const char *s_v, int at, int length, uint64_t there,
                                         bool odd, int chunks, float *scratch)
    {
        constexpr uint64_t ALL = H == 2 ? ~0ull : 0xffffffffull;
        constexpr int kHalf = kTile * L::kRow;
        const unsigned lane = lane_here(), col = lane % 16, g = lane / 16;
        // x[n][2 h + i]: positions 32 h + 16 i + 4 g + 0..3 of row 16 n + col
        f32x4 x[NQ][2 * H];
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int h = 0; h < 2 * H; ++h) x[n][h] = (f32x4)0.f;
        // (reads in groups before their products: one by one each product would wait for its own.)
        // fp32's 32 channels are summed by themselves and added, since 256 in a row round up to
        // three times as far off as a plain product's sums: 500 positions of 256 channels 3.2e-7
        // from 64 bits, 1.6e-6 in one sum, for 2 to 6 % of large calls' time.
        const typename L::RowReader row(s_k, lane);
        auto scores = [&]<bool PART>() {
            constexpr int G = C < kGroup / 2 ? C : kGroup / 2;
#pragma unroll
            for (int h = 0; h < 2 * H; h += 2)
#pragma unroll
                for (int from = 0; from < C; from += G) {
                    V8 k[G][2];
#pragma unroll
                    for (int c = 0; c < G; ++c)
#pragma unroll
                        for (int i = 0; i < 2; ++i) k[c][i] = row.template get<PART>(h + i, from + c, chunks);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int c = 0; c < G; ++c) {
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int n = 0; n < NQ; ++n) {
                                if constexpr (sizeof(T) == 2)
                                    x[n][h + i] = product(k[c][i], q[n][from + c], x[n][h + i]);
                                else
                                    x[n][h + i] += product(k[c][i], q[n][from + c], (f32x4)0.f);
                            }
                        if constexpr (sizeof(T) == 4) __builtin_amdgcn_sched_barrier(0);
                    }
                }
        };
        if (p.d == D)
            scores.template operator()<false>();
        else
            scores.template operator()<true>();
        // the first columns of V on their way while the weights are made
        // (4 at once where a wave has 32 rows: 8 would spill registers)
        constexpr int G = NQ == 2 || N < kGroup ? 4 : kGroup;
        V8 v[G];
        const typename L::ColumnReader column(s_v, lane);
#pragma unroll
        for (int i = 0; i < G; ++i) v[i] = column.get(i, 0);
        __builtin_amdgcn_sched_barrier(0);

        const bool drafted = at + H * kTile > length;
        float scale = p.scale;
        if (p.cap != 0.f) {
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 8 * H; ++e) {
                    x[n][e / 4][e % 4] = tanh_of(x[n][e / 4][e % 4] * scale) * p.cap;
                    if (e % 2) __builtin_amdgcn_sched_barrier(0);
                }
            scale = 1.f;
        }
        // the positions of these that row 16 n + col sees
        auto seen = [&](int n) {
            uint64_t s = there;
            if (drafted) {
                const int off = length - at;  // the first token
                s &= off > 0 ? word[n] << off | ((1ull << off) - 1) : -off < 64 ? word[n] >> -off : 0ull;
            }
            return s;
        };
        if (drafted || there != ALL) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                const uint64_t s = seen(n) >> (g * 4);
#pragma unroll
                for (int e = 0; e < 8 * H; ++e)
                    if (!(s >> (e / 4 * 16 + e % 4) & 1)) x[n][e / 4][e % 4] = -__builtin_inff();
            }
        }
        float most[NQ];
        bool move = false;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            most[n] = x[n][0][0];
#pragma unroll
            for (int e = 1; e + 1 < 8 * H; e += 2)
                most[n] = fmaxf(fmaxf(most[n], x[n][e / 4][e % 4]), x[n][(e + 1) / 4][(e + 1) % 4]);
            most[n] = across(fmaxf(most[n], x[n][2 * H - 1][3]));
            // (both -infinity: nothing seen yet)
            move |= (most[n] - m[n]) * scale > kRise || falls(n, most[n], scale);
        }
        // the sums' origins move only where a weight would pass 2^(kLift + kRise), or all be too small:
        // nearly no tile has them multiplied
        if (__any(move)) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                const float top = falls(n, most[n], scale) ? most[n] : fmaxf(most[n], m[n]);
                if constexpr (kNarrow) highest[n] = fmaxf(highest[n], top);
                const float shrink = m[n] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f((m[n] - top) * scale);
                m[n] = top;
                l[n] *= shrink;
#pragma unroll
                for (int i = 0; i < N; ++i) o[n][i] *= shrink;
            }
        }
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const float from = m[n] == -__builtin_inff() ? 0.f : kLift - m[n] * scale;
#pragma unroll
            for (int e = 0; e < 8 * H; ++e) {
                const float w = __builtin_amdgcn_exp2f(fmaf(x[n][e / 4][e % 4], scale, from));
                l[n] += w;
                x[n][e / 4][e % 4] = w;
            }
        }
#pragma unroll
        for (int h = 0; h < H; ++h) {
            Weights<T> weight[NQ];
#pragma unroll
            for (int n = 0; n < NQ; ++n) weight[n].set({x[n][2 * h], x[n][2 * h + 1]});
#pragma unroll
            for (int from = 0; from < N; from += G) {
                if (h || from) {
#pragma unroll
                    for (int i = 0; i < G; ++i) v[i] = column.get(from + i, h);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (odd) {
#pragma unroll
                    for (int i = 0; i < G; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[i][j] = finite((float)v[i][j]) ? v[i][j] : (T)0.f;
                }
#pragma unroll
                for (int i = 0; i < G; ++i)
#pragma unroll
                    for (int n = 0; n < NQ; ++n) o[n][from + i] = product(v[i], weight[n].first, o[n][from + i]);
                if constexpr (sizeof(T) == 2) {
#pragma unroll
                    for (int i = 0; i < G; ++i)
#pragma unroll
                        for (int n = 0; n < NQ; ++n) o[n][from + i] = product(v[i], weight[n].second, o[n][from + i]);
                }
            }
        }
        if (!odd) return;
        // a NaN or an infinity reaches the rows that see it and no other: the products were made
        // with zeros in their places, and here what they add is added position by position
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int h = 0; h < H; ++h) {
                own_lds();
#pragma unroll
                for (int e = 0; e < 8; ++e) scratch[(e / 4 * 16 + g * 4 + e % 4) * 16 + col] = x[n][2 * h + e / 4][e % 4];
                own_lds();
                const unsigned s = (unsigned)(seen(n) >> (h * kTile));
#pragma unroll 1
                for (int j = 0; j < kTile; ++j) {
                    const float w = scratch[j * 16 + col];
                    const bool sees = s >> j & 1;
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const unsigned here = lane_here() / 16 * 4;
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const float one = L::at(s_v + h * kHalf, j, i * 16 + here + c);
                            if (sees && !finite(one)) o[n][i][c] += w * one;
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
    }
};

// What a work-group has of the line, part by part.
struct Walk {
    unsigned rank, share_begin, share_end;
    int b;
    unsigned base;  // units before sequence b
    Sequence seq;
    // the part at hand
    unsigned item_begin, part_begin, part_end;
    int head, row0, rows;  // of the item: its first row among its head's, and how many it has
    int begin, end;        // positions
    bool whole;

    // from unit u on
    __device__ __forceinline__ void at(const Args &p, unsigned u)
    {
        while (u >= base + seq.cost(p.shape.heads)) {
            base += seq.cost(p.shape.heads);
            seq = sequence_of(p, ++b);
        }
        const unsigned item = (u - base) / (unsigned)seq.units;
        item_begin = base + item * seq.units;
        part_begin = u;
        part_end = item_begin + seq.units < share_end ? item_begin + seq.units : share_end;
        const int most = 1 << p.shape.rows_shift;
        head = (int)(item / (unsigned)seq.groups);
        row0 = (int)(item % (unsigned)seq.groups) * most;
        rows = seq.tokens * p.shape.group - row0 < most ? seq.tokens * p.shape.group - row0 : most;
        begin = p.shape.unit_shift < 0 ? 0 : (int)(part_begin - item_begin) << p.shape.unit_shift;
        end = part_end == item_begin + seq.units ? seq.keys : (int)(part_end - item_begin) << p.shape.unit_shift;
        whole = part_begin == item_begin && part_end == item_begin + seq.units;
    }
};

#define PK_WALK(THREADS)                                                                                       \
    const Line<THREADS> line(p, s_line);                                                                       \
    const unsigned total = line.total, each = share(total, gridDim.x), active = (total + each - 1) / each;     \
    if (blockIdx.x >= active) return;                                                                          \
    Walk walk;                                                                                                 \
    walk.rank = rank_of(blockIdx.x, active);                                                                   \
    walk.share_begin = walk.rank * each;                                                                       \
    walk.share_end = walk.share_begin + each < total ? walk.share_begin + each : total;                        \
    line.find(walk.share_begin, walk.b, walk.base);                                                            \
    walk.seq = line.get(walk.b)

// Few rows: the waves divide the positions.  Each has its own tiles, with two STAGES one
// on its way while the one before is worked on, and nothing waits for another wave until
// their sums are joined.  One stage leaves room for twice the work-groups on a CU: for
// calls in which each of them has a tile or two a wave (3 sequences of 5000 positions, 4
// heads of 64 fp32: 17.0 us in all, 2.5 less than with two; one token over 4096 positions,
// 8 heads of 128 bf16: 11.9 us and 5.0 to join under the profiler, 16.2 in all without).
template <typename T, int D, int NQ, int WAVES, bool COPIED, int STAGES>
__global__ void __launch_bounds__(WAVES * 64) stream_kernel(Args p)
{
    typedef Lds<T, D> L;
    constexpr int N = D / 16, ROWS = 16 * NQ, THREADS = WAVES * 64, STEP = WAVES * kTile;
    constexpr int kHalf = kTile * L::kRow, kWave = STAGES * 2 * kHalf;
    constexpr bool kAhead = !COPIED || STAGES == 2;  // the next tile is begun before this one is worked on
    static_assert(COPIED || STAGES == 1, "what is not copied waits in registers");
    constexpr int kSum = ROWS * (D + 4) * 4, kOwn = kWave > kSum ? kWave : (kSum + 1023) / 1024 * 1024;
    __shared__ __align__(1024) char s_raw[WAVES * kOwn];
    static_assert(kHalf % 1024 == 0 && kOwn % 1024 == 0, "tiles lie at multiples of 1 KiB");
    __shared__ typename Line<THREADS>::Shared s_line;
    __shared__ float s_m[WAVES][ROWS], s_l[WAVES][ROWS], s_scratch[WAVES][kTile * 16];
    __shared__ int s_strays[WAVES];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, g = lane / 16;
    char *const s_own = s_raw + wave * kOwn;
    Mover<T, D, kTile, COPIED> mover(p, 0);
    PK_WALK(THREADS);
    Rows<T, D, NQ> rows;

    bool careful = false;
    for (unsigned u = walk.share_begin; u < walk.share_end;) {
        walk.at(p, u);
        mover.head(walk.b, walk.head);
        const int end = walk.end, length = walk.seq.length;
        // the first turn only brings the first tile: what brings a tile is here once
        int at = walk.begin + (wave - WAVES) * kTile, stage = 0;
        int page = -1, next = mover.entry_at(at + STEP + lane % kTile, end);
        // (a second time what it has: `out` may be q's memory)
        if (!careful) rows.template load<COPIED>(p, walk.seq, walk.head, walk.row0, 16, walk.row0 + walk.rows, mover.chunks);
        rows.clear();
        for (bool first = true; at < end; at += STEP, first = false) {
            char *const s_k = s_own + stage * 2 * kHalf;
            const unsigned there = (unsigned)__ballot(page >= 0);
            if (!first) mover.end(there, s_k, s_k + kHalf);
            if (STAGES == 2) stage ^= 1;
            next = mover.page(next);
            char *const s_next = s_own + stage * 2 * kHalf;
            if (kAhead && at + STEP < end) mover.begin(at + STEP, next, s_next, s_next + kHalf);
            page = next;
            next = mover.entry_at(at + 2 * STEP + lane % kTile, end);
            if (!first) {
                own_lds();
                bool odd = false;
                if (careful || at + kTile > length || there != ~0u)
                    odd = mover.odd(s_k + kHalf, there == ~0u && !careful ? length - at : 0);
                rows.template step<1>(p, s_k, s_k + kHalf, at, length, there, odd, mover.chunks, s_scratch[wave]);
            }
            if (!kAhead && at + STEP < end) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this one has been read
                mover.begin(at + STEP, page, s_next, s_next + kHalf);
            }
        }

        // the waves' sums together
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        float *s_o = reinterpret_cast<float *>(s_own);
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float l = rows.l[n] + __shfl_xor(rows.l[n], 16);
            l += __shfl_xor(l, 32);
            if (g == 0) {
                s_m[wave][n * 16 + col] = rows.origin(p, n);
                s_l[wave][n * 16 + col] = l;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) *reinterpret_cast<f32x4 *>(s_o + (n * 16 + col) * (D + 4) + i * 16 + g * 4) = rows.o[n][i];
        }
        __syncthreads();
        bool strays = false;
        float *part = walk.whole ? nullptr : part_of<D>(p, walk.rank, slot_of(walk.part_begin, walk.share_begin));
        for (int i = threadIdx.x; i < walk.rows * (D / 4); i += THREADS) {
            const int r = i / (D / 4), c = i % (D / 4) * 4;
            float most = s_m[0][r];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) most = fmaxf(most, s_m[w][r]);
            f32x4 sum = (f32x4)0.f;
            float all = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = weight_of(s_m[w][r], most);
                sum += *reinterpret_cast<const f32x4 *>(s_raw + w * kOwn + (r * (D + 4) + c) * 4) * f;
                all += s_l[w][r] * f;
            }
            if constexpr (narrow<T>) strays |= c < p.d && stray(sum);
            if (walk.whole) {
                if (c < p.d) finish<T>(p, walk.seq, walk.head, walk.row0 + r, c, sum, all, most);
            } else {
                *reinterpret_cast<f32x4 *>(part + r * D + c) = sum;
                if (c == 0) {
                    part[ROWS * D + r] = most;
                    part[ROWS * (D + 1) + r] = all;
                }
            }
        }
        if constexpr (narrow<T>) {
            strays = __any(strays);
            if (lane == 0) s_strays[wave] = strays;
        }
        __syncthreads();
        if constexpr (narrow<T>) {
            // (waves write here again behind the next barrier)
            int any = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) any |= s_strays[w];
            careful = !careful && __builtin_amdgcn_readfirstlane(any);  // (a scalar, as the walk is)
        }
        if (!careful) u = walk.part_end;
    }
}

// Many rows: a wave has 16 NQ of them, and the work-group's waves share its tiles of K
// and V, of which each brings a fourth.  One barrier a tile: the one on its way goes
// where the one before the last was read.
// 16 trees of 16 tokens over 16384 positions, 8 heads of 128 bf16 with 4 query heads each:
// 681 MB in 139 us (4.9 TB/s).  4 trees of 64 over up to 32768 with 8 query heads: 223 us, 98
// Gflop (V's products, made twice, counted once), matrix cores busy 30 %: the rest is the softmax's
// arithmetic and waits; and row groups of one head at different places of their sequence read K
// and V past L2 each (1.03 GB; lengths that divide evenly reach 665 Tflop/s).  Copies of the
// next tile begun between the products spilled (440 us, when the whole took 200).
template <typename T, int D>
constexpr int wide_tile() { return D * (int)sizeof(T) <= 256 ? 64 : 32; }

template <typename T, int D, int NQ, bool COPIED>
__global__ void __launch_bounds__(256, D * sizeof(T) <= 512 ? 2 : 1) wide_kernel(Args p)
{
    typedef Lds<T, D> L;
    constexpr int N = D / 16, ROWS = 64 * NQ, TILE = wide_tile<T, D>(), OWN = TILE / 4, kHalf = TILE * L::kRow;
    __shared__ __align__(1024) char s_raw[4 * kHalf];
    __shared__ typename Line<256>::Shared s_line;
    static_assert(ROWS * D * 4 <= 4 * kHalf, "the sums fit the stages");
    __shared__ float s_scratch[4][kTile * 16], s_m[ROWS], s_l[ROWS];
    __shared__ int s_odd[2][4], s_strays[4];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 16, g = lane / 16;
    Mover<T, D, OWN, COPIED> mover(p, wave * OWN);
    PK_WALK(256);
    Rows<T, D, NQ> rows;

    bool careful = false;
    for (unsigned u = walk.share_begin; u < walk.share_end;) {
        walk.at(p, u);
        mover.head(walk.b, walk.head);
        const int end = walk.end, length = walk.seq.length, row0 = wave * 16;
        int at = walk.begin - TILE, stage = 0;
        int page = -1, next = mover.entry_at(at + TILE + lane % TILE, end);
        const int sixteens = row0 >= walk.rows ? 0 : NQ == 2 && row0 + 64 < walk.rows ? 2 : 1;
        const bool mine = sixteens > 0;
        // (a second time what it has: `out` may be q's memory)
        if (!careful) rows.template load<COPIED>(p, walk.seq, walk.head, walk.row0 + row0, 64, walk.row0 + walk.rows, mover.chunks);
        rows.clear();
        for (bool first = true; at < end; at += TILE, first = false) {
            char *const s_k = s_raw + stage * 2 * kHalf, *const s_v = s_k + kHalf;
            const uint64_t there = __ballot(page >= 0) & (TILE == 64 ? ~0ull : 0xffffffffull);
            const bool whole = there == (TILE == 64 ? ~0ull : 0xffffffffull) && !careful;
            const bool some = at + TILE > length || !whole;  // that not all rows see
            if (!first) {
                mover.end(there >> wave * OWN, s_k, s_v);
                if (some) {
                    own_lds();
                    const bool odd = mover.odd(s_v, whole ? length - at - wave * OWN : 0);
                    if (lane == 0) s_odd[stage][wave] = odd;
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
            }
            const int now = stage;
            stage ^= 1;
            next = mover.page(next);
            char *const s_next = s_raw + stage * 2 * kHalf;
            if (at + TILE < end) mover.begin(at + TILE, __shfl(next, wave * OWN + lane % OWN), s_next, s_next + kHalf);
            page = next;
            next = mover.entry_at(at + 2 * TILE + lane % TILE, end);
            if (first || !mine) continue;
            bool odd = false;
            if (some) odd = s_odd[now][0] | s_odd[now][1] | s_odd[now][2] | s_odd[now][3];
            rows.template step<TILE / kTile>(p, s_k, s_v, at, length, there, odd, mover.chunks, s_scratch[wave]);
        }

        // each wave's sums through LDS, where the tiles were, so that what stores them is here once
        __syncthreads();  // the last tile has been read
        bool strays = false;
        if (mine) {
            f32x4 *const s_o = reinterpret_cast<f32x4 *>(s_raw);
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                const int r = row0 + n * 64 + col;
                float l = rows.l[n] + __shfl_xor(rows.l[n], 16);
                l += __shfl_xor(l, 32);
                if (g == 0) {
                    s_m[r] = rows.origin(p, n);
                    s_l[r] = l;
                }
#pragma unroll
                for (int i = 0; i < N; ++i) s_o[r * (D / 4) + ((i * 4 + g) ^ col)] = rows.o[n][i];
            }
            own_lds();
            float *part = walk.whole ? nullptr : part_of<D>(p, walk.rank, slot_of(walk.part_begin, walk.share_begin));
            for (int i = lane; i < sixteens * 16 * (D / 4); i += 64) {
                const int c = i % (D / 4), r = row0 + i / (D / 4) / 16 * 64 + i / (D / 4) % 16;
                if (r >= walk.rows) break;
                const f32x4 o = s_o[r * (D / 4) + (c ^ (r & 15))];
                if constexpr (narrow<T>) strays |= c * 4 < p.d && stray(o);
                if (walk.whole) {
                    if (c * 4 < p.d) finish<T>(p, walk.seq, walk.head, walk.row0 + r, c * 4, o, s_l[r], s_m[r]);
                } else {
                    *reinterpret_cast<f32x4 *>(part + r * D + c * 4) = o;
                    if (c == 0) {
                        part[ROWS * D + r] = s_m[r];
                        part[ROWS * (D + 1) + r] = s_l[r];
                    }
                }
            }
        }
        if constexpr (narrow<T>) {
            strays = __any(strays);
            if (lane == 0) s_strays[wave] = strays;
        }
        __syncthreads();  // and the sums
        if constexpr (narrow<T>)
            careful = !careful && __builtin_amdgcn_readfirstlane(s_strays[0] | s_strays[1] | s_strays[2] | s_strays[3]);
        if (!careful) u = walk.part_end;
    }
}

// Joins the parts of items that more than one work-group had.  A work-group for each
// border between shares (the first border in an item does it), or for each item where
// these are fewer and sequences are lanes' (work-groups without anything to join take
// their time too: 4 trees of 64 tokens, 4 heads of 256: 43 us in all, 50 by borders, with 3 us
// less for the first launch than now).  Its
// lanes take four channels of a row each, and where there are fewer of them than lanes,
// the parts in turn: many parts (a long sequence alone) would else be read one after the
// other.  Items of many rows have a work-group for each `some` of them (the same trees by
// borders: 50 us with 16, 56 with 32).  Sums are made in an order that the call's sizes
// alone decide.
template <typename T, int D, int THREADS>
__global__ void __launch_bounds__(THREADS) join_kernel(Args p, unsigned groups, int some, bool by_item)
{
    __shared__ typename Line<THREADS>::Shared s_line;
    __shared__ float s_sum[THREADS][7];  // a maximum, a sum of exponentials, four of values; odd, for the banks
    const Line<THREADS> line(p, s_line);
    const unsigned total = line.total, each = share(total, groups);
    const int most_rows = 1 << p.shape.rows_shift;
    int b, head, group = 0, from_row;
    unsigned base;
    Sequence seq;
    if (by_item) {
        b = blockIdx.z;
        head = blockIdx.y;
        unsigned chunk = blockIdx.x;
        if (THREADS == 512) {  // (few rows are one group)
            const unsigned most_groups = (unsigned)(p.shape.most * p.shape.group + most_rows - 1) >> p.shape.rows_shift;
            group = (int)(chunk % most_groups);
            chunk /= most_groups;
        }
        from_row = (int)chunk * some;
        base = line.before(b);
        seq = line.get(b);
        if (group >= seq.groups) return;
    } else {
        const unsigned border = (blockIdx.x + 1) * each;
        if (border >= total) return;
        line.find(border, b, base);
        seq = line.get(b);
        const unsigned item = (border - base) / (unsigned)seq.units;
        head = (int)(item / (unsigned)seq.groups);
        group = (int)(item % (unsigned)seq.groups);
        from_row = blockIdx.y * some;
    }
    const unsigned begin = base + (unsigned)(head * seq.groups + group) * seq.units, end = begin + seq.units, first = begin / each;
    // nothing to join, or an earlier border's
    if ((end - 1) / each == first || (!by_item && first != blockIdx.x)) return;
    const int row0 = group * most_rows;
    const int rows = seq.tokens * p.shape.group - row0 < most_rows ? seq.tokens * p.shape.group - row0 : most_rows;
    if (from_row >= rows) return;
    const int count = rows - from_row < some ? rows - from_row : some;
    const unsigned parts = (end - 1) / each - first + 1;
    auto part = [&](unsigned i) {
        const unsigned from = (first + i) * each;
        return part_of<D>(p, first + i, slot_of(i ? from : begin, from));
    };
    // lanes to a part's sums: a power of two (with turns, one round: all elements have a lane)
    int lanes = D / 4;
    while (lanes < count * (D / 4) && lanes < THREADS) lanes *= 2;
    const int turns = THREADS / lanes, turn = threadIdx.x / lanes;
    for (int i = threadIdx.x % lanes; i - (int)(threadIdx.x % lanes) < count * (D / 4); i += lanes) {
        const int r = from_row + i / (D / 4), c = i % (D / 4) * 4;
        const bool on = i < count * (D / 4);
        float most = -__builtin_inff(), all = 0.f;
        f32x4 sum = (f32x4)0.f;
        auto add = [&](float m, float l, f32x4 o) {
            const float top = fmaxf(most, m), f = weight_of(most, top), h = weight_of(m, top);
            all = all * f + l * h;
            sum = sum * f + o * h;
            most = top;
        };
        if (on) {
            constexpr int AT_ONCE = THREADS == 1024 ? 4 : 8;  // (registers)
            for (unsigned w = turn; w < parts; w += turns * AT_ONCE) {
                float m[AT_ONCE], l[AT_ONCE];
                f32x4 o[AT_ONCE];
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i) {
                    // beyond the last part: its own place again, with no weight
                    const unsigned at = w + i * turns;
                    const float *from = part(at < parts ? at : w);
                    m[i] = from[D * most_rows + r];
                    l[i] = from[(D + 1) * most_rows + r];
                    o[i] = *reinterpret_cast<const f32x4 *>(from + r * D + c);
                }
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i)
                    if (w + i * turns < parts) add(m[i], l[i], o[i]);
            }
        }
        if (turns > 1) {
            float *mine = s_sum[threadIdx.x];
            mine[0] = most;
            mine[1] = all;
#pragma unroll
            for (int j = 0; j < 4; ++j) mine[2 + j] = sum[j];
            __syncthreads();
            if (turn == 0) {
                // their largest first, so that no turn's sum waits for another's
#pragma unroll 4
                for (int t = 1; t < turns; ++t) most = fmaxf(most, s_sum[threadIdx.x + t * lanes][0]);
                float f = weight_of(mine[0], most);
                all *= f;
                sum *= f;
#pragma unroll 4
                for (int t = 1; t < turns; ++t) {
                    const float *other = s_sum[threadIdx.x + t * lanes];
                    f = weight_of(other[0], most);
                    all = fmaf(other[1], f, all);
                    sum += f32x4{other[2], other[3], other[4], other[5]} * f;
                }
            }
        }
        if (turn == 0 && on && c < p.d) finish<T>(p, seq, head, row0 + r, c, sum, all, most);
    }
}

// ------------------------------------------------------------------ launches

// Channels that a head takes in registers and LDS.  Heads of other sizes do the products of the
// zeros beside them, and their rows are copied by a loop, not by a run of instructions: the 16 trees
// of wide_kernel's comment, all of 16384 positions, take 119 us with 64 channels, 219 with 80, 218
// with 128, its 4 trees, all of 32768, 292, 532 and 414.  Each size more would be 30 instances of
// these kernels.
int padded(int64_t d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

struct Form {
    int D, nq;
    bool wide, single;           // single: stream_kernel with one stage
    int rows;                    // of an item, at most
    int rows_shift, unit_shift;  // of an item; of a unit: what a work-group's waves have in work
    // Work-groups: what the LDS of most forms that copy lets the card hold at once.  Of the others
    // (16-bit heads of up to 64 channels with one stage, three a CU; through registers, one or two) the
    // last begin when the first have ended.
    int64_t groups;
    int64_t items;
    bool spare;    // no more units than work-groups
    size_t bytes;  // of the workspace
};

// Waves of stream_kernel: what a CU's LDS holds of their stages.
constexpr int stream_waves(int row_bytes) { return row_bytes >= 1024 ? 1 : row_bytes >= 512 ? 2 : 4; }

// The form of a call.  Up to 32 rows (16 of the widest heads) a wave has all of them, and
// the waves divide the positions; more are divided over the waves.
Form form_of(int size, int64_t d, int64_t group, int64_t heads, int64_t B, int64_t capacity, int64_t most)
{
    Form f;
    f.D = padded(d);
    const int64_t rows = most * group;
    const int row_bytes = f.D * size;
    f.wide = rows > (f.D == 256 ? 16 : 32);
    f.nq = f.D < 256 && rows > (f.wide ? 64 : 16) ? 2 : 1;
    f.rows_shift = (f.wide ? 6 : 4) + (f.nq == 2);
    f.rows = rows < 1 << f.rows_shift ? (int)rows : 1 << f.rows_shift;
    const int unit = f.wide ? 128 : stream_waves(row_bytes) * kTile;
    f.unit_shift = unit == 128 ? 7 : unit == 64 ? 6 : 5;
    f.items = B * heads * ((rows + (1 << f.rows_shift) - 1) >> f.rows_shift);
    const int64_t units = capacity <= unit ? 1 : (capacity + unit - 1) / unit;
    // A few units are sooner done one after the other than joined by a second launch (32
    // sequences of 400 positions, 8 heads of 128 bf16: 17.7 us, 24.5 divided; 1 of 250: 10.6 and
    // 12.6; with four of 32 bits 1 of 250 takes 22.7, 16.8 divided).
    const bool divided = units > (f.wide ? 1 : size == 2 ? 4 : 2) && f.items <= kMostLine / units;
    const int64_t line = divided ? f.items * units : f.items;
    f.groups = 256 * (f.wide ? (row_bytes <= 512 ? 2 : 1) : row_bytes <= 128 ? 2 : 1);
    f.single = !f.wide && (divided ? line <= 4 * f.groups : units == 1);
    if (f.single) f.groups *= 2;
    f.spare = line <= f.groups;
    if (f.spare) f.groups = line;
    f.bytes = !divided ? 0 : ((size_t)f.groups * 2 * (f.D + 2) << f.rows_shift) * sizeof(float);
    return f;
}

template <typename T, int D, int NQ, bool COPIED>
int launch(const Args &a, const Form &f, bool joined, hipStream_t s)
{
    if (f.wide) {
        hipLaunchKernelGGL((wide_kernel<T, D, NQ, COPIED>), dim3((unsigned)f.groups), dim3(256), 0, s, a);
    } else {
        constexpr int WAVES = stream_waves(D * (int)sizeof(T));
        if (f.single || !COPIED)
            hipLaunchKernelGGL((stream_kernel<T, D, NQ, WAVES, COPIED, 1>), dim3((unsigned)f.groups), dim3(WAVES * 64), 0, s, a);
        else if constexpr (COPIED)
            hipLaunchKernelGGL((stream_kernel<T, D, NQ, WAVES, COPIED, 2>), dim3((unsigned)f.groups), dim3(WAVES * 64), 0, s, a);
    }
    if (hipGetLastError() != hipSuccess) return PK_ERR_LAUNCH;
    if (!joined || f.groups == 1) return PK_OK;
    const bool by_item = a.B <= 64 && a.shape.heads <= 65535 && f.items < f.groups;
    // Rows of a work-group: of few items fewer, down to what gives a row's parts 16 turns of
    // lanes (one tree of 16 tokens over 30000 positions, 1 head with 8 query heads: 27 us in
    // all, 67 with 16 rows; 5 trees of 35 rows 18.4, 20.7).
    int some = f.wide ? 16 : 32;
    const int turn = (f.wide ? 512 : 1024) / 16 / (D / 4), least = turn > 1 ? turn : 1;
    while (by_item && some > least && f.items * ((f.rows + some - 1) / some) < 256) some /= 2;
    const unsigned chunks = (unsigned)(f.rows + some - 1) / some;
    const dim3 grid = by_item ? dim3((unsigned)(f.items / a.B / a.shape.heads) * chunks, a.shape.heads, a.B)
                              : dim3((unsigned)f.groups - 1, chunks);
    if (f.wide)
        hipLaunchKernelGGL((join_kernel<T, D, 512>), grid, dim3(512), 0, s, a, (unsigned)f.groups, some, by_item);
    else
        hipLaunchKernelGGL((join_kernel<T, D, 1024>), grid, dim3(1024), 0, s, a, (unsigned)f.groups, some, by_item);
    return hipGetLastError() == hipSuccess ? PK_OK : PK_ERR_LAUNCH;
}

template <typename T, bool COPIED>
int launch(const Args &a, const Form &f, bool joined, hipStream_t s)
{
    if (f.D == 64) return f.nq == 1 ? launch<T, 64, 1, COPIED>(a, f, joined, s) : launch<T, 64, 2, COPIED>(a, f, joined, s);
    if (f.D == 128) return f.nq == 1 ? launch<T, 128, 1, COPIED>(a, f, joined, s) : launch<T, 128, 2, COPIED>(a, f, joined, s);
    return launch<T, 256, 1, COPIED>(a, f, joined, s);
}

template <typename T>
int launch(const Args &a, const Form &f, bool copied, bool joined, hipStream_t s)
{
    return copied ? launch<T, true>(a, f, joined, s) : launch<T, false>(a, f, joined, s);
}

// What products of queries and keys are multiplied by, once q has the scale's sign (and is zero for a
// scale of 0): see Args.
float factor_of(float scale, float cap)
{
    if (scale == 0.f) return 1.f;
    return cap != 0.f ? std::fabs(scale) / cap : std::fabs(scale) * kLog2e;
}

// Whether K and V can be copied in whole chunks: 16-byte rows at 16-byte places, the
// rows of a copy (up to 8) in one page, pages and places at 32-bit strides.
bool can_copy(const pk_cache &c, int64_t d, int size)
{
    if (d * size % 16 || (uintptr_t)c.key % 16 || (uintptr_t)c.value % 16 || c.page_size % 8) return false;
    for (int i = 0; i < 3; ++i)
        if (c.key_stride[i] * size % 16 || c.value_stride[i] * size % 16) return false;
    for (const int64_t *stride : {c.key_stride, c.value_stride})
        if (stride[0] * size >= (int64_t)1 << 32 || stride[1] * size > (((int64_t)1 << 31) - 1) / c.page_size) return false;
    return true;
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
    return form_of(pk::dtype_size(dtype), d, q_heads / heads, heads, B, P * page_size, most).bytes;
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
    const float factor = factor_of(scale, cap), bound = cap * kLog2e;
    if (cap == 0.f && std::isfinite(scale) && !std::isfinite(factor)) return api_invalid(14);
    if (!(cap >= 0.f) || !std::isfinite(bound)) return api_invalid(15);
    if (cap != 0.f && std::isfinite(scale) && !std::isnormal(factor)) return api_invalid(15);
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
    const Form f = form_of(size, d, group, heads, B, P * cache->page_size, most);
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
    a.shape = {(int)M, (int)(P * cache->page_size), (int)heads, (int)group, (int)most, f.rows_shift, joined ? f.unit_shift : -1,
               // a few tokens after a context of a round length are no unit of their own, unless there are
               // work-groups for it
               f.spare ? 0 : 1 << f.unit_shift >> 1};
    a.B = (int)B;
    a.d = (int)d;
    a.page_size = (int)cache->page_size;
    a.page_shift = -1;
    for (int i = 0; i < 31; ++i)
        if ((int64_t)1 << i == cache->page_size) a.page_shift = i;
    a.sign = scale < 0.f ? -1.f : scale == 0.f ? 0.f : 1.f;
    a.scale = factor;
    a.cap = bound;
    hipStream_t s = (hipStream_t)stream;
    st = dtype == PK_F32 ? launch<float>(a, f, copied, joined, s) : dtype == PK_BF16 ? launch<bf16>(a, f, copied, joined, s) : launch<f16>(a, f, copied, joined, s);
    if (st == PK_OK) api_ran(f.wide ? (copied ? "attention_tree_wide" : "attention_tree_wide_read") : copied ? "attention_tree" : "attention_tree_read");
    return st;
}

}  // extern "C"
