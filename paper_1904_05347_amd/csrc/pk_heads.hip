// pk_heads.hip -- queries and keys between the products of an attention layer: the
// norm of each head and the rotation by its token's position, with its gradients,
// and the same on the way into a paged cache.
//
// A head's row x of d channels becomes, in fp32,
//   z = x w n,  n = 1 / sqrt(mean x^2 + eps)     (x itself without a weight)
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t) amplitude   for its pairs.
// A team of lanes holds a row, a lane two vectors of 16 bytes: of a pair's two
// channels where pairs are halves apart, of neighbours elsewhere, so that no lane
// needs another's channels and every element is read once and written once.  The
// angles of a token are common to its heads: a work-group has all heads of a token
// and makes them once, into LDS.
//
// Memory bounds large calls: 8192 tokens of 40 heads of 128 bf16, normed, move 168 MB in
// 41.3 us (4.1 TB/s, a large copy 5.1), 4100 tokens into a cache (50 heads of 128 fp16
// with its v) 101 MB in 21.1 us, gradients of the first 252 MB in 67.3 us and 4.7 (medians).
// One token takes 3.6 us, which the launch and instructions from a cold cache fill.
#include "pk_heads_checks.hpp"
#include "pk_heads_launch.hpp"
#include "pk_i8.hpp"
#include "pk_i8_checks.hpp"

namespace {

using pk::bf16;
using pk::f16;
using pk::Pack;
using pk::rounded;

// Where a side's heads lie: m * token + h * head, in elements.  (32 bits: a product of
// two and its sum to an address are one instruction.)
struct Place {
    void *p;
    unsigned token, head;
    template <typename T>
    __device__ __forceinline__ T *at(unsigned m, unsigned h) const
    {
        return (T *)p + ((uint64_t)m * token + (uint64_t)h * head);
    }
};

// The same of a cache.
struct Pages {
    void *p;
    int64_t page, place, head;
};

struct HeadsArgs {
    Place q, k, v, q_out, k_out;  // gradient: q_out, k_out the inputs' gradients
    Place q_in, k_in;             // gradient: the forward call's inputs
    Pages key, value;             // cache: where k and v go
    const void *q_weight, *k_weight;
    const int64_t *slots;  // cache: a position for each token
    const int64_t *positions;
    const double *frequencies;
    float *partial;  // gradient of the weights: a row of 2 d for each work-group
    int64_t pages;
    unsigned first, M;
    int page_size, Hq, Hk, rows;
    int d, pairs, pair_chunks, chunks, team, team_shift, teams, tokens, rounds, interleaved;
    float amplitude, eps, inv_d;
};

// The channels of a lane's two vectors: a at oa (na of them), b at ob (nb).  FULL: all of
// them, or (on false) none.
template <int E, bool FULL>
struct Chunk {
    int oa, na, ob, nb;
    bool pair, on;
    __device__ __forceinline__ Chunk(int c, int d, int pairs, int pair_chunks, int chunks, bool halves)
    {
        pair = c < pair_chunks;
        on = c < chunks;
        const int at = (pair ? c : c - pair_chunks) * 2 * E + (pair ? 0 : 2 * pairs);
        oa = pair && halves ? c * E : at;
        ob = pair && halves ? pairs + c * E : at + E;
        na = nb = E;
        if constexpr (!FULL) {
            if (pair && halves) {
                na = nb = pairs - c * E < E ? pairs - c * E : E;
            } else {
                const int n = (pair ? 2 * pairs : d) - at;
                na = n < 0 ? 0 : n < E ? n : E;
                nb = n < E ? 0 : n < 2 * E ? n - E : E;
            }
        }
    }
};

template <typename T>
using Vec = typename Pack<T>::V;

// N elements from p on, of which n are there (N of them, where FULL).
template <bool FULL, typename T, int N = 16 / (int)sizeof(T)>
__device__ __forceinline__ typename Pack<T, N>::V get(const T *p, int n)
{
    typedef typename Pack<T, N>::V V;
    if (FULL || n == N) return *reinterpret_cast<const typename Pack<T, N>::U *>(p);
    V v = (V)(T)0.f;
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (j < n) v[j] = p[j];
    return v;
}

template <bool FULL, typename T>
__device__ __forceinline__ void put(T *p, int n, const Vec<T> &v)
{
    constexpr int E = 16 / (int)sizeof(T);
    if (FULL || n == E) {
        *reinterpret_cast<typename Pack<T>::U *>(p) = v;
        return;
    }
#pragma unroll
    for (int j = 0; j < E; ++j)
        if (j < n) p[j] = v[j];
}

// The sum of v over the lanes of a team, in each of them.  Every lane of the wave
// takes part.
__device__ __forceinline__ float team_sum(float v, int team)
{
#define PK_DPP(ctrl) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, 0xf, 0xf, false))
    if (team > 1) PK_DPP(0xb1);   // lane ^ 1
    if (team > 2) PK_DPP(0x4e);   // lane ^ 2
    if (team > 4) PK_DPP(0x141);  // mirrored in 8
    if (team > 8) PK_DPP(0x140);  // mirrored in 16
#undef PK_DPP
    if (team > 16) v += __shfl_xor(v, 16);
    if (team > 32) v += __shfl_xor(v, 32);
    return v;
}

// cos and sin of position * frequency, times the amplitude.  The angle is formed in turns
// and reduced in 64 bits.  1 / (2 pi) and its product with the frequency are each held in two
// of these, and the product with the position less whole turns is rounded once, so that no
// position loses what 32 bits hold (up to 2^53, where a position is no longer exact in 64
// bits).  With one 64-bit number for each, 2^40 radians would be off by 1.6e-4.
__device__ __forceinline__ float2 turn_of(int64_t position, double frequency, float amplitude)
{
    constexpr double kHigh = 0x1.45f306dc9c883p-3, kLow = -0x1.6b01ec5417056p-57;  // of 1 / (2 pi)
    const double high = frequency * kHigh, low = fma(frequency, kHigh, -high) + frequency * kLow;
    const double p = (double)position, turns = fma(p, low, fma(p, high, -rint(p * high)));
    const float half_turns = 2.f * (float)turns;
    float s, c;
    sincospif(half_turns, &s, &c);
    return make_float2(c * amplitude, s * amplitude);
}

// The turns of `tokens` tokens from `first` on.
__device__ __forceinline__ void make_turns(const HeadsArgs &p, float2 *turns, unsigned first)
{
    for (int i = threadIdx.x; i < p.tokens * p.pairs; i += blockDim.x) {
        const int t = p.tokens > 1 ? i / p.pairs : 0;
        const unsigned m = first + t;
        turns[i] = m < p.M ? turn_of(p.positions[m], p.frequencies[i - t * p.pairs], p.amplitude) : make_float2(0.f, 0.f);
    }
}

// A lane's pairs: cos and sin of each.
template <int E>
struct Turns {
    float c[E], s[E];
    template <bool FULL>
    __device__ __forceinline__ void load(const float2 *turns, int n)
    {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            // (beyond the pairs: another's, for channels that are not stored)
            const float2 t = turns[FULL || j < n ? j : 0];
            c[j] = t.x;
            s[j] = t.y;
        }
    }
    // The pairs of z (the first vector's E values, then the second's) turned; BACK: by the
    // opposite angle.
    template <bool INTERLEAVED, bool BACK>
    __device__ __forceinline__ void rotate(float *z) const
    {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int ia = INTERLEAVED ? 2 * j : j, ib = INTERLEAVED ? 2 * j + 1 : E + j;
            const float a = z[ia], b = z[ib], t = BACK ? -s[j] : s[j];
            z[ia] = fmaf(a, c[j], -(b * t));
            z[ib] = fmaf(b, c[j], a * t);
        }
    }
};

// 1 / sqrt(mean z^2 + eps) of a row z over its team: z times root is the row normed.  A
// sum of squares that leaves the 32 bits' range, or falls where eps does not cover what
// it loses, is taken once more of z times a power of two, `up`, and z left so.
struct Factor {
    float root, up;
};

template <int E>
__device__ __forceinline__ Factor norm(float *z, float inv_d, int team, float eps)
{
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < 2 * E; ++j) ss = fmaf(z[j], z[j], ss);
    ss = team_sum(ss, team);
    float up = 1.f;
    const bool above = !(ss < 0x1p120f), below = ss < 0x1p-80f && eps < 0x1p-100f;
    if (__any(above || below)) {  // the whole wave: the sum is across lanes
        up = above ? 0x1p-70f : below ? 0x1p100f : 1.f;
        ss = 0.f;
#pragma unroll
        for (int j = 0; j < 2 * E; ++j) {
            z[j] *= up;
            ss = fmaf(z[j], z[j], ss);
        }
        ss = team_sum(ss, team);
        eps = eps * up * up;  // one by one: 2^200 is no fp32 number
    }
    return {__builtin_amdgcn_rsqf(fmaf(ss, inv_d, eps)), up};
}

// How a call's pairs lie.
enum { UNTURNED, HALVES, NEIGHBOURS };

// The sides that lanes of this wave have, one after the other, each as a scalar: its
// addresses and strides then need no selection for each lane, and most waves have
// rows of one side.
template <typename F>
__device__ __forceinline__ void each_side(int side, F f)
{
    for (bool left = true; left;) {
        const int s = __builtin_amdgcn_readfirstlane(side);
        if (side == s) {
            f(s);
            left = false;
        }
    }
}

enum { QUERY, KEY, VALUE, NONE };

// One token's heads are its queries', its keys', then its values'.  Few instructions
// count here as much as bytes: a work-group for each token (several, where its heads
// are few), whose waves' number hides what memory takes.  (Work-groups that go from token
// to token with the next one's rows ahead hold 128 registers and took 70 us where this
// took 57.)
template <typename T, typename W, bool NORM, int PAIRS, bool FULL>
__global__ void __launch_bounds__(pk::kMostHeadThreads) heads_kernel(HeadsArgs p)
{
    constexpr int E = 16 / (int)sizeof(T);
    typedef typename Pack<W, E>::V VW;
    extern __shared__ float2 s_turns[];
    const int c = threadIdx.x & (p.team - 1);
    const pk::HeadStart slot = pk::head_start(threadIdx.x >> p.team_shift, p.tokens, p.rows);
    int r = slot.row;
    const unsigned first = p.first + blockIdx.x * p.tokens, m = first + slot.token;
    const Chunk<E, FULL> k(c, p.d, PAIRS ? p.pairs : 0, PAIRS ? p.pair_chunks : 0, p.chunks, PAIRS == HALVES);

    struct Row {
        Vec<T> a, b;
        VW wa, wb;
        T *to;
        int side;
        bool weighed;
    };
    // a row's channels, and its weights, on their way
    auto fetch = [&](int row) {
        Row x;
        x.a = x.b = (Vec<T>)(T)0.f;
        x.wa = x.wb = (VW)(W)1.f;
        x.to = nullptr;
        x.weighed = false;
        x.side = m >= p.M || row >= p.rows || !k.on ? NONE : row < p.Hq ? QUERY : row < p.Hq + p.Hk ? KEY : VALUE;
        each_side(x.side, [&](int s) {
            if (s == NONE) return;
            const unsigned h = row - (s == QUERY ? 0 : s == KEY ? p.Hq : p.Hq + p.Hk);
            const T *at = (s == QUERY ? p.q : s == KEY ? p.k : p.v).template at<const T>(m, h);
            x.a = get<FULL>(at + k.oa, k.na);
            x.b = get<FULL>(at + k.ob, k.nb);
            if constexpr (NORM) {
                const W *w = (const W *)(s == QUERY ? p.q_weight : s == KEY ? p.k_weight : nullptr);
                if (w) {
                    x.weighed = true;
                    x.wa = get<FULL, W, E>(w + k.oa, k.na);
                    x.wb = get<FULL, W, E>(w + k.ob, k.nb);
                }
            }
            if (s == QUERY || !p.slots) {
                x.to = (s == QUERY ? p.q_out : p.k_out).template at<T>(m, h);
                return;
            }
            // the token's place in the cache
            const int64_t at_slot = p.slots[m];
            int64_t page, place;
            if ((uint64_t)at_slot >> 32) {
                page = (int64_t)((uint64_t)at_slot / (unsigned)p.page_size);
                place = at_slot - page * p.page_size;
            } else {
                page = (unsigned)at_slot / (unsigned)p.page_size;
                place = (unsigned)at_slot - (unsigned)page * (unsigned)p.page_size;
            }
            const Pages &to = s == KEY ? p.key : p.value;
            x.to = (T *)to.p + page * to.page + place * to.place + h * to.head;
            if (at_slot < 0 || page >= p.pages) x.side = NONE;  // has no place: nothing is stored
        });
        return x;
    };

    Row x = fetch(r);
    if constexpr (PAIRS != UNTURNED) {
        make_turns(p, s_turns, first);
        __syncthreads();
    }
    for (int i = 0;;) {
        if constexpr (NORM || PAIRS != UNTURNED) {
            float z[2 * E];
#pragma unroll
            for (int j = 0; j < E; ++j) {
                z[j] = (float)x.a[j];
                z[E + j] = (float)x.b[j];
            }
            if constexpr (NORM) {
                float y[2 * E];
#pragma unroll
                for (int j = 0; j < 2 * E; ++j) y[j] = z[j];
                const Factor f = norm<E>(y, p.inv_d, p.team, p.eps);  // every lane of the wave, whatever its row
                if (x.weighed) {
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        z[j] = y[j] * f.root * (float)x.wa[j];
                        z[E + j] = y[E + j] * f.root * (float)x.wb[j];
                    }
                }
            }
            if (x.side < VALUE) {
                if constexpr (PAIRS != UNTURNED) {
                    if (k.pair) {
                        Turns<E> turns;
                        turns.template load<FULL>(s_turns + slot.token * p.pairs + c * E, p.pairs - c * E);
                        turns.template rotate<PAIRS == NEIGHBOURS, false>(z);
                    }
                }
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    x.a[j] = rounded<T>(z[j]);
                    x.b[j] = rounded<T>(z[E + j]);
                }
            }
        }
        if (x.side != NONE) {
            put<FULL>(x.to + k.oa, k.na, x.a);
            put<FULL>(x.to + k.ob, k.nb, x.b);
        }
        if (++i >= p.rounds) break;
        r += p.teams;
        x = fetch(r);
    }
}

// Gradients: with g the output's gradient turned back, u = x n,
//   dx = n (g w - u mean(g w u)),  dw = sum g u.
// A lane has the same channels of every row, so a work-group keeps its part of dw
// in registers over all its tokens; its rows are added up by weights_kernel in the
// order of the work-groups.  The next token's rows are on their way while one is
// worked on.
// ONE: a team has the same head of every token, so that its lanes have one side's
// weights and sums.
// (67.3 us for 252 MB, 8192 tokens of 40 heads of 128 bf16, 61 at the least; a tenth less than the
// forward kernel's rate: 21 % of the waves' cycles issue arithmetic, 61 % wait.)
template <typename T, typename W, bool NORM, int PAIRS, bool FULL, bool ONE>
__global__ void __launch_bounds__(pk::kMostHeadThreads, ONE ? 4 : 3) heads_grad_kernel(HeadsArgs p)
{
    constexpr int E = 16 / (int)sizeof(T);
    typedef typename Pack<W, E>::V VW;
    extern __shared__ float2 s_turns[];
    const int c = threadIdx.x & (p.team - 1);
    const pk::HeadStart slot = pk::head_start(threadIdx.x >> p.team_shift, p.tokens, p.rows);
    const Chunk<E, FULL> ck(c, p.d, PAIRS ? p.pairs : 0, PAIRS ? p.pair_chunks : 0, p.chunks, PAIRS == HALVES);
    constexpr int SUMS = NORM ? 2 * E : 1;
    float sum_q[SUMS], sum_k[SUMS];  // ONE: sum_q is that side's
#pragma unroll
    for (int j = 0; j < SUMS; ++j) sum_q[j] = sum_k[j] = 0.f;
    const W *const weight_one = NORM ? (const W *)(slot.row < p.Hq ? p.q_weight : p.k_weight) : nullptr;
    VW wa = (VW)(W)0.f, wb = wa;
    if (NORM && ONE && weight_one && ck.on) {
        wa = get<FULL, W, E>(weight_one + ck.oa, ck.na);
        wb = get<FULL, W, E>(weight_one + ck.ob, ck.nb);
    }

    struct Row {
        Vec<T> a, b, xa, xb;  // the gradient, the input
        T *to;
        int side;
    };
    auto fetch = [&](unsigned first, int row) {
        Row x;
        const unsigned m = first + slot.token;
        x.a = x.b = x.xa = x.xb = (Vec<T>)(T)0.f;
        x.to = nullptr;
        x.side = m >= p.M || row >= p.rows || !ck.on ? NONE : row < p.Hq ? QUERY : KEY;
        each_side(x.side, [&](int s) {
            if (s == NONE) return;
            const unsigned h = row - (s == QUERY ? 0 : p.Hq);
            const T *at = (s == QUERY ? p.q : p.k).template at<const T>(m, h);
            x.a = get<FULL>(at + ck.oa, ck.na);
            x.b = get<FULL>(at + ck.ob, ck.nb);
            if constexpr (NORM) {
                if (s == QUERY ? p.q_weight : p.k_weight) {
                    const T *px = (s == QUERY ? p.q_in : p.k_in).template at<const T>(m, h);
                    x.xa = get<FULL>(px + ck.oa, ck.na);
                    x.xb = get<FULL>(px + ck.ob, ck.nb);
                }
            }
            x.to = (s == QUERY ? p.q_out : p.k_out).template at<T>(m, h);
        });
        return x;
    };

    const unsigned step = gridDim.x * p.tokens;
    int half = 0;
    unsigned first = blockIdx.x * p.tokens;
    Row x = fetch(first, slot.row);
    for (; first < p.M; first += step, half ^= 1) {
        float2 *turns_here = s_turns + half * p.tokens * p.pairs;
        if constexpr (PAIRS != UNTURNED) {
            // the other half may still be read
            make_turns(p, turns_here, first);
            __syncthreads();
        }
        int r = slot.row;
        for (int i = 0; i < (ONE ? 1 : p.rounds); ++i) {
            Row now = x;
            x = !ONE && i + 1 < p.rounds ? fetch(first, r + p.teams) : fetch(first + step, slot.row);
            r += p.teams;
            float g[2 * E];
#pragma unroll
            for (int j = 0; j < E; ++j) {
                g[j] = (float)now.a[j];
                g[E + j] = (float)now.b[j];
            }
            if constexpr (PAIRS != UNTURNED) {
                if (ck.pair) {
                    Turns<E> turns;
                    turns.template load<FULL>(turns_here + slot.token * p.pairs + c * E, p.pairs - c * E);
                    turns.template rotate<PAIRS == NEIGHBOURS, true>(g);
                }
            }
            if constexpr (NORM) {
                const W *weight = ONE ? weight_one : (const W *)(now.side == QUERY ? p.q_weight : p.k_weight);
                float u[2 * E], dot = 0.f;
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    u[j] = (float)now.xa[j];
                    u[E + j] = (float)now.xb[j];
                }
                const Factor f = norm<E>(u, p.inv_d, p.team, p.eps);
                // rows that are not there, and sides without a weight, add nothing
                const bool weighed = now.side != NONE && weight;
                if (weighed) {
                    if constexpr (!ONE) {
                        wa = get<FULL, W, E>(weight + ck.oa, ck.na);
                        wb = get<FULL, W, E>(weight + ck.ob, ck.nb);
                    }
#pragma unroll
                    for (int j = 0; j < 2 * E; ++j) u[j] *= f.root;
                    if (ONE || now.side == QUERY) {
#pragma unroll
                        for (int j = 0; j < 2 * E; ++j) sum_q[j] = fmaf(g[j], u[j], sum_q[j]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 2 * E; ++j) sum_k[j] = fmaf(g[j], u[j], sum_k[j]);
                    }
#pragma unroll
                    for (int j = 0; j < 2 * E; ++j) {
                        g[j] *= (float)(j < E ? wa[j % E] : wb[j % E]);
                        dot = fmaf(g[j], u[j], dot);
                    }
                }
                dot = team_sum(dot, p.team) * p.inv_d;
                if (weighed) {
#pragma unroll
                    for (int j = 0; j < 2 * E; ++j) g[j] = fmaf(-u[j], dot, g[j]) * f.root;
                    if (f.up != 1.f) {
#pragma unroll
                        for (int j = 0; j < 2 * E; ++j) g[j] *= f.up;
                    }
                }
            }
            if (now.side != NONE) {
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    now.a[j] = rounded<T>(g[j]);
                    now.b[j] = rounded<T>(g[E + j]);
                }
                put<FULL>(now.to + ck.oa, ck.na, now.a);
                put<FULL>(now.to + ck.ob, ck.nb, now.b);
            }
        }
    }
    if constexpr (NORM) {
        if (ONE) {
            const bool query = slot.row < p.Hq;
#pragma unroll
            for (int j = 0; j < 2 * E; ++j) {
                sum_k[j] = query ? 0.f : sum_q[j];
                sum_q[j] = query ? sum_q[j] : 0.f;
            }
        }
        // over the teams of a wave, then over the waves
        for (int o = p.team; o < 64; o *= 2) {
#pragma unroll
            for (int j = 0; j < 2 * E; ++j) {
                sum_q[j] += __shfl_xor(sum_q[j], o);
                sum_k[j] += __shfl_xor(sum_k[j], o);
            }
        }
        float *s_sum = (float *)s_turns;
        __syncthreads();  // the turns have been read
        const int wave = threadIdx.x / 64, waves = blockDim.x / 64;
        if (threadIdx.x % 64 < p.team && ck.on) {
            float *q = s_sum + wave * 2 * p.d, *k = q + p.d;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                if (j < ck.na) {
                    q[ck.oa + j] = sum_q[j];
                    k[ck.oa + j] = sum_k[j];
                }
                if (j < ck.nb) {
                    q[ck.ob + j] = sum_q[E + j];
                    k[ck.ob + j] = sum_k[E + j];
                }
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * p.d; i += blockDim.x) {
            float v = 0.f;
            for (int w = 0; w < waves; ++w) v += s_sum[w * 2 * p.d + i];
            p.partial[(int64_t)blockIdx.x * 2 * p.d + i] = v;
        }
    }
}

// The rows of `partial` added up: 16 columns a work-group, 64 lanes a column.  (3.5 us
// for 1003 rows of 192: a launch, a lane's 16 loads and the columns' sums.)
template <typename W>
__global__ void __launch_bounds__(1024) weights_kernel(const float *partial, int groups, int d, W *q, W *k)
{
    __shared__ float s_v[16][17];
    const int x = threadIdx.x % 16, y = threadIdx.x / 16, col = blockIdx.x * 16 + x;
    float v = 0.f;
    if (col < 2 * d) {
        // 16 rows at once, the last in the place of those beyond it: the loads of a loop over
        // what is left of them would be waited for one by one (7.2 us)
        for (int g = y; g < groups; g += 16 * 64) {
            float row[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int at = g + 64 * i;
                row[i] = partial[(int64_t)(at < groups ? at : groups - 1) * 2 * d + col];
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) v += g + 64 * i < groups ? row[i] : 0.f;
        }
    }
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
    if (y % 4 == 0) s_v[y / 4][x] = v;
    __syncthreads();
    if (y || col >= 2 * d) return;
    v = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += s_v[i][x];
    W *to = col < d ? q : k;
    if (to) to[col < d ? col : col - d] = (W)v;
}

// ---------------------------------------------------------------- launches

constexpr int64_t kMostGroups = 1 << 22;  // of a launch: 512 work-items each stay below 2^32
constexpr int kGradGroups = 1024;         // rows of partial sums, at most

int log2_of(int v)
{
    int s = 0;
    while (1 << s < v) ++s;
    return s;
}

// The tiling of `a` for its type's vectors.
pk::HeadGroup lay_out(HeadsArgs &a, int rows, int size)
{
    const pk::HeadTiling t = pk::head_tiling(a.d, a.pairs, 16 / size);
    const pk::HeadGroup g = pk::head_group(rows, t.team, a.pairs);
    a.rows = rows;
    a.pair_chunks = t.pair_chunks;
    a.chunks = t.chunks;
    a.team = t.team;
    a.team_shift = log2_of(t.team);
    a.teams = g.teams;
    a.tokens = g.tokens;
    a.rounds = g.tokens > 1 ? 1 : (rows + g.teams - 1) / g.teams;
    return g;
}

template <typename T, typename W, bool NORM, int PAIRS, bool FULL>
int launch_heads(HeadsArgs a, int rows, hipStream_t s)
{
    const pk::HeadGroup g = lay_out(a, rows, (int)sizeof(T));
    const size_t lds = (size_t)a.tokens * a.pairs * sizeof(float2);
    for (int64_t left = ((int64_t)a.M + a.tokens - 1) / a.tokens; left > 0; left -= kMostGroups) {
        const int64_t now = left < kMostGroups ? left : kMostGroups;
        hipLaunchKernelGGL((heads_kernel<T, W, NORM, PAIRS, FULL>), dim3((unsigned)now), dim3(g.threads), lds, s, a);
        if (hipGetLastError() != hipSuccess) return PK_ERR_LAUNCH;
        a.first += (unsigned)(now * a.tokens);
    }
    return PK_OK;
}

template <typename T, typename W, bool NORM, int PAIRS, bool FULL>
int launch_grad(HeadsArgs a, int rows, int64_t *groups, hipStream_t s)
{
    const pk::HeadGroup g = lay_out(a, rows, (int)sizeof(T));
    // what the card holds at once, by the registers, and as many tokens to each
    const bool one = a.rounds == 1;
    const int waves = g.threads / 64, resident = (one ? 16 : 12) / waves > 0 ? (one ? 16 : 12) / waves : 1;
    *groups = ((int64_t)a.M + a.tokens - 1) / a.tokens;
    if (*groups > 256 * resident) {
        const int64_t turns = (*groups + 256 * resident - 1) / (256 * resident);
        *groups = (*groups + turns - 1) / turns;
    }
    if (*groups > kGradGroups) *groups = kGradGroups;
    size_t lds = (size_t)2 * a.tokens * a.pairs * sizeof(float2);
    const size_t sums = NORM ? (size_t)(g.threads / 64) * 2 * a.d * sizeof(float) : 0;
    if (lds < sums) lds = sums;
    if (one)
        hipLaunchKernelGGL((heads_grad_kernel<T, W, NORM, PAIRS, FULL, true>), dim3((unsigned)*groups), dim3(g.threads), lds, s, a);
    else
        hipLaunchKernelGGL((heads_grad_kernel<T, W, NORM, PAIRS, FULL, false>), dim3((unsigned)*groups), dim3(g.threads), lds, s, a);
    return hipGetLastError() == hipSuccess ? PK_OK : PK_ERR_LAUNCH;
}

// The instance for a call's types, weights and pairs; FULL: every lane's vectors are whole.
#define PK_HEADS_FULL(FN, T, W, NORM, PAIRS, ...)                                                            \
    (a.pairs % (16 / (int)sizeof(T)) == 0 && (a.d - 2 * a.pairs) % (32 / (int)sizeof(T)) == 0                 \
         ? FN<T, W, NORM, PAIRS, true>(__VA_ARGS__)                                                          \
         : FN<T, W, NORM, PAIRS, false>(__VA_ARGS__))
#define PK_HEADS(FN, T, W, NORM, ...)                                                  \
    (!a.pairs         ? PK_HEADS_FULL(FN, T, W, NORM, UNTURNED, __VA_ARGS__)          \
     : a.interleaved  ? PK_HEADS_FULL(FN, T, W, NORM, NEIGHBOURS, __VA_ARGS__)        \
                      : PK_HEADS_FULL(FN, T, W, NORM, HALVES, __VA_ARGS__))
#define PK_HEADS_TYPES(FN, ...)                                                                                       \
    (!a.q_weight && !a.k_weight ? (dtype == PK_F32    ? PK_HEADS(FN, float, float, false, __VA_ARGS__)                 \
                                   : dtype == PK_BF16 ? PK_HEADS(FN, bf16, bf16, false, __VA_ARGS__)                   \
                                                      : PK_HEADS(FN, f16, f16, false, __VA_ARGS__))                    \
     : dtype == PK_F32         ? PK_HEADS(FN, float, float, true, __VA_ARGS__)                                         \
     : weight_dtype == PK_F32  ? (dtype == PK_BF16 ? PK_HEADS(FN, bf16, float, true, __VA_ARGS__)                       \
                                                   : PK_HEADS(FN, f16, float, true, __VA_ARGS__))                       \
     : dtype == PK_BF16        ? PK_HEADS(FN, bf16, bf16, true, __VA_ARGS__)                                           \
                               : PK_HEADS(FN, f16, f16, true, __VA_ARGS__))

int run_heads(int dtype, int weight_dtype, const HeadsArgs &a, int rows, hipStream_t s)
{
    return PK_HEADS_TYPES(launch_heads, a, rows, s);
}

template <typename W>
int launch_weights(const HeadsArgs &a, int64_t groups, void *q, void *k, hipStream_t s)
{
    hipLaunchKernelGGL((weights_kernel<W>), dim3((2 * a.d + 15) / 16), dim3(1024), 0, s, a.partial, (int)groups, a.d, (W *)q,
                       (W *)k);
    return hipGetLastError() == hipSuccess ? PK_OK : PK_ERR_LAUNCH;
}

int run_grad(int dtype, int weight_dtype, const HeadsArgs &a, int rows, void *q_weight_grad, void *k_weight_grad, hipStream_t s)
{
    int64_t groups = 0;
    if (rows && a.M) {
        const int st = PK_HEADS_TYPES(launch_grad, a, rows, &groups, s);
        if (st != PK_OK) return st;
    }
    if (!q_weight_grad && !k_weight_grad) return PK_OK;
    return weight_dtype == PK_F32    ? launch_weights<float>(a, groups, q_weight_grad, k_weight_grad, s)
           : weight_dtype == PK_BF16 ? launch_weights<bf16>(a, groups, q_weight_grad, k_weight_grad, s)
                                     : launch_weights<f16>(a, groups, q_weight_grad, k_weight_grad, s);
}

// What every call checks of its rotation: 0, or the status.
int check_rotation(const pk_rotation *rot, int64_t d, bool read)
{
    if (!rot) return PK_OK;
    if (rot->pairs < 0 || rot->pairs > d / 2) return PK_ERR_INVALID_VALUE;
    if (rot->pairs && read &&
        (!rot->positions || !rot->frequencies || (uintptr_t)rot->positions % 8 || (uintptr_t)rot->frequencies % 8))
        return PK_ERR_INVALID_VALUE;
    return PK_OK;
}

void set_rotation(HeadsArgs &a, const pk_rotation *rot)
{
    if (!rot || !rot->pairs) return;
    a.positions = rot->positions;
    a.frequencies = rot->frequencies;
    a.pairs = (int)rot->pairs;
    a.interleaved = rot->interleaved != 0;
    a.amplitude = rot->amplitude;
}

Place place(const pk_heads *t)
{
    if (!t) return {nullptr, 0, 0};
    return {t->data, (unsigned)t->token_stride, (unsigned)t->head_stride};
}

// Whether an output shares memory with the rotation's arrays or a weight.
bool over_small(const pk::heads::Region &out, const pk_rotation *rot, int64_t M, const void *qw, const void *kw, int64_t wbytes)
{
    using namespace pk::heads;
    if (rot && rot->pairs && (shared(out, flat(rot->positions, 8 * M)) || shared(out, flat(rot->frequencies, 8 * rot->pairs))))
        return true;
    return (qw && shared(out, flat(qw, wbytes))) || (kw && shared(out, flat(kw, wbytes)));
}

}  // namespace

extern "C" {

int pk_rope_qk(int dtype, int64_t M, int64_t d, const pk_heads *q, const pk_heads *k, const pk_rotation *rotation,
               const void *q_weight, const void *k_weight, int weight_dtype, float eps, const pk_heads *q_out,
               const pk_heads *k_out, void *stream)
{
    using namespace pk;
    using namespace pk::heads;
    api_begin();
    const int size = dtype_size(dtype), wsize = dtype_size(weight_dtype);
    if (!size) return api_invalid(1);
    if (M < 0) return api_invalid(2);
    if (d < 1) return api_invalid(3);
    if (q_weight && !q) return api_invalid(7);
    if (k_weight && !k) return api_invalid(8);
    if ((q_weight || k_weight) && weight_dtype != PK_F32 && weight_dtype != dtype) return api_invalid(9);
    if ((q_weight || k_weight) && !(eps >= 0.f)) return api_invalid(10);
    if (!q_out != !q || (q && q_out->heads != q->heads)) return api_invalid(11);
    if (!k_out != !k || (k && k_out->heads != k->heads)) return api_invalid(12);
    if (M > kMostSize || d > 256) return PK_ERR_NOT_SUPPORTED;
    int st;
    if (check_rotation(rotation, d, M > 0)) return api_invalid(6);
    if (q && (st = check_heads(*q, M, size, false, d))) return st == PK_ERR_INVALID_VALUE ? api_invalid(4) : st;
    if (k && (st = check_heads(*k, M, size, false, d))) return st == PK_ERR_INVALID_VALUE ? api_invalid(5) : st;
    if (q && (st = check_heads(*q_out, M, size, true, d))) return st == PK_ERR_INVALID_VALUE ? api_invalid(11) : st;
    if (k && (st = check_heads(*k_out, M, size, true, d))) return st == PK_ERR_INVALID_VALUE ? api_invalid(12) : st;
    if (q_weight && (uintptr_t)q_weight % (uintptr_t)wsize) return api_invalid(7);
    if (k_weight && (uintptr_t)k_weight % (uintptr_t)wsize) return api_invalid(8);
    const int64_t Hq = q ? q->heads : 0, Hk = k ? k->heads : 0;
    if (M == 0 || Hq + Hk == 0) return PK_OK;
    const Region none = flat(nullptr, 0), rq = q ? of_heads(*q, M, d, size) : none, rk = k ? of_heads(*k, M, d, size) : none;
    const Region oq = q ? of_heads(*q_out, M, d, size) : none, ok = k ? of_heads(*k_out, M, d, size) : none;
    if (shared(oq, rk) || (shared(oq, rq) && !same_place(*q, *q_out, M)) ||
        over_small(oq, rotation, M, q_weight, k_weight, d * wsize))
        return api_invalid(11);
    if (shared(ok, rq) || shared(ok, oq) || (shared(ok, rk) && !same_place(*k, *k_out, M)) ||
        over_small(ok, rotation, M, q_weight, k_weight, d * wsize))
        return api_invalid(12);
    HeadsArgs a = {};
    a.q = place(q);
    a.k = place(k);
    a.q_out = place(q_out);
    a.k_out = place(k_out);
    a.q_weight = q_weight;
    a.k_weight = k_weight;
    a.M = (unsigned)M;
    a.Hq = (int)Hq;
    a.Hk = (int)Hk;
    a.d = (int)d;
    a.eps = eps;
    a.inv_d = 1.f / (float)d;
    set_rotation(a, rotation);
    st = run_heads(dtype, weight_dtype, a, (int)(Hq + Hk), (hipStream_t)stream);
    if (st == PK_OK) api_ran("rope_qk");
    return st;
}

size_t pk_rope_qk_backward_workspace_bytes(int64_t M, int64_t d)
{
    if (M < 1 || d < 1 || d > 256) return 0;
    return (size_t)(M < kGradGroups ? M : kGradGroups) * 2 * (size_t)d * sizeof(float);
}

int pk_rope_qk_backward(int dtype, int64_t M, int64_t d, const pk_heads *dq, const pk_heads *dk, const pk_heads *q,
                        const pk_heads *k, const pk_rotation *rotation, const void *q_weight, const void *k_weight,
                        int weight_dtype, float eps, const pk_heads *q_grad, const pk_heads *k_grad,
                        void *q_weight_grad, void *k_weight_grad, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace pk;
    using namespace pk::heads;
    api_begin();
    const int size = dtype_size(dtype), wsize = dtype_size(weight_dtype);
    const bool weights = q_weight || k_weight;
    if (!size) return api_invalid(1);
    if (M < 0) return api_invalid(2);
    if (d < 1) return api_invalid(3);
    if (q_weight && (!q || !dq || q->heads != dq->heads)) return api_invalid(6);
    if (k_weight && (!k || !dk || k->heads != dk->heads)) return api_invalid(7);
    if (weights && weight_dtype != PK_F32 && weight_dtype != dtype) return api_invalid(11);
    if (weights && !(eps >= 0.f)) return api_invalid(12);
    if (!q_grad != !dq || (dq && q_grad->heads != dq->heads)) return api_invalid(13);
    if (!k_grad != !dk || (dk && k_grad->heads != dk->heads)) return api_invalid(14);
    if (!q_weight_grad != !q_weight) return api_invalid(15);
    if (!k_weight_grad != !k_weight) return api_invalid(16);
    if (M > kMostSize || d > 256) return PK_ERR_NOT_SUPPORTED;
    if (!q_weight) q = nullptr;  // not read
    if (!k_weight) k = nullptr;
    int st;
    if (check_rotation(rotation, d, M > 0)) return api_invalid(8);
    const pk_heads *in[6] = {dq, dk, q, k, q_grad, k_grad};
    const int at[6] = {4, 5, 6, 7, 13, 14};
    for (int i = 0; i < 6; ++i)
        if (in[i] && (st = check_heads(*in[i], M, size, i >= 4, d))) return st == PK_ERR_INVALID_VALUE ? api_invalid(at[i]) : st;
    if (weights) {
        const void *vectors[4] = {q_weight, k_weight, q_weight_grad, k_weight_grad};
        const int where[4] = {9, 10, 15, 16};
        for (int i = 0; i < 4; ++i)
            if (vectors[i] && (uintptr_t)vectors[i] % (uintptr_t)wsize) return api_invalid(where[i]);
    }
    Region r[6];
    for (int i = 0; i < 6; ++i) r[i] = in[i] ? of_heads(*in[i], M, d, size) : flat(nullptr, 0);
    for (int o = 4; o < 6; ++o) {
        for (int i = 0; i < o; ++i) {
            const bool own = i == o - 4 && in[i] && same_place(*in[i], *in[o], M);
            if (shared(r[o], r[i]) && !own) return api_invalid(at[o]);
        }
        if (over_small(r[o], rotation, M, q_weight, k_weight, d * wsize)) return api_invalid(at[o]);
    }
    const int64_t wbytes = weights ? d * wsize : 0;
    void *wg[2] = {q_weight_grad, k_weight_grad};
    for (int o = 0; o < 2; ++o) {
        if (!wg[o]) continue;
        const Region w = flat(wg[o], wbytes);
        for (int i = 0; i < 6; ++i)
            if (shared(w, r[i])) return api_invalid(15 + o);
        if (over_small(w, rotation, M, q_weight, k_weight, wbytes) || (o && wg[0] && shared(w, flat(wg[0], wbytes))))
            return api_invalid(15 + o);
    }
    const int64_t Hq = dq ? dq->heads : 0, Hk = dk ? dk->heads : 0;
    const bool work = M > 0 && Hq + Hk > 0;
    if (weights) {
        const size_t need = work ? pk_rope_qk_backward_workspace_bytes(M, d) : 0;
        if (workspace_bytes < need || (need && !workspace)) return PK_ERR_WORKSPACE;
        if ((uintptr_t)workspace % 16) return api_invalid(17);
        const Region ws = flat(workspace, (int64_t)need);
        for (int i = 0; i < 6; ++i)
            if (shared(ws, r[i])) return api_invalid(17);
        for (int o = 0; o < 2; ++o)
            if (wg[o] && shared(ws, flat(wg[o], wbytes))) return api_invalid(17);
        if (over_small(ws, rotation, M, q_weight, k_weight, wbytes)) return api_invalid(17);
    }
    if (!work && !weights) return PK_OK;
    HeadsArgs a = {};
    a.q = place(dq);
    a.k = place(dk);
    a.q_in = place(q);
    a.k_in = place(k);
    a.q_out = place(q_grad);
    a.k_out = place(k_grad);
    a.q_weight = q_weight;
    a.k_weight = k_weight;
    a.partial = (float *)workspace;
    a.M = (unsigned)M;
    a.Hq = (int)Hq;
    a.Hk = (int)Hk;
    a.d = (int)d;
    a.eps = eps;
    a.inv_d = 1.f / (float)d;
    set_rotation(a, rotation);
    st = run_grad(dtype, weight_dtype, a, (int)(Hq + Hk), q_weight_grad, k_weight_grad, (hipStream_t)stream);
    if (st == PK_OK) api_ran("rope_qk_backward");
    return st;
}

int pk_cache_append(int dtype, int64_t M, int64_t d, const pk_heads *q, const pk_heads *k, const pk_heads *v,
                    const pk_rotation *rotation, const void *q_weight, const void *k_weight, int weight_dtype, float eps,
                    const pk_heads *q_out, const pk_cache *cache, const int64_t *slots, void *stream)
{
    using namespace pk;
    using namespace pk::heads;
    api_begin();
    const int size = dtype_size(dtype), wsize = dtype_size(weight_dtype);
    if (!size) return api_invalid(1);
    if (M < 0) return api_invalid(2);
    if (d < 1) return api_invalid(3);
    if (!k) return api_invalid(5);
    if (!v || v->heads != k->heads) return api_invalid(6);
    if (q_weight && !q) return api_invalid(8);
    if ((q_weight || k_weight) && weight_dtype != PK_F32 && weight_dtype != dtype) return api_invalid(10);
    if ((q_weight || k_weight) && !(eps >= 0.f)) return api_invalid(11);
    if (!q_out != !q || (q && q_out->heads != q->heads)) return api_invalid(12);
    if (!cache || cache->heads != k->heads) return api_invalid(13);
    if (M > kMostSize || d > 256) return PK_ERR_NOT_SUPPORTED;
    int st;
    if (check_rotation(rotation, d, M > 0)) return api_invalid(7);
    if (q && (st = check_heads(*q, M, size, false, d))) return st == PK_ERR_INVALID_VALUE ? api_invalid(4) : st;
    if ((st = check_heads(*k, M, size, false, d))) return st == PK_ERR_INVALID_VALUE ? api_invalid(5) : st;
    if ((st = check_heads(*v, M, size, false, d))) return st == PK_ERR_INVALID_VALUE ? api_invalid(6) : st;
    if (q && (st = check_heads(*q_out, M, size, true, d))) return st == PK_ERR_INVALID_VALUE ? api_invalid(12) : st;
    if ((st = check_cache(*cache, size, true, d))) return st == PK_ERR_INVALID_VALUE ? api_invalid(13) : st;
    if (q_weight && (uintptr_t)q_weight % (uintptr_t)wsize) return api_invalid(8);
    if (k_weight && (uintptr_t)k_weight % (uintptr_t)wsize) return api_invalid(9);
    const int64_t Hq = q ? q->heads : 0, Hk = k->heads;
    if (M == 0 || Hq + Hk == 0) return PK_OK;
    if (!slots || (uintptr_t)slots % 8) return api_invalid(14);
    const Region none = flat(nullptr, 0), rq = q ? of_heads(*q, M, d, size) : none, rk = of_heads(*k, M, d, size),
                 rv = of_heads(*v, M, d, size), rs = flat(slots, 8 * M);
    const Region oq = q ? of_heads(*q_out, M, d, size) : none, kc = of_cache(cache->key, cache->key_stride, *cache, d, size),
                 vc = of_cache(cache->value, cache->value_stride, *cache, d, size);
    if (shared(oq, rk) || shared(oq, rv) || shared(oq, rs) || (shared(oq, rq) && !same_place(*q, *q_out, M)) ||
        over_small(oq, rotation, M, q_weight, k_weight, d * wsize))
        return api_invalid(12);
    for (const Region &c : {kc, vc})
        if (shared(c, rq) || shared(c, rk) || shared(c, rv) || shared(c, rs) || shared(c, oq) ||
            over_small(c, rotation, M, q_weight, k_weight, d * wsize))
            return api_invalid(13);
    HeadsArgs a = {};
    a.q = place(q);
    a.k = place(k);
    a.v = place(v);
    a.q_out = place(q_out);
    a.key = {cache->key, cache->key_stride[0], cache->key_stride[1], cache->key_stride[2]};
    a.value = {cache->value, cache->value_stride[0], cache->value_stride[1], cache->value_stride[2]};
    a.slots = slots;
    a.pages = cache->pages;
    a.page_size = (int)cache->page_size;
    a.q_weight = q_weight;
    a.k_weight = k_weight;
    a.M = (unsigned)M;
    a.Hq = (int)Hq;
    a.Hk = (int)Hk;
    a.d = (int)d;
    a.eps = eps;
    a.inv_d = 1.f / (float)d;
    set_rotation(a, rotation);
    st = run_heads(dtype, weight_dtype, a, (int)(Hq + 2 * Hk), (hipStream_t)stream);
    if (st == PK_OK) api_ran("cache_append");
    return st;
}

}  // extern "C"
