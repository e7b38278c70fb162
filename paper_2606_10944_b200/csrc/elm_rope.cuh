// Rotary positions: what the rotation kernel and the kernel that stores rows in 4 bits share.
#pragma once
#include <math.h>

#include "elm_common.cuh"
#include "elm_sm100.cuh"

namespace elm {

constexpr int ROPE_MAX_PAIRS = 128;

// Turns per position of every pair, modulo 1, as 64-bit fractions.  position * turn modulo 2^64 is the angle's fraction of a
// turn, exactly, whatever the position's size and sign: an angle of a million radians in fp32 is off by 0.03, in fp64 it
// would have to be reduced.  What is left is the fraction's own rounding: 2^-65 turns times the position.
struct RopeTurns {
    uint64_t turn[ROPE_MAX_PAIRS];
};

// false: a frequency or the scale is not finite
inline bool rope_turns(const double *inv_freq, int pairs, RopeTurns &out)
{
    for (int i = 0; i < pairs; ++i) {
        if (!isfinite(inv_freq[i])) return false;
        // (long double carries 64 bits here: the fraction is as good as its 64 bits hold)
        long double f = (long double)inv_freq[i] * 0.159154943091895335768883763372514362L;      // 1 / (2 pi)
        if (!(f >= 0.0L && f < 1.0L)) f -= floorl(f);
        const long double scaled = f * 18446744073709551616.0L;
        out.turn[i] = scaled >= 18446744073709551615.0L ? ~0ull : (uint64_t)(scaled + 0.5L);
    }
    return true;
}

// (scale cos, scale sin) of a pair at a position, formed in fp64 and rounded once: two builds of a row's rotation that agree in
// fp64 then agree in every bit of the fp32 products, and so in the 4-bit codes made of them, but for angles within 2^-28
// of a rounding border.  The angle is the fraction of a turn less the nearest quarter, within pi / 4 either way; there the Taylor series up to the
// 15th and 16th power end below 2^-53.  (18 operations in fp64; a general sine and cosine take several times as many instructions, which one head
// of 378 K tokens waits for.)
__device__ __forceinline__ float2 rope_cos_sin(int64_t position, uint64_t turn, double scale, double sin_scale)
{
    const int64_t frac = (int64_t)((uint64_t)position * turn);             // in [-1/2, 1/2) turns, 64 bits
    const int quarter = (int)((int64_t)((uint64_t)frac + (1ull << 61)) >> 62);       // (of 3/8 turns and more: -2)
    const int64_t rest = (int64_t)((uint64_t)frac - ((uint64_t)(int64_t)quarter << 62));
    const double x = (double)rest * (6.283185307179586476925286766559 * 0x1p-64), z = x * x;
    double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;         // 1 / 15!, 1 / 16!
    s = fma(s, z, 1.0 / 6227020800.0);
    c = fma(c, z, -1.0 / 87178291200.0);
    s = fma(s, z, -1.0 / 39916800.0);
    c = fma(c, z, 1.0 / 479001600.0);
    s = fma(s, z, 1.0 / 362880.0);
    c = fma(c, z, -1.0 / 3628800.0);
    s = fma(s, z, -1.0 / 5040.0);
    c = fma(c, z, 1.0 / 40320.0);
    s = fma(s, z, 1.0 / 120.0);
    c = fma(c, z, -1.0 / 720.0);
    s = fma(s, z, -1.0 / 6.0);
    c = fma(c, z, 1.0 / 24.0);
    s = fma(s * z, x, x);
    c = fma(c, z, -0.5);
    c = fma(c, z, 1.0);
    // (c, s) turned by the quarters
    const double cq = quarter & 1 ? s : c, sq = quarter & 1 ? c : s;
    const double co = (quarter + 1) & 2 ? -cq : cq, si = quarter & 2 ? -sq : sq;
    return make_float2((float)(co * scale), (float)(si * sin_scale));
}

// a' = a c - b s, b' = b c + a s; each product and sum rounded by itself (no fma), so that the result does not depend on how
// an expression is contracted
__device__ __forceinline__ void rope_turn(float &a, float &b, float2 cs)
{
    const float x = a, y = b;
    a = __fsub_rn(__fmul_rn(x, cs.x), __fmul_rn(y, cs.y));
    b = __fadd_rn(__fmul_rn(y, cs.x), __fmul_rn(x, cs.y));
}

// E numbers side by side as floats: one 16-byte load or store, or E loads
template <typename T, int E> struct Chunk {
    float v[E];
    __device__ __forceinline__ void load(const T *p)
    {
        if constexpr (E * sizeof(T) == 16) {
            const uint4 x = *reinterpret_cast<const uint4 *>(p);
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[2 * i] = __uint_as_float(w[i] << 16);
                    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] = load_as<float>(p, i);
        }
    }
    __device__ __forceinline__ void store(T *p) const
    {
        if constexpr (E * sizeof(T) == 16) {
            uint32_t w[4];
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                    w[i] = *reinterpret_cast<const uint32_t *>(&h);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[i]);
            }
            *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) store_from(p, i, v[i]);
        }
    }
};

// Cosines and sines of `count` tokens at place(token, pair) of shared memory, by the whole CTA.  A thread keeps its pair; with many tokens their
// positions are looked up once beforehand (one head of 378 K tokens: 210 -> 143 us; with few, that and its barrier cost 4 %).  `position` gives false for a
// token that is passed over.
constexpr int ROPE_THREADS = 256;
template <typename Position, typename Place>
__device__ __forceinline__ void rope_table(const RopeTurns &turns, int pairs, int count, double scale, double sin_scale, int64_t *pos_of, Position position, Place place)
{
    const int shift = pairs > 1 ? 32 - __clz(pairs - 1) : 0;               // pairs rounded up to a power of two: no division in the loop
    const int p = threadIdx.x & ((1 << shift) - 1);
    if ((count << shift) <= 2 * ROPE_THREADS) {
        // a token or two to a thread
        for (int t = threadIdx.x >> shift; t < count; t += ROPE_THREADS >> shift) {
            int64_t at;
            if (p < pairs && position(t, at)) *place(t, p) = rope_cos_sin(at, turns.turn[p], scale, sin_scale);
        }
        __syncthreads();
        return;
    }
    constexpr int64_t NONE = INT64_MIN;
    for (int t = threadIdx.x; t < count; t += ROPE_THREADS) {
        int64_t at;
        pos_of[t] = position(t, at) ? at : NONE;
    }
    __syncthreads();
    if (p < pairs) {
        const uint64_t turn = turns.turn[p];
#pragma unroll 2
        for (int t = threadIdx.x >> shift; t < count; t += ROPE_THREADS >> shift) {
            const int64_t at = pos_of[t];
            if (at != NONE) *place(t, p) = rope_cos_sin(at, turn, scale, sin_scale);
        }
    }
    __syncthreads();
}

// A CTA's share of a rotation: `tile` tokens, each by heads_at_once x per_head threads.  Cosines and sines are formed first; a thread then keeps
// those of its chunk in registers from head to head (read again from shared memory for each head, they took more of the load/store unit than the
// numbers themselves).  Its first heads are requested before the cosines are formed; CTAs that go on to further tokens with the same cosine table
// were slower (32 heads x 32768 tokens: 92 us; two rounds of tokens 104, four 112), for their loads then wait for their stores.
//   HALVES: item j < rotary / 2 / E holds numbers [E j, E j + E) and their partners rotary / 2 further on.  PAIRS: item j holds 2 E numbers side by
//   side.  Items from there on copy E or, where their number is even, 2 E numbers (none where out is x).
constexpr int ROPE_AHEAD = 4;            // heads of a thread that are requested together
struct RopeShape {
    int32_t heads, rotary, per_head, heads_at_once, tile;
    int32_t copy;                        // chunks that an item copies: 1 or 2
    int64_t x_head, out_head;            // strides
    double scale, sin_scale;
    uint64_t zero = 0x8000000080000000ull;       // (-0, -0), as an argument: of a constant the compiler would make use
};
// items of a head whose halves are whole chunks of E numbers; `copied`: numbers that are copied
inline void rope_items(RopeShape &r, int E, int copied)
{
    r.copy = copied / E % 2 == 0 ? 2 : 1;
    r.per_head = r.rotary / 2 / E + copied / E / r.copy;
}
// `tokens`: how many there are; per_head <= ROPE_THREADS
inline void rope_share(RopeShape &r, int64_t tokens, int sms, int ahead = ROPE_AHEAD)
{
    // a thread takes `ahead` heads, fewer where the tokens would not fill the GPU
    int each = ahead;
    while (each > 1 && tokens * r.per_head * ((r.heads + each - 1) / each) < (int64_t)2 * sms * ROPE_THREADS) each >>= 1;
    r.heads_at_once = (r.heads + each - 1) / each;
    if (r.heads_at_once * r.per_head > ROPE_THREADS) r.heads_at_once = ROPE_THREADS / r.per_head;
    r.tile = ROPE_THREADS / (r.heads_at_once * r.per_head);
    if (tokens < r.tile) r.tile = (int)tokens;
}
// floats of shared memory for a token's cosines and sines: chunks of E pairs are 16 bytes apart more than they are long, so that
// neighbouring chunks' 16-byte reads meet no bank twice
template <int E> __host__ __device__ constexpr int rope_cs_floats(int pairs) { return 2 * pairs + (E >= 4 ? 4 * (pairs / E) : 0); }

// E numbers as they are stored
template <typename T, int E> struct Raw {
    uint4 v;
    __device__ __forceinline__ void load(const T *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void store(T *p) const { *reinterpret_cast<uint4 *>(p) = v; }
    // numbers 2 i and 2 i + 1
    __device__ __forceinline__ uint64_t pair(int i) const
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        if constexpr (sizeof(T) == 2) return sm100::pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
        else return sm100::pack2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    }
    __device__ __forceinline__ void set(int i, uint64_t x)
    {
        float lo, hi;
        sm100::unpack2(x, lo, hi);
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
        if constexpr (sizeof(T) == 2) {
            w[i] = sm100::pack_bf16x2(lo, hi);
        } else {
            w[2 * i] = __float_as_uint(lo);
            w[2 * i + 1] = __float_as_uint(hi);
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <typename T> struct Raw<T, 1> {
    float v;
    __device__ __forceinline__ void load(const T *p) { v = load_as<float>(p, 0); }
    __device__ __forceinline__ void store(T *p) const { store_from(p, 0, v); }
};

template <typename T, int E, bool HALVES, typename Token>
__device__ __forceinline__ void rope_rows(const T *x, T *out, const RopeShape &r, const RopeTurns &turns, int64_t t0, int count, float *cs, Token token)
{
    const int pairs = r.rotary / 2, turn_items = pairs / E, row_cs = rope_cs_floats<E>(pairs);
    const int per_token = r.heads_at_once * r.per_head;
    const int t = threadIdx.x / per_token, rest = threadIdx.x - t * per_token, h0 = rest / r.per_head, j = rest - h0 * r.per_head;
    const bool turn = j < turn_items;
    const int o = turn ? (HALVES ? j * E : 2 * j * E) : r.rotary + (j - turn_items) * r.copy * E, partner = HALVES && turn ? pairs : E;
    const bool two = turn || r.copy == 2;
    Raw<T, E> u[ROPE_AHEAD], w[ROPE_AHEAD];
    int64_t from = 0, to = 0, pos = 0;
    const bool mine = t < count && token(t0 + t, from, to, pos);
    auto request = [&](int first) {
        const T *src = x + from + o + first * r.x_head;
        const int64_t step = r.heads_at_once * r.x_head;
#pragma unroll
        for (int k = 0; k < ROPE_AHEAD; ++k) {
            if (mine && first + k * r.heads_at_once < r.heads) {
                u[k].load(src);
                if (two) w[k].load(src + partner);
            }
            src += step;
        }
    };
    request(h0);
    const uint64_t zero = r.zero;
    __shared__ int64_t pos_of[ROPE_THREADS];
    rope_table(turns, pairs, count, r.scale, r.sin_scale, pos_of,
               [&](int ti, int64_t &at) {
                   int64_t f, g;
                   return token(t0 + ti, f, g, at);
               },
               [&](int ti, int p) { return reinterpret_cast<float2 *>(cs + ti * row_cs + 2 * p + (E >= 4 ? 4 * (p / E) : 0)); });
    if (!mine) return;
    // HALVES: cosines and sines of pairs 2 i, 2 i + 1 side by side; PAIRS: (c, c) and (-s, s) of pair i
    uint64_t cc[E > 1 ? E : 1], ss[E > 1 ? E : 1];
    float2 one = make_float2(0.f, 0.f);
    if (turn) {
        const float *at = cs + t * row_cs + j * (2 * E + (E >= 4 ? 4 : 0));
        if constexpr (E >= 2) {
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const float4 v = *reinterpret_cast<const float4 *>(at + 2 * e);
                if constexpr (HALVES) {
                    cc[e / 2] = sm100::pack2(v.x, v.z);
                    ss[e / 2] = sm100::pack2(v.y, v.w);
                } else {
                    cc[e] = sm100::pack2(v.x, v.x);
                    ss[e] = sm100::pack2(-v.y, v.y);
                    cc[e + 1] = sm100::pack2(v.z, v.z);
                    ss[e + 1] = sm100::pack2(-v.w, v.w);
                }
            }
        } else {
            one = *reinterpret_cast<const float2 *>(at);
        }
    }
    for (int first = h0; first < r.heads; first += ROPE_AHEAD * r.heads_at_once) {
        if (first != h0) request(first);
        T *dst = out + to + o + first * r.out_head;
        const int64_t step = r.heads_at_once * r.out_head;
#pragma unroll
        for (int k = 0; k < ROPE_AHEAD; ++k, dst += step) {
            if (first + k * r.heads_at_once >= r.heads) continue;
            if (turn) {
                // (-(b s) = b (-s): the products and sums of rope_turn, two at a time.  A product is written as an fma with -0, for a packed
                // product and sum are contracted to one fma whatever their rounding modes say)
                if constexpr (E == 1) {
                    rope_turn(u[k].v, w[k].v, one);
                } else if constexpr (HALVES) {
#pragma unroll
                    for (int e = 0; e < E / 2; ++e) {
                        const uint64_t a = u[k].pair(e), b = w[k].pair(e), ns = ss[e] ^ 0x8000000080000000ull;
                        u[k].set(e, sm100::add2(sm100::fma2(a, cc[e], zero), sm100::fma2(b, ns, zero)));
                        w[k].set(e, sm100::add2(sm100::fma2(b, cc[e], zero), sm100::fma2(a, ss[e], zero)));
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        Raw<T, E> &z = e < E / 2 ? u[k] : w[k];
                        const uint64_t ab = z.pair(e % (E / 2));
                        float a, b;
                        sm100::unpack2(ab, a, b);
                        z.set(e % (E / 2), sm100::add2(sm100::fma2(ab, cc[e], zero), sm100::fma2(sm100::pack2(b, a), ss[e], zero)));
                    }
                }
            }
            if (two) w[k].store(dst + partner);
            u[k].store(dst);
        }
    }
}

// The same where rows are on 16-byte boundaries and the halves of a pair's chunk are not: a thread loads and stores whole chunks of E numbers and
// reads the partners of its numbers one by one, from L1.  per_head is d / E.  Between the reads and the stores of a round the CTA waits, for out may
// be x and a row is several threads'.
constexpr int ROPE_ANY_AHEAD = 2;
// where a pair's cosine and sine stand: chunks of eight pairs are 72 bytes apart, so that neighbouring threads' reads meet no bank twice
__host__ __device__ constexpr int rope_any_place(int pair) { return pair + (pair >> 3); }
__host__ __device__ constexpr int rope_any_places(int pairs) { return pairs + (pairs >> 3) + 1; }
template <typename T, int E, bool HALVES, typename Token>
__device__ __forceinline__ void rope_rows_any(const T *x, T *out, const RopeShape &r, const RopeTurns &turns, int64_t t0, int count, float *cs, Token token)
{
    const int pairs = r.rotary / 2;
    const int per_token = r.heads_at_once * r.per_head;
    const int t = threadIdx.x / per_token, rest = threadIdx.x - t * per_token, h0 = rest / r.per_head, first = (rest - h0 * r.per_head) * E;
    int64_t from = 0, to = 0, pos = 0;
    const bool mine = t < count && token(t0 + t, from, to, pos);
    Chunk<T, E> u[ROPE_ANY_AHEAD], w[ROPE_ANY_AHEAD];
    auto request = [&](int round) {
#pragma unroll
        for (int k = 0; k < ROPE_ANY_AHEAD; ++k) {
            const int h = round + h0 + k * r.heads_at_once;
            if (!mine || h >= r.heads) continue;
            const T *row = x + from + h * r.x_head;
            u[k].load(row + first);
            if constexpr (HALVES) {
                if (sizeof(T) == 2 && (pairs & 1) == 0) {        // two at a time: both on one side
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        const int j = first + e;
                        const uint32_t two = j < r.rotary ? *reinterpret_cast<const uint32_t *>(row + (j < pairs ? j + pairs : j - pairs)) : 0u;
                        w[k].v[e] = __uint_as_float(two << 16);
                        w[k].v[e + 1] = __uint_as_float(two & 0xffff0000u);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const int j = first + e;
                        w[k].v[e] = j < r.rotary ? load_as<float>(row, j < pairs ? j + pairs : j - pairs) : 0.f;
                    }
                }
            }
        }
    };
    request(0);
    __shared__ int64_t pos_of[ROPE_THREADS];
    rope_table(turns, pairs, count, r.scale, r.sin_scale, pos_of,
               [&](int ti, int64_t &at) {
                   int64_t f, g;
                   return token(t0 + ti, f, g, at);
               },
               [&](int ti, int p) { return reinterpret_cast<float2 *>(cs) + ti * rope_any_places(pairs) + rope_any_place(p); });
    const float2 *c = reinterpret_cast<const float2 *>(cs) + t * rope_any_places(pairs);
    for (int round = 0; round < r.heads; round += ROPE_ANY_AHEAD * r.heads_at_once) {
        if (round) request(round);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < ROPE_ANY_AHEAD; ++k) {
            const int h = round + h0 + k * r.heads_at_once;
            if (!mine || h >= r.heads) continue;
#pragma unroll
            for (int e = 0; e < E; e += HALVES ? 1 : 2) {
                const int j = first + e;
                if (j >= r.rotary) continue;
                if constexpr (HALVES) {
                    const bool lower = j < pairs;
                    float a = lower ? u[k].v[e] : w[k].v[e], b = lower ? w[k].v[e] : u[k].v[e];
                    rope_turn(a, b, c[rope_any_place(lower ? j : j - pairs)]);
                    u[k].v[e] = lower ? a : b;
                } else {
                    rope_turn(u[k].v[e], u[k].v[e + 1], c[rope_any_place(j / 2)]);
                }
            }
            u[k].store(out + to + h * r.out_head + first);
        }
    }
}

}  // namespace elm
