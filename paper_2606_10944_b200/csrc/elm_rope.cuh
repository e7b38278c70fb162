// Rotary positions: what the rotation kernel and the kernel that stores rows in 4 bits share.
#pragma once
#include <math.h>

#include "elm_common.cuh"

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
        long double f = (long double)inv_freq[i] / 6.283185307179586476925286766559005768L;
        f -= floorl(f);
        const long double scaled = f * 18446744073709551616.0L;
        out.turn[i] = scaled >= 18446744073709551615.0L ? ~0ull : (uint64_t)(scaled + 0.5L);
    }
    return true;
}

// (scale cos, scale sin) of a pair at a position, formed in fp64 and rounded once: two builds of a row's rotation that agree in
// fp64 then agree in every bit of the fp32 products, and so in the 4-bit codes made of them, but for angles within 2^-28
// of a rounding border.
__device__ __forceinline__ float2 rope_cos_sin(int64_t position, uint64_t turn, double scale, double sin_scale)
{
    const int64_t frac = (int64_t)((uint64_t)position * turn);             // in [-1/2, 1/2) turns
    double s, c;
    sincospi((double)frac * 0x1p-63, &s, &c);
    return make_float2((float)(c * scale), (float)(s * sin_scale));
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

}  // namespace elm
