// Rows held in 4 bits: their layout, and how codes and scales are made and read.
#pragma once
#include <cuda_fp16.h>

#include "elm_common.cuh"

namespace elm {

constexpr int C4_GROUP = 16;                                     // numbers that share a scale

// A row: codes of the key, codes of the value, scales of the key, scales of the value.  Key and value stand together because no reader
// wants one without the other: a row of 144 bytes is nine 16-byte copies from five sectors, where four arrays of codes and scales
// would take six sectors of a row that stands alone.  (d = 64: padded to whole 16-byte chunks.)
template <int D> struct Row4 {
    static constexpr int CODES = D / 2;                          // bytes of a key's codes, and of a value's
    static constexpr int GROUPS = D / C4_GROUP;                  // scales of a key, and of a value
    static constexpr int SCALES = 2 * CODES;                     // offset of the scales
    static constexpr int BYTES = (2 * CODES + 2 * GROUPS + 15) / 16 * 16;
    static constexpr int CHUNKS = BYTES / 16;
};
inline int row4_bytes(int d) { return d == 64 ? Row4<64>::BYTES : Row4<128>::BYTES; }

// Where the pool's rows are.  Every number that comes from the caller's tables is checked before it becomes an address: a bad page
// is a row that is not there.
struct Pool4 {
    const unsigned char *rows;
    const int32_t *table;
    int32_t n_pages, max_pages, page_shift, kv_heads;
};
constexpr uint32_t NO_ROW = 0xffffffffu;
// number of the pool's row that holds row r (>= 0) of request b and KV head h
__device__ __forceinline__ uint32_t pool_row(const Pool4 &p, int b, int h, int64_t r)
{
    const int64_t entry = r >> p.page_shift;
    if (r < 0 || entry >= p.max_pages) return NO_ROW;
    const int32_t page = p.table[(int64_t)b * p.max_pages + entry];
    if ((uint32_t)page >= (uint32_t)p.n_pages) return NO_ROW;
    return (((uint32_t)page * (uint32_t)p.kv_heads + (uint32_t)h) << p.page_shift) + ((uint32_t)r & ((1u << p.page_shift) - 1u));
}

inline int page_shift_of(int page_rows)                          // -1: not a size of page
{
    if (page_rows < 16 || page_rows > 1024 || (page_rows & (page_rows - 1))) return -1;
    int s = 4;
    while ((1 << s) < page_rows) ++s;
    return s;
}
inline bool pool_fits(int n_pages, int page_rows, int kv_heads)
{
    const int64_t rows = (int64_t)n_pages * page_rows;
    return n_pages >= 1 && kv_heads >= 1 && rows <= 0x7fffffff && rows * kv_heads < 0xffffffffll;
}

// the scale's byte as fp16: sign left out, 5 exponent and 3 mantissa bits in the places of an fp16 number's upper ones
__device__ __forceinline__ uint32_t scale4_half_bits(uint32_t byte) { return byte << 7; }
// two of them side by side (products: the units that shift and convert have more to do than those that multiply)
__device__ __forceinline__ uint32_t scale4_half2(uint32_t low, uint32_t high) { return low * 0x80u + high * 0x800000u; }
__device__ __forceinline__ uint32_t scale4_half2(uint32_t both) { return both * 0x00800080u; }

// The eight codes of a word as pairs of fp16 numbers, the lower half of each byte first.  Codes are at most 6, scales at most 10240 with 4 bits, products
// have 6 bits and are at most 61440: fp16 holds them exactly, and so does bf16.
__device__ __forceinline__ void codes8_to_half2(uint32_t word, uint32_t (&out)[4])
{
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(out[0]), "=r"(out[1]), "=r"(out[2]), "=r"(out[3]) : "r"(word));
}
__device__ __forceinline__ uint32_t hmul2_bits(uint32_t a, uint32_t b)
{
    const __half2 r = __hmul2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}

// The 16 numbers of a group as 8 bytes of codes; the scale's byte is returned.
//   scale = nearest (ties to even) to max |x| / 6 of the numbers with 4 significant bits (multiples of 2^-17 below 2^-14), at most
//   10240; a code is the nearest (ties to even) E2M1 number to x / scale.
// x / scale is formed from the correctly rounded reciprocal r by q = x r, q + r (x - q scale): correctly rounded for every quotient that
// matters (Markstein 1990), so that a number halfway between two codes is seen as that - a product with the rounded reciprocal
// alone would put half of those to the wrong side, and of bf16 numbers one in a hundred is a tie.
__device__ __forceinline__ float max_nan(float a, float b)      // NaN if either is
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint32_t quantise4(float (&x)[C4_GROUP], uint2 &codes)
{
    constexpr float LARGEST = 61440.f;
    float top = fabsf(x[0]);
#pragma unroll
    for (int i = 1; i < C4_GROUP; ++i) top = max_nan(top, fabsf(x[i]));
    if (!(top <= LARGEST)) {
        if (top != top) {
            codes = make_uint2(0u, 0u);
            return 0xffu;                                                       // fp16 NaN times any code
        }
#pragma unroll
        for (int i = 0; i < C4_GROUP; ++i) x[i] = fminf(fmaxf(x[i], -LARGEST), LARGEST);
        top = LARGEST;
    }
    const float q = __fdiv_rn(top, 6.f);
    uint32_t byte;
    if (q >= 0x1p-14f) {
        const uint32_t u = __float_as_uint(q);
        byte = ((u + 0x7ffffu + ((u >> 20) & 1u)) >> 20) - (112u << 3);
    } else {
        byte = (uint32_t)__float2int_rn(q * 131072.f);
    }
    const float s = __half2float(__ushort_as_half((unsigned short)scale4_half_bits(byte)));
    const float r = byte ? __fdiv_rn(1.f, s) : 0.f;
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < C4_GROUP; i += 2) {
        float y[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float y0 = x[i + k] * r;
            y[k] = copysignf(fmaf(fmaf(-y0, s, x[i + k]), r, y0), x[i + k]);    // (-0 stays -0)
        }
        uint32_t two;
        asm("{\n\t.reg .b8 b;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %1, %2;\n\tcvt.u32.u8 %0, b;\n\t}" : "=r"(two) : "f"(y[1]), "f"(y[0]));
        w[i >> 3] |= two << (4 * (i & 7));
    }
    codes = make_uint2(w[0], w[1]);
    return byte;
}

}  // namespace elm
