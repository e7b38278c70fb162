// Rotary positions (elm_rope, elm_rope_frequencies).
//
//   a' = a c - b s,  b' = b c + a s,  (c, s) = scale (cos, sin)(position * inv_freq[i])
//
// One pass over X: HBM-bound (2 d numbers moved per head and token; 32 heads x 32768 tokens x 128 in bf16: 83 us in halves, 88 in pairs, for a floor of
// 82).  A CTA takes a few tokens; cosines and sines are formed once for all heads of a token (fp64, see elm_rope.cuh), which few heads wait for: one head of
// 378 K tokens 142 us for a floor of 30.
#include "elm_rope.cuh"

namespace elm {
namespace {

struct RopeArgs {
    const void *x;
    void *out;
    const int32_t *positions;
    int64_t first;
    int64_t xs[2], os[2];                // batch, token
    RopeShape shape;
    int32_t n_tokens;
    int64_t tokens;                      // batch * n_tokens
};

// WHOLE: the halves of a pair's chunk are whole chunks (or E is 1)
template <typename T, int E, bool HALVES, bool WHOLE>
__global__ void __launch_bounds__(ROPE_THREADS, 3) rope_kernel(const __grid_constant__ RopeArgs a, const __grid_constant__ RopeTurns turns)
{
    extern __shared__ __align__(16) float cs[];
    cudaGridDependencySynchronize();
    const int64_t t0 = (int64_t)blockIdx.x * a.shape.tile;
    const int count = (int)(a.tokens - t0 < a.shape.tile ? a.tokens - t0 : a.shape.tile);
    auto token = [&](int64_t t, int64_t &from, int64_t &to, int64_t &pos) {
        const uint32_t b = (uint32_t)t / (uint32_t)a.n_tokens, n = (uint32_t)t - b * (uint32_t)a.n_tokens;
        from = b * a.xs[0] + n * a.xs[1];
        to = b * a.os[0] + n * a.os[1];
        pos = a.positions ? (int64_t)a.positions[t] : a.first + n;
        return true;
    };
    if constexpr (WHOLE) rope_rows<T, E, HALVES>((const T *)a.x, (T *)a.out, a.shape, turns, t0, count, cs, token);
    else rope_rows_any<T, E, HALVES>((const T *)a.x, (T *)a.out, a.shape, turns, t0, count, cs, token);
}

template <typename T, int E, bool WHOLE> int launch_rope(RopeArgs &a, int d, const RopeTurns &turns, bool halves, bool in_place, cudaStream_t st)
{
    const int pairs = a.shape.rotary / 2;
    if (WHOLE) rope_items(a.shape, E, in_place ? 0 : d - a.shape.rotary);
    else a.shape.per_head = d / E;
    rope_share(a.shape, a.tokens, device_sm_count(), WHOLE ? ROPE_AHEAD : ROPE_ANY_AHEAD);
    const int64_t ctas = (a.tokens + a.shape.tile - 1) / a.shape.tile;
    if (ctas > 0x7fffffff) return ELM_ERR_SHAPE;
    const size_t smem = (size_t)a.shape.tile * (WHOLE ? rope_cs_floats<E>(pairs) : 2 * rope_any_places(pairs)) * sizeof(float);
    auto kern = halves ? rope_kernel<T, E, true, WHOLE> : rope_kernel<T, E, false, WHOLE>;
    ELM_CUDA_TRY(launch_after(kern, dim3((unsigned)ctas), dim3(ROPE_THREADS), smem, st, a, turns));
    count_launches(1);
    return cuda_status(cudaGetLastError());
}

bool zeros(const int64_t (&s)[3]) { return s[0] == 0 && s[1] == 0 && s[2] == 0; }

}  // namespace
}  // namespace elm

using namespace elm;

extern "C" int elm_rope(const void *X, const int32_t *positions, int64_t first_position, const elm_rope_params *p, void *out, void *stream)
{
    if (!p || !X || !out || !p->inv_freq) return ELM_ERR_NULL;
    if (p->dtype != ELM_F32 && p->dtype != ELM_BF16) return ELM_ERR_DTYPE;
    if (p->batch < 1 || p->heads < 1 || p->n_tokens < 1 || p->d < 2 || p->d > 2 * ROPE_MAX_PAIRS || (p->d & 1)) return ELM_ERR_SHAPE;
    if (p->rotary_dim < 2 || p->rotary_dim > p->d || (p->rotary_dim & 1)) return ELM_ERR_SHAPE;
    if (p->layout != ELM_ROPE_HALVES && p->layout != ELM_ROPE_PAIRS) return ELM_ERR_SHAPE;
    if (p->heads > 65535 || (int64_t)p->batch * p->n_tokens > 0x7fffffff) return ELM_ERR_SHAPE;
    if (!isfinite(p->scale)) return ELM_ERR_SHAPE;
    RopeTurns turns;
    if (!rope_turns(p->inv_freq, p->rotary_dim / 2, turns)) return ELM_ERR_SHAPE;
    RopeArgs a;
    const int64_t dense[3] = {(int64_t)p->heads * p->n_tokens * p->d, (int64_t)p->n_tokens * p->d, p->d};
    int64_t xs[3], os[3], all = 0;
    for (int i = 0; i < 3; ++i) {
        xs[i] = zeros(p->x_stride) ? dense[i] : p->x_stride[i];
        os[i] = zeros(p->out_stride) ? dense[i] : p->out_stride[i];
        all |= xs[i] | os[i];
    }
    // rows of out that would be written twice
    if ((p->batch > 1 && os[0] == 0) || (p->heads > 1 && os[1] == 0) || (p->n_tokens > 1 && os[2] == 0)) return ELM_ERR_SHAPE;
    const bool in_place = X == out;
    if (in_place)
        for (int i = 0; i < 3; ++i)
            if (xs[i] != os[i]) return ELM_ERR_SHAPE;
    const int item = (int)elt_bytes(p->dtype);
    if (((uintptr_t)X | (uintptr_t)out) & (item - 1)) return ELM_ERR_ALIGN;
    if (positions && ((uintptr_t)positions & 3)) return ELM_ERR_ALIGN;
    a.x = X;
    a.out = out;
    a.positions = positions;
    a.first = first_position;
    for (int i = 0; i < 2; ++i) {
        a.xs[i] = xs[2 * i];
        a.os[i] = os[2 * i];
    }
    a.shape = RopeShape{p->heads, p->rotary_dim, 0, 0, 0, 1, xs[1], os[1], p->scale, p->inverse ? -p->scale : p->scale};
    a.n_tokens = p->n_tokens;
    a.tokens = (int64_t)p->batch * p->n_tokens;
    cudaStream_t st = (cudaStream_t)stream;
    const bool halves = p->layout == ELM_ROPE_HALVES;
    // 16 bytes at a time where every row starts on a 16-byte boundary
    const int E = 16 / item;
    const bool wide = !(((uintptr_t)X | (uintptr_t)out) & 15) && all % E == 0 && p->d % E == 0, whole = p->rotary_dim / 2 % E == 0;
    typedef __nv_bfloat16 bf;
    if (p->dtype == ELM_BF16)
        return !wide ? launch_rope<bf, 1, true>(a, p->d, turns, halves, in_place, st)
               : whole ? launch_rope<bf, 8, true>(a, p->d, turns, halves, in_place, st) : launch_rope<bf, 8, false>(a, p->d, turns, halves, in_place, st);
    return !wide ? launch_rope<float, 1, true>(a, p->d, turns, halves, in_place, st)
           : whole ? launch_rope<float, 4, true>(a, p->d, turns, halves, in_place, st) : launch_rope<float, 4, false>(a, p->d, turns, halves, in_place, st);
}

extern "C" int elm_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double original, double low, double high,
                                    double *inv_freq_host, double *scale_host)
{
    if (!inv_freq_host || !scale_host) return ELM_ERR_NULL;
    if (rotary_dim < 2 || rotary_dim > 2 * ROPE_MAX_PAIRS || (rotary_dim & 1)) return ELM_ERR_SHAPE;
    if (!(base > 1.0) || !isfinite(base)) return ELM_ERR_SHAPE;
    if (scaling < ELM_ROPE_PLAIN || scaling > ELM_ROPE_SMOOTH) return ELM_ERR_SHAPE;
    if (scaling != ELM_ROPE_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return ELM_ERR_SHAPE;
    if (scaling >= ELM_ROPE_RAMP && (!(original > 0.0) || !(low > 0.0) || !(high > low) || !isfinite(original) || !isfinite(high))) return ELM_ERR_SHAPE;
    if (scaling == ELM_ROPE_BASE && rotary_dim == 2) return ELM_ERR_SHAPE;
    const double r = rotary_dim, two_pi = 6.283185307179586;
    if (scaling == ELM_ROPE_BASE) base *= pow(factor, r / (r - 2.0));
    // RAMP: the pair that makes t turns over `original` positions is number r ln(original / (2 pi t)) / (2 ln base)
    double first = 0.0, last = 0.0;
    if (scaling == ELM_ROPE_RAMP) {
        first = fmax(0.0, floor(r * log(original / (two_pi * high)) / (2.0 * log(base))));
        last = fmin(r - 1.0, ceil(r * log(original / (two_pi * low)) / (2.0 * log(base))));
    }
    for (int i = 0; i < rotary_dim / 2; ++i) {
        const double f = pow(base, -2.0 * i / r);
        double keep = 1.0;
        if (scaling == ELM_ROPE_LINEAR) keep = 0.0;
        else if (scaling == ELM_ROPE_RAMP) keep = 1.0 - fmin(1.0, fmax(0.0, (i - first) / fmax(last - first, 0.001)));
        else if (scaling == ELM_ROPE_SMOOTH) keep = fmin(1.0, fmax(0.0, (original * f / two_pi - low) / (high - low)));
        inv_freq_host[i] = keep == 1.0 ? f : f * keep + f / factor * (1.0 - keep);
    }
    *scale_host = scaling == ELM_ROPE_RAMP ? 0.1 * log(factor) + 1.0 : 1.0;
    return ELM_OK;
}
