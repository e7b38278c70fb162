// Rotary positions (elm_rope, elm_rope_frequencies).
//
//   a' = a c - b s,  b' = b c + a s,  (c, s) = scale (cos, sin)(position * inv_freq[i])
//
// One pass over X: HBM-bound (2 d numbers moved per head and token).  A CTA takes a few tokens: its threads first form the
// tokens' cosines and sines once for all heads (fp64, see elm_rope.cuh), then walk over (token, head, chunk), 16 bytes of each half of
// a pair per thread.
#include "elm_rope.cuh"

namespace elm {
namespace {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_TILE = 128;           // tokens of a CTA at most
constexpr int ROPE_UNROLL = 4;           // chunks (pairs of chunks) a thread has in flight

struct RopeArgs {
    const void *x;
    void *out;
    const int32_t *positions;
    int64_t first;
    int64_t xs[3], os[3];
    double scale, sin_scale;
    int32_t heads, n_tokens, d, rotary, tile, copy_chunks;
    int64_t tokens;                      // batch * n_tokens
};

// HALVES: item j < rotary / 2 / E holds numbers [E j, E j + E) and their partners rotary / 2 further on.  PAIRS: item j holds
// 2 E numbers side by side.  Items from there on copy E numbers (copy_chunks of them; none when out is X).
template <typename T, int E, bool HALVES>
__global__ void __launch_bounds__(ROPE_THREADS) rope_kernel(const __grid_constant__ RopeArgs a, const __grid_constant__ RopeTurns turns)
{
    __shared__ int64_t row_of[ROPE_TILE][2];                   // a token's first row in X and in out
    extern __shared__ float2 cs[];                             // [tile][rotary / 2]
    const int pairs = a.rotary / 2;
    const int64_t t0 = (int64_t)blockIdx.x * a.tile;
    const int count = (int)(a.tokens - t0 < a.tile ? a.tokens - t0 : a.tile);
    for (int i = threadIdx.x; i < count * pairs; i += ROPE_THREADS) {
        const int t = i / pairs, p = i - t * pairs;
        const int64_t pos = a.positions ? (int64_t)a.positions[t0 + t] : a.first + (t0 + t) % a.n_tokens;
        cs[i] = rope_cos_sin(pos, turns.turn[p], a.scale, a.sin_scale);
    }
    for (int t = threadIdx.x; t < count; t += ROPE_THREADS) {
        const int64_t b = (t0 + t) / a.n_tokens, n = (t0 + t) - b * a.n_tokens;
        row_of[t][0] = b * a.xs[0] + n * a.xs[2];
        row_of[t][1] = b * a.os[0] + n * a.os[2];
    }
    __syncthreads();
    const int turn_items = pairs / E;
    const int per_head = turn_items + a.copy_chunks;
    const int per_token = per_head * a.heads;
    const int total = count * per_token;
    const T *x = (const T *)a.x;
    T *out = (T *)a.out;
    for (int i0 = threadIdx.x; i0 < total; i0 += ROPE_THREADS * ROPE_UNROLL) {
        Chunk<T, E> u[ROPE_UNROLL], w[ROPE_UNROLL];
        int64_t to[ROPE_UNROLL];
        int kind[ROPE_UNROLL];                                 // first pair of the item, -1: copied, -2: none
#pragma unroll
        for (int k = 0; k < ROPE_UNROLL; ++k) {
            const int i = i0 + k * ROPE_THREADS;
            kind[k] = -2;
            if (i < total) {
                const int t = i / per_token, r = i - t * per_token;
                const int h = r / per_head, j = r - h * per_head;
                const int64_t from = row_of[t][0] + h * a.xs[1];
                to[k] = row_of[t][1] + h * a.os[1];
                if (j < turn_items) {
                    kind[k] = t * pairs + j * E;
                    const int o = HALVES ? j * E : 2 * j * E;
                    to[k] += o;
                    u[k].load(x + from + o);
                    w[k].load(x + from + o + (HALVES ? pairs : E));
                } else {
                    kind[k] = -1;
                    const int o = a.rotary + (j - turn_items) * E;
                    to[k] += o;
                    u[k].load(x + from + o);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < ROPE_UNROLL; ++k) {
            if (kind[k] >= 0) {
                const float2 *c = cs + kind[k];
                if constexpr (HALVES) {
#pragma unroll
                    for (int e = 0; e < E; ++e) rope_turn(u[k].v[e], w[k].v[e], c[e]);
                } else if constexpr (E == 1) {
                    rope_turn(u[k].v[0], w[k].v[0], c[0]);
                } else {
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        rope_turn(u[k].v[e], u[k].v[e + 1], c[e / 2]);
                        rope_turn(w[k].v[e], w[k].v[e + 1], c[E / 2 + e / 2]);
                    }
                }
                u[k].store(out + to[k]);
                w[k].store(out + to[k] + (HALVES ? pairs : E));
            } else if (kind[k] == -1) {
                u[k].store(out + to[k]);
            }
        }
    }
}

template <typename T, int E> int launch_rope(RopeArgs &a, const RopeTurns &turns, bool halves, bool in_place, cudaStream_t st)
{
    a.copy_chunks = in_place ? 0 : (a.d - a.rotary) / E;
    const int pairs = a.rotary / 2;
    // tokens per CTA: about two rounds of its threads' chunks (cosines of a token cost as much as a few chunks, so that one
    // token of one head alone is dear), as few as that where the tokens would not fill the GPU
    const int per_token = (pairs / E + a.copy_chunks) * a.heads;
    int tile = (2 * ROPE_THREADS * ROPE_UNROLL + per_token - 1) / per_token;
    const int64_t fill = a.tokens / (4 * (int64_t)device_sm_count());
    if (tile > fill) tile = fill < 1 ? 1 : (int)fill;
    const int most = 32768 / (pairs * (int)sizeof(float2));
    if (tile > most) tile = most;
    if (tile > ROPE_TILE) tile = ROPE_TILE;
    a.tile = tile;
    const int64_t ctas = (a.tokens + tile - 1) / tile;
    if (ctas > 0x7fffffff) return ELM_ERR_SHAPE;
    const size_t smem = (size_t)tile * pairs * sizeof(float2);
    if (halves) rope_kernel<T, E, true><<<(unsigned)ctas, ROPE_THREADS, smem, st>>>(a, turns);
    else rope_kernel<T, E, false><<<(unsigned)ctas, ROPE_THREADS, smem, st>>>(a, turns);
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
    int64_t all = 0;
    for (int i = 0; i < 3; ++i) {
        a.xs[i] = zeros(p->x_stride) ? dense[i] : p->x_stride[i];
        a.os[i] = zeros(p->out_stride) ? dense[i] : p->out_stride[i];
        all |= a.xs[i] | a.os[i];
    }
    // rows of out that would be written twice
    if ((p->batch > 1 && a.os[0] == 0) || (p->heads > 1 && a.os[1] == 0) || (p->n_tokens > 1 && a.os[2] == 0)) return ELM_ERR_SHAPE;
    const bool in_place = X == out;
    if (in_place)
        for (int i = 0; i < 3; ++i)
            if (a.xs[i] != a.os[i]) return ELM_ERR_SHAPE;
    const int item = (int)elt_bytes(p->dtype);
    if (((uintptr_t)X | (uintptr_t)out) & (item - 1)) return ELM_ERR_ALIGN;
    if (positions && ((uintptr_t)positions & 3)) return ELM_ERR_ALIGN;
    a.x = X;
    a.out = out;
    a.positions = positions;
    a.first = first_position;
    a.scale = p->scale;
    a.sin_scale = p->inverse ? -p->scale : p->scale;
    a.heads = p->heads;
    a.n_tokens = p->n_tokens;
    a.d = p->d;
    a.rotary = p->rotary_dim;
    a.tokens = (int64_t)p->batch * p->n_tokens;
    cudaStream_t st = (cudaStream_t)stream;
    const bool halves = p->layout == ELM_ROPE_HALVES;
    // 16 bytes at a time where every chunk starts on a 16-byte boundary and both numbers of a pair lie in whole chunks
    const int E = 16 / item;
    const bool wide = !(((uintptr_t)X | (uintptr_t)out) & 15) && all % E == 0 && p->d % E == 0 && p->rotary_dim / 2 % E == 0;
    if (p->dtype == ELM_BF16)
        return wide ? launch_rope<__nv_bfloat16, 8>(a, turns, halves, in_place, st) : launch_rope<__nv_bfloat16, 1>(a, turns, halves, in_place, st);
    return wide ? launch_rope<float, 4>(a, turns, halves, in_place, st) : launch_rope<float, 1>(a, turns, halves, in_place, st);
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
