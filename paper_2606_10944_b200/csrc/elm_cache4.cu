// New tokens into a pool of rows held in 4 bits (elm_cache4_append), and rows back (elm_cache4_read).
//
// Both are one pass over their rows.  Append reads 2 d numbers per token and KV head and writes a row (144 bytes at d = 128), besides the queries'
// 2 d per query head; read the other way round.  Bound by the launch in a decode step (16 tokens: 8 us the two), by HBM and the latency of a CTA's one round in
// long ones (10 K tokens of 32 + 8 + 8 heads, 222 MB: 46 us = 4.8 TB/s; rows back, 178 MB written: 32 us = 5.6 TB/s).
#include "elm_cache4.cuh"
#include "elm_rope.cuh"

namespace elm {
namespace {

constexpr int APP_THREADS = ROPE_THREADS;

struct AppendArgs {
    const void *q, *k, *v;
    void *q_out;
    const int32_t *positions, *slots;
    unsigned char *rows;
    int64_t qs[2], ks[2], vs[2], qos[2];
    RopeShape query;                     // of the CTAs that turn queries
    double scale;
    int32_t n_tokens, q_heads, kv_heads, rotary, page_shift, tile;
    int32_t q_ctas;                      // CTAs from 0 on that turn queries; the others store rows
    uint32_t n_slots;
};

// the 16 numbers from `first` on of a head's row, rotated where they are rotated
template <typename T, bool WIDE>
__device__ __forceinline__ void load_group(const T *row, int first, float (&x)[C4_GROUP])
{
    if constexpr (WIDE) {
        constexpr int E = 16 / (int)sizeof(T);
#pragma unroll
        for (int i = 0; i < C4_GROUP / E; ++i) {
            Chunk<T, E> c;
            c.load(row + first + i * E);
#pragma unroll
            for (int e = 0; e < E; ++e) x[i * E + e] = c.v[e];
        }
    } else {
#pragma unroll
        for (int i = 0; i < C4_GROUP; ++i) x[i] = load_as<float>(row, first + i);
    }
}

// HALVES: WIDE means that halves are whole chunks of 16 bytes, so that the partners of a chunk are one as well; a partner is loaded by the other
// half's thread, too: from L1.
template <typename T, bool WIDE, bool HALVES>
__device__ __forceinline__ void rotate_group(const T *row, int first, int rotary, const float2 *cs, float (&x)[C4_GROUP])
{
    if (first >= rotary) return;
    const int half = rotary / 2;
    if constexpr (!HALVES) {
#pragma unroll
        for (int i = 0; i < C4_GROUP; i += 2)
            if (first + i < rotary) rope_turn(x[i], x[i + 1], cs[(first + i) / 2]);
    } else {
        constexpr int E = WIDE ? 16 / (int)sizeof(T) : 1;
#pragma unroll
        for (int i = 0; i < C4_GROUP; i += E) {
            const int j = first + i;
            if (j >= rotary) continue;
            const bool lower = j < half;
            Chunk<T, E> other;
            other.load(row + (lower ? j + half : j - half));
            const float2 *c = cs + (lower ? j : j - half);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float a = lower ? x[i + e] : other.v[e], b = lower ? other.v[e] : x[i + e];
                rope_turn(a, b, c[e]);
                x[i + e] = lower ? a : b;
            }
        }
    }
}

template <typename T, int E, bool HALVES, bool WHOLE> __device__ __forceinline__ void turn_queries(const AppendArgs &a, const RopeTurns &turns, float *cs)
{
    const int64_t t0 = (int64_t)blockIdx.x * a.query.tile;
    const int count = min(a.query.tile, a.n_tokens - (int)t0);
    auto token = [&](int64_t t, int64_t &from, int64_t &to, int64_t &pos) {
        from = t * a.qs[0];
        to = t * a.qos[0];
        pos = a.rotary ? a.positions[t] : 0;
        return (uint32_t)a.slots[t] < a.n_slots;
    };
    if constexpr (WHOLE) rope_rows<T, E, HALVES>((const T *)a.q, (T *)a.q_out, a.query, turns, t0, count, cs, token);
    else rope_rows_any<T, E, HALVES>((const T *)a.q, (T *)a.q_out, a.query, turns, t0, count, cs, token);
}

// Queries are turned by the first CTAs as elm_rope does it; the others store rows, a thread two groups of 16 numbers: of a key that
// is rotated in halves both halves of its pairs.  The groups of a row are neighbouring lanes, so that its codes leave in one piece.
// (four CTAs per SM with bf16 numbers: 80 -> 78 us for prompts stored and read back)
template <typename T, int D, bool HALVES>
__global__ void __launch_bounds__(APP_THREADS, sizeof(T) == 2 ? 4 : 2) append4_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ RopeTurns turns)
{
    using R = Row4<D>;
    constexpr int G = R::GROUPS, E = 16 / (int)sizeof(T), HALF = G / 2;
    extern __shared__ __align__(16) float cs[];
    cudaGridDependencySynchronize();
    if ((int)blockIdx.x < a.q_ctas) {
        turn_queries<T, E, HALVES, true>(a, turns, cs);
        return;
    }
    // items: (token, head, key or value, pair of groups); a thread requests its first one's numbers before the cosines are formed
    const int pairs = a.rotary / 2, row_cs = rope_cs_floats<16>(pairs);
    const int t0 = ((int)blockIdx.x - a.q_ctas) * a.tile;
    const int count = min(a.tile, a.n_tokens - t0), total = count * a.kv_heads * G;
    int t, h, g0, g1, p;
    bool key, halves, there;
    uint32_t slot;
    Raw<T, E> raw[2][C4_GROUP / E];
    const int turned_key = a.rotary / C4_GROUP;                  // groups of a key that are rotated
    auto request = [&](int i) {
        const bool live = i < total;
        const int j = i % G, th = live ? i / G : 0;
        t = th / a.kv_heads;
        h = th - t * a.kv_heads;
        slot = (uint32_t)a.slots[t0 + t];
        there = live && slot < a.n_slots;
        key = j < HALF;
        p = key ? j : j - HALF;
        // the two groups: halves of pairs where they are rotated in halves, else side by side
        halves = HALVES && key && 2 * p < turned_key;
        g0 = halves ? p : 2 * p;
        g1 = halves ? p + turned_key / 2 : 2 * p + 1;
        if (there) {
            const T *src = key ? (const T *)a.k + (int64_t)(t0 + t) * a.ks[0] + h * a.ks[1] : (const T *)a.v + (int64_t)(t0 + t) * a.vs[0] + h * a.vs[1];
#pragma unroll
            for (int e = 0; e < C4_GROUP / E; ++e) {
                raw[0][e].load(src + g0 * C4_GROUP + e * E);
                raw[1][e].load(src + g1 * C4_GROUP + e * E);
            }
        }
    };
    request(threadIdx.x);
    __shared__ int64_t pos_of[APP_THREADS];
    if (pairs > 0)
        rope_table(turns, pairs, count, a.scale, a.scale, pos_of, [&](int ti, int64_t &at) { at = a.positions[t0 + ti]; return true; },
                   [&](int ti, int pi) { return reinterpret_cast<float2 *>(cs + ti * row_cs + 2 * pi + 4 * (pi / 16)); });
    for (int i0 = threadIdx.x & ~31; i0 < total; i0 += APP_THREADS) {        // (whole warps stay together: lanes exchange scales)
        if (i0 >= APP_THREADS) request(i0 + (threadIdx.x & 31));
        uint32_t byte0 = 0, byte1 = 0;
        unsigned char *row = nullptr;
        if (there) {
            float x[C4_GROUP], y[C4_GROUP];
#pragma unroll
            for (int e = 0; e < C4_GROUP; e += 2) {
                sm100::unpack2(raw[0][e / E].pair(e % E / 2), x[e], x[e + 1]);
                sm100::unpack2(raw[1][e / E].pair(e % E / 2), y[e], y[e + 1]);
            }
            if (halves) {
                const float *c = cs + t * row_cs + p * 36;
#pragma unroll
                for (int e = 0; e < C4_GROUP; e += 2) {
                    const float4 v = *reinterpret_cast<const float4 *>(c + 2 * e);
                    rope_turn(x[e], y[e], make_float2(v.x, v.y));
                    rope_turn(x[e + 1], y[e + 1], make_float2(v.z, v.w));
                }
            } else if (!HALVES && key && g0 < turned_key) {      // (rotary is a multiple of 32: both groups or none)
                const float *c = cs + t * row_cs + p * 36;
#pragma unroll
                for (int e = 0; e < C4_GROUP; e += 4) {
                    const float4 v = *reinterpret_cast<const float4 *>(c + e), w = *reinterpret_cast<const float4 *>(c + 16 + e);
                    rope_turn(x[e], x[e + 1], make_float2(v.x, v.y));
                    rope_turn(x[e + 2], x[e + 3], make_float2(v.z, v.w));
                    rope_turn(y[e], y[e + 1], make_float2(w.x, w.y));
                    rope_turn(y[e + 2], y[e + 3], make_float2(w.z, w.w));
                }
            }
            uint2 c0, c1;
            byte0 = quantise4(x, c0);
            byte1 = quantise4(y, c1);
            const uint32_t page = slot >> a.page_shift, in_page = slot & ((1u << a.page_shift) - 1u);
            row = a.rows + ((((uint64_t)page * (uint32_t)a.kv_heads + h) << a.page_shift) + in_page) * R::BYTES;
            uint2 *codes = reinterpret_cast<uint2 *>(row + (key ? 0 : R::CODES));
            codes[g0] = c0;
            codes[g1] = c1;
        }
        // scales of the row's key or value, this thread's two and its neighbours', as words: of groups 0 .. 3 and 4 .. 7
        uint32_t w0 = 0, w1 = 0;
        if (g0 < 4) w0 |= byte0 << (8 * g0);
        else w1 |= byte0 << (8 * (g0 - 4));
        if (g1 < 4) w0 |= byte1 << (8 * g1);
        else w1 |= byte1 << (8 * (g1 - 4));
#pragma unroll
        for (int o = 1; o < HALF; o <<= 1) {
            w0 |= __shfl_xor_sync(0xffffffffu, w0, o);
            if (G == 8) w1 |= __shfl_xor_sync(0xffffffffu, w1, o);
        }
        if (row && p == 0) {
            unsigned char *scales = row + R::SCALES + (key ? 0 : G);
            if (G == 8) {
                *reinterpret_cast<uint2 *>(scales) = make_uint2(w0, w1);
            } else {
                *reinterpret_cast<uint32_t *>(scales) = w0;
                *reinterpret_cast<uint32_t *>(row + R::SCALES + 2 * G + (key ? 0 : 4)) = 0u;       // (the unused bytes)
            }
        }
    }
}

// Rows whose numbers are not on 16-byte boundaries, or of which a part is rotated that is not whole groups on both sides: a thread takes one group of
// 16 numbers of a key or a value.  WIDE: rows on 16-byte boundaries; WHOLE: halves of the rotated part, too (or neither).
template <typename T, int D, bool WIDE, bool HALVES, bool WHOLE>
__global__ void __launch_bounds__(APP_THREADS) append4_any_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ RopeTurns turns)
{
    using R = Row4<D>;
    constexpr int G = R::GROUPS;
    extern __shared__ __align__(16) float cs_floats[];
    cudaGridDependencySynchronize();
    if ((int)blockIdx.x < a.q_ctas) {
        turn_queries<T, WIDE ? 16 / (int)sizeof(T) : 1, HALVES, WHOLE>(a, turns, cs_floats);
        return;
    }
    float2 *cs = reinterpret_cast<float2 *>(cs_floats);        // [tile][rotary / 2]
    const int pairs = a.rotary / 2;
    const int t0 = ((int)blockIdx.x - a.q_ctas) * a.tile;
    const int count = min(a.tile, a.n_tokens - t0);
    __shared__ int64_t pos_of[APP_THREADS];
    if (pairs > 0)
        rope_table(turns, pairs, count, a.scale, a.scale, pos_of, [&](int ti, int64_t &at) { at = a.positions[t0 + ti]; return true; },
                   [&](int ti, int pi) { return cs + ti * pairs + pi; });
    const int total = count * a.kv_heads * 2 * G;
    for (int i0 = threadIdx.x & ~31; i0 < total; i0 += APP_THREADS) {        // (whole warps stay together: lanes exchange scales)
        const int i = i0 + (threadIdx.x & 31);
        const bool live = i < total;
        const int j = i % (2 * G), th = live ? i / (2 * G) : 0;               // the row's group: keys, then values
        const int t = th / a.kv_heads, h = th - t * a.kv_heads;
        const uint32_t slot = (uint32_t)a.slots[t0 + t];
        uint32_t byte = 0;
        unsigned char *row = nullptr;
        if (live && slot < a.n_slots) {
            const int64_t tok = t0 + t;
            const bool key = j < G;
            const T *src = key ? (const T *)a.k + tok * a.ks[0] + h * a.ks[1] : (const T *)a.v + tok * a.vs[0] + h * a.vs[1];
            const int first = (key ? j : j - G) * C4_GROUP;
            float x[C4_GROUP];
            load_group<T, WIDE>(src, first, x);
            if (key) rotate_group<T, WIDE && WHOLE, HALVES>(src, first, a.rotary, cs + t * pairs, x);
            uint2 codes;
            byte = quantise4(x, codes);
            const uint32_t page = slot >> a.page_shift, in_page = slot & ((1u << a.page_shift) - 1u);
            row = a.rows + ((((uint64_t)page * (uint32_t)a.kv_heads + h) << a.page_shift) + in_page) * R::BYTES;
            *reinterpret_cast<uint2 *>(row + j * 8) = codes;
        }
        // scales: a row's lanes are neighbours and start at a multiple of 4 lanes, so four of them fill a word
        uint32_t word = byte << (8 * (j & 3));
        word |= __shfl_xor_sync(0xffffffffu, word, 1);
        word |= __shfl_xor_sync(0xffffffffu, word, 2);
        if (row && (j & 3) == 0) {
            *reinterpret_cast<uint32_t *>(row + R::SCALES + j) = word;
            if (2 * G + R::SCALES < R::BYTES && j == 0) *reinterpret_cast<uint2 *>(row + R::SCALES + 2 * G) = make_uint2(0u, 0u);
        }
    }
}

struct ReadArgs {
    Pool4 pool;
    const int32_t *length, *idx;
    void *k, *v;
    int32_t n;
    int64_t rows;                        // batch * kv_heads * n
    int32_t each;                        // rows of a warp
};

// A warp takes up to 32 rows, whose places its lanes look up side by side, and makes one (d = 64: two) at a time: a lane 8 numbers, from 4
// bytes of codes, so that its stores are whole lines.
constexpr int READ_AHEAD = 8;            // rows (pairs of rows) requested together
template <typename T, int D> __global__ void __launch_bounds__(256) read4_kernel(const __grid_constant__ ReadArgs a)
{
    using R = Row4<D>;
    constexpr int AT_ONCE = 128 / D, LANES = 32 / AT_ONCE;       // rows of a step, lanes of a row
    cudaGridDependencySynchronize();
    const int lane = threadIdx.x & 31;
    const int64_t first = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * a.each;
    if (first >= a.rows) return;
    uint32_t place = NO_ROW;
    if (lane < a.each && first + lane < a.rows) {
        const int64_t out_row = first + lane, problem = out_row / a.n, e = out_row - problem * a.n;
        const int b = (int)(problem / a.pool.kv_heads), h = (int)(problem - (int64_t)b * a.pool.kv_heads);
        const int64_t r = a.idx ? a.idx[out_row] : e;
        if (r >= 0 && (!a.length || r < a.length[b])) place = pool_row(a.pool, b, h, r);
    }
    const int j = lane % LANES;
    const bool key = j < LANES / 2;
    T *out = (T *)(key ? a.k : a.v) + (j % (LANES / 2)) * 8;
    const int64_t left = min((int64_t)a.each, a.rows - first);
    for (int s0 = 0; s0 * AT_ONCE < left; s0 += READ_AHEAD) {
        uint32_t codes[READ_AHEAD], scale[READ_AHEAD];
#pragma unroll
        for (int s = 0; s < READ_AHEAD; ++s) {
            const uint32_t row = __shfl_sync(0xffffffffu, place, (s0 + s) * AT_ONCE + lane / LANES);
            codes[s] = scale[s] = 0;
            if (row != NO_ROW) {
                const unsigned char *p = a.pool.rows + (uint64_t)row * R::BYTES;
                codes[s] = *reinterpret_cast<const uint32_t *>(p + 4 * j);
                scale[s] = p[R::SCALES + j / 2];
            }
        }
#pragma unroll
        for (int s = 0; s < READ_AHEAD; ++s) {
            const int at = (s0 + s) * AT_ONCE + lane / LANES;
            uint32_t half2s[4];
            codes8_to_half2(codes[s], half2s);
            const uint32_t sc = scale4_half2(scale[s]);
#pragma unroll
            for (int k = 0; k < 4; ++k) half2s[k] = hmul2_bits(half2s[k], sc);
            if (at >= left) continue;
            constexpr int E = 16 / (int)sizeof(T);
#pragma unroll
            for (int k = 0; k < 8; k += E) {
                Chunk<T, E> c;
#pragma unroll
                for (int x = 0; x < E; x += 2) {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&half2s[(k + x) / 2]));
                    c.v[x] = f.x;
                    c.v[x + 1] = f.y;
                }
                c.store(out + (first + at) * D + k);
            }
        }
    }
}

template <typename T, int D> int launch_append(AppendArgs &a, const RopeTurns &turns, bool halves, bool aligned, cudaStream_t st)
{
    constexpr int E = 16 / (int)sizeof(T);
    const int sms = device_sm_count(), pairs = a.rotary / 2;
    const bool whole = pairs % E == 0, groups = aligned && a.rotary % 32 == 0;
    int64_t q_ctas = 0;
    size_t smem = 0;
    a.query = RopeShape{a.q_heads, a.rotary, 0, 0, 0, 1, a.qs[1], a.qos[1], a.scale, a.scale};
    if (a.q_heads > 0) {
        const bool any = aligned && !whole;
        if (any) a.query.per_head = D / E;
        else rope_items(a.query, aligned ? E : 1, a.q == a.q_out ? 0 : D - a.rotary);        // (in place, numbers that are not rotated stay)
        if (a.query.per_head > 0) {
            rope_share(a.query, a.n_tokens, sms, any ? ROPE_ANY_AHEAD : ROPE_AHEAD);
            q_ctas = ((int64_t)a.n_tokens + a.query.tile - 1) / a.query.tile;
            smem = (size_t)a.query.tile * (any ? 2 * rope_any_places(pairs) : aligned ? rope_cs_floats<E>(pairs) : rope_cs_floats<1>(pairs)) * sizeof(float);
        }
    }
    // an item a thread; fewer tokens per CTA where they would not fill the GPU
    a.tile = APP_THREADS / (a.kv_heads * (D / C4_GROUP) * (groups ? 1 : 2));
    if (a.tile > a.n_tokens / (2 * sms)) a.tile = a.n_tokens / (2 * sms);
    if (a.tile < 1) a.tile = 1;
    const size_t rows_smem = (size_t)a.tile * (groups ? rope_cs_floats<16>(pairs) : 2 * pairs) * sizeof(float);
    if (rows_smem > smem) smem = rows_smem;
    const int64_t ctas = q_ctas + ((int64_t)a.n_tokens + a.tile - 1) / a.tile;
    if (ctas > 0x7fffffff) return ELM_ERR_SHAPE;
    a.q_ctas = (int)q_ctas;
    auto kern = groups ? (halves ? append4_kernel<T, D, true> : append4_kernel<T, D, false>)
                : !aligned ? (halves ? append4_any_kernel<T, D, false, true, true> : append4_any_kernel<T, D, false, false, true>)
                : whole ? (halves ? append4_any_kernel<T, D, true, true, true> : append4_any_kernel<T, D, true, false, true>)
                        : (halves ? append4_any_kernel<T, D, true, true, false> : append4_any_kernel<T, D, true, false, false>);
    ELM_CUDA_TRY(launch_after(kern, dim3((unsigned)ctas), dim3(APP_THREADS), smem, st, a, turns));
    count_launches(1);
    return cuda_status(cudaGetLastError());
}

}  // namespace
}  // namespace elm

using namespace elm;

extern "C" int elm_cache4_row_bytes(int32_t d, size_t *bytes)
{
    if (!bytes) return ELM_ERR_NULL;
    if (d != 64 && d != 128) return ELM_ERR_SHAPE;
    *bytes = (size_t)row4_bytes(d);
    return ELM_OK;
}

extern "C" int elm_cache4_append(const void *Q, const void *K, const void *V, const int32_t *positions, const int32_t *slots,
                                 const elm_append_params *p, void *Q_out, void *rows, void *stream)
{
    if (!p || !K || !V || !slots || !rows) return ELM_ERR_NULL;
    if (p->dtype != ELM_F32 && p->dtype != ELM_BF16) return ELM_ERR_DTYPE;
    if (p->n_tokens < 1 || p->q_heads < 0 || p->kv_heads < 1 || (p->d != 64 && p->d != 128)) return ELM_ERR_SHAPE;
    if (p->q_heads > 65535 || p->kv_heads > 65535) return ELM_ERR_SHAPE;
    const int shift = page_shift_of(p->page_rows);
    if (shift < 0 || !pool_fits(p->n_pages, p->page_rows, p->kv_heads)) return ELM_ERR_SHAPE;
    if (p->rotary_dim < 0 || p->rotary_dim > p->d || (p->rotary_dim & 1)) return ELM_ERR_SHAPE;
    if (p->layout != ELM_ROPE_HALVES && p->layout != ELM_ROPE_PAIRS) return ELM_ERR_SHAPE;
    if (p->q_heads > 0 && (!Q || !Q_out)) return ELM_ERR_NULL;
    RopeTurns turns;
    if (p->rotary_dim > 0) {
        if (!positions || !p->inv_freq) return ELM_ERR_NULL;
        if (!isfinite(p->scale) || !rope_turns(p->inv_freq, p->rotary_dim / 2, turns)) return ELM_ERR_SHAPE;
    }
    const int item = (int)elt_bytes(p->dtype);
    AppendArgs a = {};
    a.q = Q;
    a.k = K;
    a.v = V;
    a.q_out = Q_out;
    a.positions = positions;
    a.slots = slots;
    a.rows = (unsigned char *)rows;
    auto strides = [&](const int64_t (&in)[2], int heads, int64_t (&out)[2]) {
        const bool dense = in[0] == 0 && in[1] == 0;
        out[0] = dense ? (int64_t)heads * p->d : in[0];
        out[1] = dense ? p->d : in[1];
        return out[0] | out[1];
    };
    int64_t all = strides(p->k_stride, p->kv_heads, a.ks) | strides(p->v_stride, p->kv_heads, a.vs);
    uintptr_t at = (uintptr_t)K | (uintptr_t)V;
    if (p->q_heads > 0) {
        all |= strides(p->q_stride, p->q_heads, a.qs) | strides(p->q_out_stride, p->q_heads, a.qos);
        at |= (uintptr_t)Q | (uintptr_t)Q_out;
        // rows of Q_out that would be written twice; in place only where every number stays in its place
        if ((p->n_tokens > 1 && a.qos[0] == 0) || (p->q_heads > 1 && a.qos[1] == 0)) return ELM_ERR_SHAPE;
        if (Q == Q_out && (a.qs[0] != a.qos[0] || a.qs[1] != a.qos[1])) return ELM_ERR_SHAPE;
    }
    if ((at & (item - 1)) || (((uintptr_t)positions | (uintptr_t)slots) & 3) || ((uintptr_t)rows & 15)) return ELM_ERR_ALIGN;
    a.scale = p->scale;
    a.n_tokens = p->n_tokens;
    a.q_heads = p->q_heads;
    a.kv_heads = p->kv_heads;
    a.rotary = p->rotary_dim;
    a.page_shift = shift;
    a.n_slots = (uint32_t)((int64_t)p->n_pages << shift);
    const bool wide = !(at & 15) && all % (16 / item) == 0, halves = p->layout == ELM_ROPE_HALVES;
    cudaStream_t st = (cudaStream_t)stream;
    if (p->dtype == ELM_BF16)
        return p->d == 64 ? launch_append<__nv_bfloat16, 64>(a, turns, halves, wide, st) : launch_append<__nv_bfloat16, 128>(a, turns, halves, wide, st);
    return p->d == 64 ? launch_append<float, 64>(a, turns, halves, wide, st) : launch_append<float, 128>(a, turns, halves, wide, st);
}

extern "C" int elm_cache4_read(const void *rows, const int32_t *table, const int32_t *length, const int32_t *idx, const elm_cache4_params *p,
                               void *K_out, void *V_out, void *stream)
{
    if (!p || !rows || !table || !K_out || !V_out) return ELM_ERR_NULL;
    if (p->dtype != ELM_F32 && p->dtype != ELM_BF16) return ELM_ERR_DTYPE;
    if (p->batch < 1 || p->kv_heads < 1 || p->kv_heads > 65535 || p->n_kv < 1 || p->max_pages < 1 || (p->d != 64 && p->d != 128)) return ELM_ERR_SHAPE;
    const int shift = page_shift_of(p->page_rows);
    if (shift < 0 || !pool_fits(p->n_pages, p->page_rows, p->kv_heads)) return ELM_ERR_SHAPE;
    if (((uintptr_t)rows | (uintptr_t)K_out | (uintptr_t)V_out) & 15) return ELM_ERR_ALIGN;
    if (((uintptr_t)table | (uintptr_t)length | (uintptr_t)idx) & 3) return ELM_ERR_ALIGN;
    ReadArgs a;
    a.pool = Pool4{(const unsigned char *)rows, table, p->n_pages, p->max_pages, shift, p->kv_heads};
    a.length = length;
    a.idx = idx;
    a.k = K_out;
    a.v = V_out;
    a.n = p->n_kv;
    a.rows = (int64_t)p->batch * p->kv_heads * p->n_kv;
    // rows of a warp: 32 in long calls (they are looked up side by side), fewer where the warps would not fill the GPU
    a.each = 32;
    while (a.each > 8 && a.rows / a.each < (int64_t)32 * device_sm_count()) a.each >>= 1;
    const int64_t ctas = (a.rows + 8 * a.each - 1) / (8 * a.each);
    if (ctas > 0x7fffffff) return ELM_ERR_SHAPE;
    auto kern = p->dtype == ELM_BF16 ? (p->d == 64 ? read4_kernel<__nv_bfloat16, 64> : read4_kernel<__nv_bfloat16, 128>)
                                     : (p->d == 64 ? read4_kernel<float, 64> : read4_kernel<float, 128>);
    ELM_CUDA_TRY(launch_after(kern, dim3((unsigned)ctas), dim3(256), 0, (cudaStream_t)stream, a));
    count_launches(1);
    return cuda_status(cudaGetLastError());
}
