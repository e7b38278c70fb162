// Attention over rows held in 4 bits (elm_cache4_attend): a request's rows up to its length, or a weighted list of them.
//
//   O[j,:] = sum_c w_c exp(<q_j,k_c>/sqrt(d)) v_c / sum_c w_c exp(<q_j,k_c>/sqrt(d))      Eq. (def:att_approx)
//
// A problem is N = 8 or 16 query vectors of one KV head (its query heads, and neighbouring tokens) over that head's rows.  A warp takes
// 32 rows at a time.  Both contractions run on mma.sync m16n8k16 with fp16 operands and fp32 accumulators and with the QUERY VECTORS as
// the narrow side, so that the few there are fill it:
//   S^T = K Q^T   (16 rows x 8 vectors):  a lane's part of the K operand is one stretch of 32 numbers (d = 64: 16) of rows g and g + 8, read as
//                 16 (8) bytes of codes; which numbers make up a step of the contraction is free as long as Q is laid out alike.
//   O^T = V^T P^T (16 numbers x 8 vectors): the V operand wants two neighbouring rows' numbers in one register: nibbles of the two
//                 rows' words are put side by side (one logic operation and a shift per eight numbers), so that converting a byte gives the pair.
//                 P^T comes from the accumulator layout of S^T by one 8x8 transposition (movmatrix) per 16 rows and half.
// Codes become fp16 numbers by one conversion per two and are multiplied by their scales, exactly (elm_cache4.cuh).  A query vector is scaled to
// a largest magnitude of 2^11 .. 2^12 before it is rounded to fp16 (bf16 numbers have fewer bits: exact but for those 2^-25 below the
// largest); probabilities are exp2 of the distance to a running reference + 8, so that fp16 holds them down to 2^-32 of the largest, and the
// reference moves only when the maximum has passed it by 2^6.  fp32 queries and outputs: queries and probabilities as two fp16 parts (22
// bits), and each tile's sums go to fp32 accumulators by ordinary additions, since the matrix instruction cuts off low bits.
//
// The rows of all problems form one line of tiles, and every CTA takes an equal stretch of it, whatever the requests' lengths are - they are on
// the device, and the stretch is found there.  A problem that lies in one stretch is finished there; the parts of one that several CTAs share go to the
// workspace and are joined by a second launch.  Short problems go to a CTA or a cluster each, in one launch.
//
// What bounds it: its floor is reading each row once (144 bytes at d = 128), which it does; the time is the issue of 575 instructions per tile, 225 of them on
// the integer and conversion pipe at two cycles each.  48 requests x 16384 rows x 8 heads, d = 128: 162 us = 5.6 TB/s, 85 % of the measured copy rate (16
// vectors 225 us, fp32 224 us, d = 64 109 us); 48 requests of 1 .. 32768 rows, lengths spread over the logarithm, 48 us for a floor of 27.
#include <cooperative_groups.h>
#include <math.h>

#include <atomic>

#include "elm_attend.cuh"
#include "elm_cache4.cuh"
#include "elm_sm100.cuh"

namespace elm {
namespace {

constexpr int A4_WARPS = 4;
constexpr int A4_THREADS = 32 * A4_WARPS;
constexpr int A4_TILE = 32;              // rows of a warp's tile
constexpr int A4_STAGES = 2;             // tiles in flight per warp (three: 65 against 60 us, for one CTA less per SM)
constexpr int A4_START = 12;             // what a problem's beginning and end cost, in tiles (8: 54, 12: 49, 16: 50 us for 48 ragged requests)
constexpr int A4_MAX_BATCH = 1024, A4_SOME = 511, A4_FEW = 127;        // requests of a call; of calls whose line is short
constexpr int A4_CTA_PLACES = 8;         // a CTA's stretch holds at least these
constexpr float A4_LIFT = 8.f;           // probabilities are 2^8 times their share of the reference's
constexpr float A4_SLACK = 6.f;          // how far the maximum may pass the reference: fp16 ends at 2^16

struct Attend4Args {
    Pool4 pool;
    const void *q;
    void *o;
    const int32_t *length, *cu, *idx;
    const float *w;
    float *part;                         // sums [2 * ctas][N][D], then (reference, denominator) [2 * ctas][N]
    int64_t qs[3], os[3];
    int32_t batch, q_heads, rep, n_kv, n_q, n_tokens, causal;
    int32_t cluster;                     // CTAs of the cluster that does a problem; 0: the line of tiles is cut into stretches
    int32_t max_groups;                  // groups of query vectors of a request at most
    int32_t q_wide;                      // every row of Q starts on an 8-byte boundary
};

// Where the problems of every request begin in the line of tiles.  A request of n query vectors (rep * its tokens) over t tiles has
// kv_heads * ceil(n / N) problems of A4_START + t places each, one after the other, KV head slowest.  The first A4_START places of a problem hold no
// tile: they stand for what it costs whatever its length (48 requests of 1 .. 32768 rows, lengths spread over the logarithm: the CTAs that
// met many short ones took 2.5 times as long as the others).
// what is known of a request, and what follows from it
struct Request {
    int32_t rows, tokens, first_token, groups, tiles, places;
    int32_t seen0;                       // rows that the first token sees, of all the request's tokens (some may be cut off): <= 0 is none
};
__device__ __forceinline__ Request request_from(const Attend4Args &a, int4 known, int n_vec)
{
    Request r;
    r.rows = known.x;
    r.tokens = known.y;
    r.first_token = known.z;
    r.seen0 = r.rows - known.w + 1;
    r.groups = (r.tokens * a.rep + n_vec - 1) / n_vec;
    r.tiles = max(1, (r.rows + A4_TILE - 1) / A4_TILE);
    r.places = A4_START + r.tiles;
    return r;
}
__device__ __forceinline__ int4 look_at_request(const Attend4Args &a, int b)
{
    int4 r = make_int4(a.n_kv, a.n_q, 0, a.n_q);
    if (!a.idx) r.x = a.length[b];
    if (a.cu) {
        r.z = a.cu[b];
        r.w = r.y = a.cu[b + 1] - r.z;
        // only tokens that Q has; which rows those see goes by all of them
        if (r.z < 0 || r.y < 0) r.y = 0;
        else if ((int64_t)r.z + r.y > a.n_tokens) r.y = max(0, a.n_tokens - r.z);
        r.y = min(r.y, a.n_q);
    }
    r.x = min(max(r.x, 0), a.n_kv);
    return r;
}

__device__ __forceinline__ void cp16(uint32_t dst, const void *src, bool live)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the same without sums from before
__device__ __forceinline__ void mma_f16_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// what is left of two numbers after their rounding to fp16, as fp16
__device__ __forceinline__ uint32_t half2_rest(float lo, float hi, uint32_t rounded)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&rounded));
    return half2_bits(lo - f.x, hi - f.y);
}
// bytes whose low halves are a's and whose high halves are b's, in one operation
__device__ __forceinline__ uint32_t low_of_high_of(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, 0x0f0f0f0f, 0xe4;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// shared memory of the line of tiles: a prefix and four words for each request
constexpr int line_bytes(int batch) { return (batch + 2) * 8 + batch * 16; }

template <int D, int NT, int PARTS> struct A4 {
    using R = Row4<D>;
    static constexpr int N = 8 * NT;
    static constexpr int KS = D / 16;                            // steps of the contraction over d
    static constexpr int TILE_BYTES = A4_TILE * R::BYTES;
    static constexpr int OD = D + 4;                             // floats between vectors of a warp's result (bank offset)
    // per warp: the ring of tiles; over it, at the end of a stretch, the warp's result.  Then the rows' biases per stage, the line of tiles, Q.
    static constexpr int WARP_BYTES = A4_STAGES * TILE_BYTES > N * OD * 4 ? A4_STAGES * TILE_BYTES : N * OD * 4;
    static constexpr int OFF_BIAS = A4_WARPS * WARP_BYTES;
    static constexpr int OFF_ML = OFF_BIAS + A4_WARPS * A4_STAGES * A4_TILE * 4;
    static constexpr int OFF_QS = OFF_ML + A4_WARPS * N * 2 * 4;  // [N] scale of the logits of a vector
    static constexpr int OFF_Q = (OFF_QS + N * 4 + 15) / 16 * 16; // [PARTS][NT][KS / 2][32 lanes] 16 bytes
    static constexpr int OFF_LINE = OFF_Q + PARTS * NT * (KS / 2) * 512;                   // (a multiple of 16)
    static int total(int batch) { return OFF_LINE + line_bytes(batch); }
};

// prefix[b] = places before request b, known[b] = what is known of it; every thread returns the total.  The requests are looked at side by side,
// then every thread adds up a run of them and the runs are summed in one scan.
__device__ __forceinline__ int4 *line_known(int64_t *prefix, int batch) { return reinterpret_cast<int4 *>(prefix + ((batch + 2) & ~1)); }
__device__ __forceinline__ int64_t lay_line(const Attend4Args &a, int n_vec, int64_t *prefix, int64_t *part)
{
    int4 *known = line_known(prefix, a.batch);
    for (int b = threadIdx.x; b < a.batch; b += blockDim.x) known[b] = look_at_request(a, b);
    __syncthreads();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, run = (a.batch + blockDim.x - 1) / blockDim.x;
    const int b0 = min(a.batch, (int)threadIdx.x * run), b1 = min(a.batch, b0 + run);
    int64_t mine = 0;
    for (int b = b0; b < b1; ++b) {
        const Request r = request_from(a, known[b], n_vec);
        mine += (int64_t)(a.pool.kv_heads * r.groups) * r.places;
    }
    int64_t x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) part[warp] = x;
    __syncthreads();
    int64_t total = 0, at = x - mine;
    for (int i = 0; i < (int)(blockDim.x >> 5); ++i) {
        if (i < warp) at += part[i];
        total += part[i];
    }
    for (int b = b0; b < b1; ++b) {
        const Request r = request_from(a, known[b], n_vec);
        prefix[b] = at;
        at += (int64_t)(a.pool.kv_heads * r.groups) * r.places;
    }
    if (threadIdx.x == 0) prefix[a.batch] = total;
    __syncthreads();
    return total;
}
// a / b and a * b / c of numbers that are mostly small: a division of 64 bits takes several times as long
__device__ __forceinline__ int64_t div_small(int64_t x, int64_t y)
{
    return ((uint64_t)x | (uint64_t)y) >> 32 ? x / y : (int64_t)((uint32_t)x / (uint32_t)y);
}
__host__ __device__ __forceinline__ int stretches(int64_t total, int ctas)
{
    const int64_t most = (total + A4_CTA_PLACES - 1) / A4_CTA_PLACES;
    return (int)(most < ctas ? most : ctas);
}
// request that place f belongs to: the last with prefix[b] <= f (requests without places are passed over)
__device__ __forceinline__ int request_of(const int64_t *prefix, int batch, int64_t f)
{
    int lo = 0, hi = batch - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (prefix[mid] <= f) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// LIST: entries idx with weights w, looked up row by row; else a request's rows, in pages of at least 16: half a tile lies in one page.
template <typename T, int D, int NT, int PARTS, bool LIST>
__global__ void __launch_bounds__(A4_THREADS, NT == 1 && PARTS == 1 ? 4 : 3) attend4_kernel(const __grid_constant__ Attend4Args a)
{
    using C = A4<D, NT, PARTS>;
    using R = Row4<D>;
    constexpr int N = C::N, KS = C::KS;
    constexpr int KB = D / 8, VB = D / 16;                       // bytes of codes a lane reads of a key row, of a value row
    extern __shared__ __align__(16) unsigned char smem[];
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    float *ml = reinterpret_cast<float *>(smem + C::OFF_ML);
    float *q_scale = reinterpret_cast<float *>(smem + C::OFF_QS);
    uint4 *q_frag = reinterpret_cast<uint4 *>(smem + C::OFF_Q);
    int64_t *prefix = reinterpret_cast<int64_t *>(smem + C::OFF_LINE);
    unsigned char *ring = smem + warp * C::WARP_BYTES;
    float *bias = reinterpret_cast<float *>(smem + C::OFF_BIAS) + warp * A4_STAGES * A4_TILE;
    const uint32_t ring_u32 = (uint32_t)__cvta_generic_to_shared(ring);

    cudaGridDependencySynchronize();
    // (the launch that joins the parts may come in as CTAs end: it waits for all of this one before it reads them)
    cudaTriggerProgrammaticLaunchCompletion();
    const float logit_scale = (float)(1.4426950408889634 / sqrt((double)D));
    int64_t begin = 0, end = 1;
    int b = blockIdx.x / max(1, a.cluster * a.pool.kv_heads * a.max_groups);
    if (!a.cluster) {
        const int64_t total = lay_line(a, N, prefix, reinterpret_cast<int64_t *>(smem));
        const int ctas = stretches(total, gridDim.x);
        if ((int)blockIdx.x >= ctas) return;
        begin = div_small(total * blockIdx.x, ctas);
        end = div_small(total * (blockIdx.x + 1), ctas);
        b = request_of(prefix, a.batch, begin);
    }
    for (int64_t f = begin; f < end;) {
        if (!a.cluster)
            while (prefix[b + 1] <= f) ++b;
        const Request rq = request_from(a, a.cluster ? look_at_request(a, b) : line_known(prefix, a.batch)[b], N);
        int h, group, tile0, tile1;
        const bool first_segment = f == begin;
        if (a.cluster) {
            // the tiles of a problem in equal shares; a CTA without any still takes part in the joining
            f = end;
            const int problem = blockIdx.x / a.cluster - b * a.pool.kv_heads * a.max_groups, rank = blockIdx.x % a.cluster;
            h = problem / a.max_groups;
            group = problem - h * a.max_groups;
            if (group >= rq.groups) return;                      // (the whole cluster)
            tile0 = (int)((int64_t)rq.tiles * rank / a.cluster);
            tile1 = (int)((int64_t)rq.tiles * (rank + 1) / a.cluster);
        } else {
            const int64_t in_request = f - prefix[b];
            const int problem = (int)div_small(in_request, rq.places), place0 = (int)(in_request - (int64_t)problem * rq.places);
            const int place1 = (int)min((int64_t)rq.places, place0 + (end - f));
            f += place1 - place0;
            tile0 = max(0, place0 - A4_START);
            tile1 = place1 - A4_START;
            if (tile1 <= tile0) continue;                        // (only what stands for a problem's beginning)
            h = problem / rq.groups;
            group = problem - h * rq.groups;
        }
        const bool whole = tile0 == 0 && tile1 == rq.tiles;
        const int vec0 = group * N;                              // vector v of the group is token (vec0 + v) / rep, head h rep + (vec0 + v) % rep
        const int vectors = min(N, rq.tokens * a.rep - vec0);
        // rows a vector sees: the last token of the request all of them, the one before it one less
        const bool tail = !LIST && a.causal;
        const int last_seen = tail ? rq.seen0 + (vec0 + vectors - 1) / a.rep : rq.rows;
        const int first_seen = tail ? rq.seen0 + vec0 / a.rep : rq.rows;
        const int tile_end = min(tile1, (last_seen + A4_TILE - 1) / A4_TILE);

        // ---- the queries are asked for first: vector q_vec by PER threads ----
        constexpr int PER = A4_THREADS / N, EACH = D / PER;      // threads to a vector, numbers to a thread
        const int q_vec = threadIdx.x / PER, q_sub = threadIdx.x % PER;
        uint32_t q_raw[EACH * sizeof(T) / 4];
#pragma unroll
        for (int i = 0; i < (int)(EACH * sizeof(T) / 4); ++i) q_raw[i] = 0u;
        if (q_vec < vectors) {
            const int vv = vec0 + q_vec, tok = vv / a.rep, head = h * a.rep + vv % a.rep;
            const T *src = (const T *)a.q + (a.cu ? (int64_t)(rq.first_token + tok) * a.qs[2] : b * a.qs[0] + tok * a.qs[2]) + head * a.qs[1] + q_sub * EACH;
            if (a.q_wide) {
#pragma unroll
                for (int i = 0; i < (int)(EACH * sizeof(T) / 8); ++i) {
                    const uint2 w = reinterpret_cast<const uint2 *>(src)[i];
                    q_raw[2 * i] = w.x;
                    q_raw[2 * i + 1] = w.y;
                }
            } else {
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    if constexpr (sizeof(T) == 2) q_raw[i / 2] |= (uint32_t)__bfloat16_as_ushort(src[i]) << (16 * (i & 1));
                    else q_raw[i] = __float_as_uint(src[i]);
                }
            }
        }

        // ---- the rows of this warp's tiles, looked up a tile before they are fetched ----
        uint32_t next_row[2] = {NO_ROW, NO_ROW};                 // LIST: [0] is lane's row of the tile; else the first rows of its halves
        float next_bias = -INFINITY;
        const int share = (tile_end - tile0 + A4_WARPS - 1) / A4_WARPS, mine0 = tile0 + warp * share, mine1 = min(mine0 + share, tile_end);
        const int page_mask = (1 << a.pool.page_shift) - 1;
        auto look_up = [&](int tile) {
            if (tile >= mine1) return;
            if constexpr (LIST) {
                next_row[0] = NO_ROW;
                next_bias = -INFINITY;
                const int e = tile * A4_TILE + lane;
                if (e < rq.rows) {
                    const int64_t at = ((int64_t)b * a.pool.kv_heads + h) * a.n_kv + e;
                    const float w = a.w[at];
                    if (w > 0.f) next_row[0] = pool_row(a.pool, b, h, a.idx[at]);
                    if (next_row[0] != NO_ROW) next_bias = log2f(w);
                }
            } else {
                const int e = tile * A4_TILE;                    // (below the rows that are seen)
                if (a.pool.page_shift == 4) {
                    next_row[0] = pool_row(a.pool, b, h, e);
                    next_row[1] = e + 16 < rq.rows ? pool_row(a.pool, b, h, e + 16) : NO_ROW;
                } else if (tile == mine0 || (e & page_mask) == 0) {
                    next_row[0] = pool_row(a.pool, b, h, e);
                } else if (next_row[0] != NO_ROW) {
                    next_row[0] += A4_TILE;                      // (the same page)
                }
            }
        };
        uint32_t gone = 0;                                       // two bits for each tile in flight: halves that are on no page
        auto fetch = [&](int stage, bool any, int order) {
            if (any) {
                const uint32_t dst = ring_u32 + stage * C::TILE_BYTES + lane * 16;
                if constexpr (LIST) {
                    bias[stage * A4_TILE + lane] = next_bias;
#pragma unroll
                    for (int i = 0; i < R::CHUNKS; ++i) {
                        const int c = i * 32 + lane, row = c / R::CHUNKS, chunk = c - row * R::CHUNKS;
                        const uint32_t from = __shfl_sync(0xffffffffu, next_row[0], row);
                        // (a row that is not there is filled with zeros: codes and scales of 0)
                        cp16(dst + i * 512, a.pool.rows + (from != NO_ROW ? (uint64_t)from * R::BYTES + chunk * 16 : 0), from != NO_ROW);
                    }
                } else {
                    // (nothing is read for what is not there)
                    const bool there0 = next_row[0] != NO_ROW;
                    const unsigned char *p0 = a.pool.rows + (there0 ? (uint64_t)next_row[0] * R::BYTES : 0) + lane * 16;
                    if (a.pool.page_shift > 4) {
#pragma unroll
                        for (int i = 0; i < R::CHUNKS; ++i) cp16(dst + i * 512, p0 + i * 512, there0);
                        if (!there0) gone |= 3u << (2 * order);
                    } else {
                        // the second half begins with chunk 16 CHUNKS, in the middle of the middle round
                        constexpr int MID = R::CHUNKS / 2;
                        const bool there1 = next_row[1] != NO_ROW, up = lane >= 16;
                        const unsigned char *p1 = a.pool.rows + (there1 ? (uint64_t)next_row[1] * R::BYTES : 0) + lane * 16;
#pragma unroll
                        for (int i = 0; i < MID; ++i) cp16(dst + i * 512, p0 + i * 512, there0);
                        cp16(dst + MID * 512, up ? p1 - 256 : p0 + MID * 512, up ? there1 : there0);
#pragma unroll
                        for (int i = MID + 1; i < R::CHUNKS; ++i) cp16(dst + i * 512, p1 + (i * 512 - MID * 512 - 256), there1);
                        gone |= ((there0 ? 0u : 1u) | (there1 ? 0u : 2u)) << (2 * order);
                    }
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        int ahead = mine0;
        look_up(ahead);
#pragma unroll
        for (int s = 0; s < A4_STAGES - 1; ++s) {
            fetch(s, ahead < mine1, s);
            look_up(++ahead);
        }

        // ---- queries: scaled by a power of two, laid out as the lanes want them ----
        {
            float x[EACH];
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                if constexpr (sizeof(T) == 2) x[i] = __uint_as_float(i & 1 ? q_raw[i / 2] & 0xffff0000u : q_raw[i / 2] << 16);
                else x[i] = __uint_as_float(q_raw[i]);
                top = fmaxf(top, fabsf(x[i]));
            }
#pragma unroll
            for (int o = PER / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            // 2^(11 - e) with e the exponent of the largest (at most 2^127: of tiny ones)
            const int e = top == 0.f ? 11 : min(127, (int)(__float_as_uint(top) >> 23) - 127);
            const float up = __uint_as_float((uint32_t)(127 + min(127, 11 - e)) << 23);
            const int v = q_vec;
            if (q_sub == 0) q_scale[v] = logit_scale / up;
            // lane (v % 8, lane_t) of tile v / 8 has numbers [D / 4 lane_t, D / 4 (lane_t + 1)), a step of the contraction four of them
#pragma unroll
            for (int i = 0; i < EACH; i += 2) {
                const int n = q_sub * EACH + i, lane_t = n / (D / 4), in = n % (D / 4);
                const int step = in / 4, pair = (in / 2) % 2;
                uint32_t hi = half2_bits(x[i] * up, x[i + 1] * up);
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    uint32_t *to = reinterpret_cast<uint32_t *>(q_frag + ((p * NT + v / 8) * (KS / 2) + step / 2) * 32 + (v % 8) * 4 + lane_t);
                    to[(step % 2) * 2 + pair] = hi;
                    if (p + 1 < PARTS) hi = half2_rest(x[i] * up, x[i + 1] * up, hi);
                }
            }
        }
        __syncthreads();

        // ---- the warp's tiles ----
        float o[NT][KS][4], l[NT][2], ref[NT][2], qs[NT][2];
        float limit[NT][2], lift[NT][2];                         // what moves the reference; what a logit is raised by
        int seen[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int v = n * 8 + 2 * t + x;
                l[n][x] = 0.f;
                ref[n][x] = limit[n][x] = -INFINITY;
                lift[n][x] = 0.f;
                qs[n][x] = q_scale[v];
                seen[n][x] = tail ? rq.seen0 + (vec0 + v) / a.rep : rq.rows;
            }
#pragma unroll
            for (int i = 0; i < KS; ++i)
#pragma unroll
                for (int x = 0; x < 4; ++x) o[n][i][x] = 0.f;
        }
        int stage = 0;
        const int cut_tile = first_seen / A4_TILE;               // from this one on some vector does not see all rows
        for (int tile = mine0; tile < mine1; ++tile) {
            asm volatile("cp.async.wait_group %0;" ::"n"(A4_STAGES - 2) : "memory");
            __syncwarp();
            const unsigned char *rows = ring + stage * C::TILE_BYTES;
            const float *rb = bias + stage * A4_TILE;
            const uint32_t gone_now = gone & 3u;
            gone >>= 2;
            {
                // the stage read in the last round is free
                const int to = stage + A4_STAGES - 1;
                fetch(to >= A4_STAGES ? to - A4_STAGES : to, ahead < mine1, A4_STAGES - 2);
                look_up(++ahead);
            }
            stage = stage + 1 == A4_STAGES ? 0 : stage + 1;

            const bool cut = tile >= cut_tile;
            // a value that is NaN must not reach a vector that does not see its row through 0 x NaN: such scales are taken out here and put
            // back as NaN sums of those that see it
            uint32_t nan_groups = 0, nan_rows = 0;
            if (!LIST && cut) {
                // rows behind the last one came with their page, whatever they hold: nothing
                if (tile * A4_TILE + lane >= rq.rows) *reinterpret_cast<uint4 *>(ring + (rows - ring) + lane * R::BYTES + R::SCALES) = make_uint4(0u, 0u, 0u, 0u);
                unsigned char *vscale = ring + (rows - ring) + lane * R::BYTES + R::SCALES + R::GROUPS;
#pragma unroll
                for (int i = 0; i < R::GROUPS; ++i)
                    if (vscale[i] >= 0xf8u) {
                        nan_groups |= 1u << i;
                        vscale[i] = 0;
                    }
                nan_rows = __ballot_sync(0xffffffffu, nan_groups != 0);
                __syncwarp();
            }

            // ---- logits: s[block of 16 rows][tile of vectors] = rows g, g + 8 x vectors 2t, 2t + 1 ----
            float s[2][NT][4];
            uint32_t codes[2][2][KB / 4], scale[2][2][D / 64];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const unsigned char *row = rows + (kb * 16 + x * 8 + g) * R::BYTES;
                    if constexpr (D == 128) {
                        const uint4 c = *reinterpret_cast<const uint4 *>(row + t * KB);
                        codes[kb][x][0] = c.x; codes[kb][x][1] = c.y; codes[kb][x][2] = c.z; codes[kb][x][3] = c.w;
                    } else {
                        const uint2 c = *reinterpret_cast<const uint2 *>(row + t * KB);
                        codes[kb][x][0] = c.x; codes[kb][x][1] = c.y;
                    }
#pragma unroll
                    for (int y = 0; y < D / 64; ++y) scale[kb][x][y] = scale4_half2(row[R::SCALES + D / 64 * t + y]);
                }
#pragma unroll
            for (int w = 0; w < KB / 4; ++w) {                   // a word: eight numbers, two steps
                uint4 q[PARTS][NT];
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int n = 0; n < NT; ++n) q[p][n] = q_frag[((p * NT + n) * (KS / 2) + w) * 32 + lane];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    uint32_t half[2][4];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        codes8_to_half2(codes[kb][x][w], half[x]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) half[x][i] = hmul2_bits(half[x][i], scale[kb][x][w / 2]);
                    }
                    const uint32_t a0[4] = {half[0][0], half[1][0], half[0][1], half[1][1]};
                    const uint32_t a1[4] = {half[0][2], half[1][2], half[0][3], half[1][3]};
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        if constexpr (PARTS == 1) {
                            if (w == 0) mma_f16_first(s[kb][n], a0, q[0][n].x, q[0][n].y);
                            else mma_f16(s[kb][n], a0, q[0][n].x, q[0][n].y);
                            mma_f16(s[kb][n], a1, q[0][n].z, q[0][n].w);
                        } else {
                            // a chain of four, the small parts first
                            float c[4];
                            mma_f16_first(c, a0, q[1][n].x, q[1][n].y);
                            mma_f16(c, a1, q[1][n].z, q[1][n].w);
                            mma_f16(c, a0, q[0][n].x, q[0][n].y);
                            mma_f16(c, a1, q[0][n].z, q[0][n].w);
#pragma unroll
                            for (int x = 0; x < 4; ++x) s[kb][n][x] = w == 0 ? c[x] : s[kb][n][x] + c[x];
                        }
                    }
                }
            }

            // ---- what is not seen is -inf whatever it holds; LIST: logits in base 2 with the weights, else as they are (times qs: base 2) ----
            float top[NT][2];
            if (!LIST && (cut || gone_now)) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int at = tile * A4_TILE + kb * 16 + x * 8 + g;
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int y = 0; y < 2; ++y)
                                if (at >= seen[n][y] || ((gone_now >> kb) & 1u)) s[kb][n][2 * x + y] = -INFINITY;
                    }
            }
            if constexpr (LIST) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const float lw = rb[kb * 16 + x * 8 + g];
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int y = 0; y < 2; ++y) s[kb][n][2 * x + y] = fmaf(s[kb][n][2 * x + y], qs[n][y], lw);
                    }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    top[n][y] = fmaxf(sm100::max3(s[0][n][y], s[0][n][2 + y], s[1][n][y]), s[1][n][2 + y]);
                    if (!LIST) top[n][y] *= qs[n][y];
                }
            // The reference moves when some row has passed it by A4_SLACK (the first rows seen do: it is -inf); only then the lanes that hold a
            // vector's rows ask one another for the largest.
            bool moved = false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int y = 0; y < 2; ++y) moved |= top[n][y] > limit[n][y];
            if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
#pragma unroll
                        for (int off = 4; off < 32; off <<= 1) top[n][y] = fmaxf(top[n][y], __shfl_xor_sync(0xffffffffu, top[n][y], off));
                        const float to = fmaxf(ref[n][y], top[n][y]);
                        const float f2 = ref[n][y] == -INFINITY ? 0.f : exp2_fast(ref[n][y] - to);
                        ref[n][y] = to;
                        limit[n][y] = to + A4_SLACK;
                        lift[n][y] = to == -INFINITY ? 0.f : A4_LIFT - to;
                        l[n][y] *= f2;
#pragma unroll
                        for (int i = 0; i < KS; ++i) {
                            o[n][i][y] *= f2;
                            o[n][i][2 + y] *= f2;
                        }
                    }
            }
            // ---- probabilities: the P operand of rows [16 kb, 16 kb + 16) ----
            uint32_t pb[PARTS][2][NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const float p0 = exp2_fast(LIST ? s[kb][n][2 * x] + lift[n][0] : fmaf(s[kb][n][2 * x], qs[n][0], lift[n][0]));
                        const float p1 = exp2_fast(LIST ? s[kb][n][2 * x + 1] + lift[n][1] : fmaf(s[kb][n][2 * x + 1], qs[n][1], lift[n][1]));
                        l[n][0] += p0;
                        l[n][1] += p1;
                        const uint32_t hi = half2_bits(p0, p1);
                        pb[0][kb][n][x] = transpose8x8(hi);
                        if constexpr (PARTS == 2) pb[1][kb][n][x] = transpose8x8(half2_rest(p0, p1, hi));
                    }
            }
            // ---- O^T += V^T P^T: lane row g of step i has numbers D / 8 g + 2 i and, 8 rows on, + 2 i + 1 ----
            uint32_t vw[2][2][2][VB / 4], vs[2][2];              // [block][rows 2t, 2t + 8][row, next row][word]
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const unsigned char *row = rows + (kb * 16 + x * 8 + 2 * t) * R::BYTES;
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        if constexpr (D == 128) {
                            const uint2 c = *reinterpret_cast<const uint2 *>(row + y * R::BYTES + R::CODES + g * VB);
                            vw[kb][x][y][0] = c.x;
                            vw[kb][x][y][1] = c.y;
                        } else {
                            vw[kb][x][y][0] = *reinterpret_cast<const uint32_t *>(row + y * R::BYTES + R::CODES + g * VB);
                        }
                    }
                    const int sg = R::SCALES + R::GROUPS + (D == 128 ? g : g / 2);
                    vs[kb][x] = scale4_half2(row[sg], row[R::BYTES + sg]);
                }
#pragma unroll
            for (int w = 0; w < VB / 4; ++w) {
                uint32_t even[2][2][4], odd[2][2][4];            // numbers 2 i and 2 i + 1 of rows (2t, 2t + 1), i = 4 w ..
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const uint32_t r0 = vw[kb][x][0][w], r1 = vw[kb][x][1][w];
                        codes8_to_half2(low_of_high_of(r0, r1 << 4), even[kb][x]);
                        codes8_to_half2(low_of_high_of(r0 >> 4, r1), odd[kb][x]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            even[kb][x][i] = hmul2_bits(even[kb][x][i], vs[kb][x]);
                            odd[kb][x][i] = hmul2_bits(odd[kb][x][i], vs[kb][x]);
                        }
                    }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t a0[4] = {even[0][0][i], odd[0][0][i], even[0][1][i], odd[0][1][i]};
                    const uint32_t a1[4] = {even[1][0][i], odd[1][0][i], even[1][1][i], odd[1][1][i]};
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float(&acc)[4] = o[n][4 * w + i];
                        if constexpr (PARTS == 1) {
                            mma_f16(acc, a0, pb[0][0][n][0], pb[0][0][n][1]);
                            mma_f16(acc, a1, pb[0][1][n][0], pb[0][1][n][1]);
                        } else {
                            float c[4];
                            mma_f16_first(c, a0, pb[1][0][n][0], pb[1][0][n][1]);
                            mma_f16(c, a1, pb[1][1][n][0], pb[1][1][n][1]);
                            mma_f16(c, a0, pb[0][0][n][0], pb[0][0][n][1]);
                            mma_f16(c, a1, pb[0][1][n][0], pb[0][1][n][1]);
#pragma unroll
                            for (int x = 0; x < 4; ++x) acc[x] += c[x];
                        }
                    }
                }
            }
            while (nan_rows) {
                const int row = __ffs(nan_rows) - 1;
                nan_rows &= nan_rows - 1;
                const uint32_t groups = __shfl_sync(0xffffffffu, nan_groups, row);
                if ((groups >> (D == 128 ? g : g / 2)) & 1u)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int y = 0; y < 2; ++y)
                            if (tile * A4_TILE + row < seen[n][y])
#pragma unroll
                                for (int i = 0; i < KS; ++i) o[n][i][y] = o[n][i][2 + y] = __int_as_float(0x7fffffff);
            }
            __syncwarp();                                        // (the next round overwrites this stage)
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();

        // ---- the warps' results, joined in the order of the warps ----
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int y = 0; y < 2; ++y) {
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) l[n][y] += __shfl_xor_sync(0xffffffffu, l[n][y], off);
                // (a maximum passes over NaN: a vector all of whose logits are NaN has seen something, too)
                if (ref[n][y] == -INFINITY && l[n][y] != 0.f) ref[n][y] = 0.f;
                const int v = n * 8 + 2 * t + y;
                if (g == 0) {
                    ml[(warp * N + v) * 2] = ref[n][y];
                    ml[(warp * N + v) * 2 + 1] = l[n][y];
                }
                float *to = reinterpret_cast<float *>(ring) + v * C::OD + g * (D / 8);
#pragma unroll
                for (int i = 0; i < KS; i += 2)
                    *reinterpret_cast<float4 *>(to + 2 * i) = make_float4(o[n][i][y], o[n][i][2 + y], o[n][i + 1][y], o[n][i + 1][2 + y]);
            }
        }
        __syncthreads();
        {
            const int v = q_vec, sub = q_sub;
            float m = -INFINITY;
#pragma unroll
            for (int i = 0; i < A4_WARPS; ++i) m = fmaxf(m, ml[(i * N + v) * 2]);
            float den = 0.f, acc[EACH];
#pragma unroll
            for (int e = 0; e < EACH; ++e) acc[e] = 0.f;
#pragma unroll
            for (int i = 0; i < A4_WARPS; ++i) {
                const float mi = ml[(i * N + v) * 2];
                if (mi == -INFINITY) continue;                   // (has seen nothing)
                const float share = exp2_fast(mi - m);
                den = fmaf(ml[(i * N + v) * 2 + 1], share, den);
                const float *from = reinterpret_cast<const float *>(smem + i * C::WARP_BYTES) + v * C::OD;
#pragma unroll
                for (int e = 0; e < EACH; ++e) acc[e] = fmaf(from[sub + e * PER], share, acc[e]);
            }
            if (a.cluster > 1) {
                // joined among the cluster's CTAs in their order: each leaves its sums in its shared memory and takes a share of the numbers
                __syncthreads();
                float *sums = reinterpret_cast<float *>(smem);
                float2 *own = reinterpret_cast<float2 *>(ml);
#pragma unroll
                for (int e = 0; e < EACH; ++e) sums[v * D + sub + e * PER] = acc[e];
                if (sub == 0) own[v] = make_float2(m, den);
                namespace cg = cooperative_groups;
                cg::cluster_group cluster = cg::this_cluster();
                cluster.sync();
                const int share_of = N * D / a.cluster, x0 = (int)(blockIdx.x % a.cluster) * share_of;
                for (int x = x0 + threadIdx.x; x < x0 + share_of; x += A4_THREADS) {
                    const int vx = x / D;
                    float mx = -INFINITY, dx = 0.f, ox = 0.f;
#pragma unroll 4
                    for (int i = 0; i < a.cluster; ++i) mx = fmaxf(mx, cluster.map_shared_rank(own, i)[vx].x);
#pragma unroll 4
                    for (int i = 0; i < a.cluster; ++i) {
                        const float2 part = cluster.map_shared_rank(own, i)[vx];
                        const float share = part.x == -INFINITY ? 0.f : exp2_fast(part.x - mx);
                        dx = fmaf(part.y, share, dx);
                        ox = fmaf(cluster.map_shared_rank(sums, i)[x], share, ox);
                    }
                    if (vx < vectors) {
                        const int vv = vec0 + vx, tok = vv / a.rep, head = h * a.rep + vv % a.rep;
                        T *to = (T *)a.o + (a.cu ? (int64_t)(rq.first_token + tok) * a.os[2] : b * a.os[0] + tok * a.os[2]) + head * a.os[1];
                        store_from(to, x % D, dx == 0.f ? 0.f : ox / dx);
                    }
                }
                cluster.sync();                                  // (nobody leaves while its shared memory is read)
            } else if (whole) {
                if (v < vectors) {
                    const int vv = vec0 + v, tok = vv / a.rep, head = h * a.rep + vv % a.rep;
                    T *to = (T *)a.o + (a.cu ? (int64_t)(rq.first_token + tok) * a.os[2] : b * a.os[0] + tok * a.os[2]) + head * a.os[1];
                    const float inv = m == -INFINITY ? 0.f : 1.f / den;
#pragma unroll
                    for (int e = 0; e < EACH; ++e) store_from(to, sub + e * PER, acc[e] * inv);
                }
            } else {
                const int64_t slot = (2 * blockIdx.x + (first_segment ? 0 : 1)) * N + v;
                float *to = a.part + slot * D;
#pragma unroll
                for (int e = 0; e < EACH; ++e) to[sub + e * PER] = acc[e];
                if (sub == 0) reinterpret_cast<float2 *>(a.part + (int64_t)2 * gridDim.x * N * D)[slot] = make_float2(m, den);
            }
        }
        __syncthreads();
    }
}

// Joins the parts of a problem (request, KV head, group) that stretches share, in their order; a CTA per problem and slice of its numbers, or, with
// more problems than stretches, a CTA per stretch but the first, which takes the problem that its stretch goes on with if no stretch before it did
// (so that a bound of the queries that is far too high costs nothing).
// With few problems of many parts a problem's numbers are cut into slices, so that more CTAs read (8 problems of 32768 rows, 74 parts each:
// one CTA per problem took longer than the attention itself).  Each number's parts are dealt to SHARE threads.
constexpr int A4_MERGE_THREADS = 256;
constexpr int A4_MERGE_PARTS = 64;       // parts whose shares are held at a time
template <typename T, int D, int NT, int SLICES>
__global__ void __launch_bounds__(A4_MERGE_THREADS) attend4_merge_kernel(const __grid_constant__ Attend4Args a, int ctas_launched, int max_groups)
{
    constexpr int N = 8 * NT, SLICE = N * D / SLICES;            // numbers of a CTA
    constexpr int SHARE = SLICE < A4_MERGE_THREADS ? A4_MERGE_THREADS / SLICE : 1, EACH = SLICE * SHARE / A4_MERGE_THREADS;
    constexpr int ROWS = A4_MERGE_THREADS / N;
    extern __shared__ __align__(16) unsigned char smem[];
    int64_t *prefix = reinterpret_cast<int64_t *>(smem);
    __shared__ int64_t part[A4_MERGE_THREADS / 32];
    __shared__ float top[ROWS][N], share[A4_MERGE_PARTS][N], den_of[A4_MERGE_PARTS][N], sums[SHARE][2][SHARE > 1 ? SLICE : 1];
    // lengths and cu are older than the launch before this one, whose CTAs let this one start when they had waited for them.  Its parts are
    // not: every CTA waits for it, those without anything to join too, for what follows in the stream waits for this launch alone.
    const int64_t total = lay_line(a, N, prefix, part);
    cudaGridDependencySynchronize();
    const int ctas = stretches(total, ctas_launched);
    int b, h, group;
    Request rq;
    if (max_groups > 0) {
        b = blockIdx.x / (a.pool.kv_heads * max_groups);
        const int rest = blockIdx.x % (a.pool.kv_heads * max_groups);
        h = rest / max_groups;
        group = rest % max_groups;
        rq = request_from(a, line_known(prefix, a.batch)[b], N);
        if (group >= rq.groups) return;
    } else {
        if ((int)blockIdx.x + 1 >= ctas) return;
        const int64_t f = div_small(total * (blockIdx.x + 1), ctas);
        b = request_of(prefix, a.batch, f);
        rq = request_from(a, line_known(prefix, a.batch)[b], N);
        const int problem = (int)div_small(f - prefix[b], rq.places);
        h = problem / rq.groups;
        group = problem - h * rq.groups;
    }
    const int64_t f0 = prefix[b] + (int64_t)(h * rq.groups + group) * rq.places, f1 = f0 + rq.places;
    // stretch c is [total c / ctas, total (c + 1) / ctas): the one that place f is in
    const int64_t c0 = div_small((f0 + A4_START + 1) * ctas - 1, total), c1 = div_small(f1 * ctas - 1, total);
    if (c0 == c1 || (max_groups == 0 && c0 != (int64_t)blockIdx.x)) return;
    const int count = (int)(c1 - c0 + 1);
    // its second segment at most: the first stretch may have begun with another problem
    const int64_t slot0 = 2 * c0 + (div_small(total * c0, ctas) >= f0 ? 0 : 1);
    auto slot = [&](int i) { return i == 0 ? slot0 : 2 * (c0 + i); };
    const float2 *ml = reinterpret_cast<const float2 *>(a.part + (int64_t)2 * ctas_launched * N * D);
    const int v = threadIdx.x % N, r = threadIdx.x / N;
    // (reads of many parts are asked for eight at a time: one after the other each would take the time of a trip to L2)
    constexpr int AHEAD = SLICES > 1 ? 8 : 1;
    float m = -INFINITY;
    for (int i = r; i < count; i += AHEAD * ROWS) {
        float x[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) x[k] = i + k * ROWS < count ? ml[slot(i + k * ROWS) * N + v].x : -INFINITY;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) m = fmaxf(m, x[k]);
    }
    top[r][v] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ROWS; ++i) m = fmaxf(m, top[i][v]);
    const int sub = SHARE > 1 ? threadIdx.x / SLICE : 0, x0 = blockIdx.y * SLICE + (SHARE > 1 ? threadIdx.x % SLICE : threadIdx.x);
    float den[EACH], acc[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) den[e] = acc[e] = 0.f;
    for (int i0 = 0; i0 < count; i0 += A4_MERGE_PARTS) {
        const int here = min(A4_MERGE_PARTS, count - i0);
#pragma unroll
        for (int k = 0; k < (A4_MERGE_PARTS + ROWS - 1) / ROWS; ++k) {
            const int i = r + k * ROWS;
            if (i >= A4_MERGE_PARTS) continue;
            const float2 x = i < here ? ml[slot(i0 + i) * N + v] : make_float2(-INFINITY, 0.f);
            share[i][v] = x.x == -INFINITY ? 0.f : exp2_fast(x.x - m);
            den_of[i][v] = x.y;
        }
        __syncthreads();
        constexpr int BATCH = SLICES > 1 ? 8 : EACH > 4 ? 2 : 4;
        for (int i = sub; i < here; i += BATCH * SHARE) {
            float x[BATCH][EACH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k)
#pragma unroll
                for (int e = 0; e < EACH; ++e)
                    x[k][e] = i + k * SHARE < here ? a.part[slot(i0 + i + k * SHARE) * N * D + x0 + e * A4_MERGE_THREADS] : 0.f;
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int at = min(i + k * SHARE, A4_MERGE_PARTS - 1);
                if (i + k * SHARE >= here) continue;
#pragma unroll
                for (int e = 0; e < EACH; ++e) {
                    const int ve = (x0 + e * A4_MERGE_THREADS) / D;
                    acc[e] = fmaf(x[k][e], share[at][ve], acc[e]);
                    den[e] = fmaf(den_of[at][ve], share[at][ve], den[e]);
                }
            }
        }
        __syncthreads();
    }
    if constexpr (SHARE > 1) {
        sums[sub][0][threadIdx.x % SLICE] = acc[0];
        sums[sub][1][threadIdx.x % SLICE] = den[0];
        __syncthreads();
        if (sub) return;
#pragma unroll
        for (int i = 1; i < SHARE; ++i) {
            acc[0] += sums[i][0][threadIdx.x];
            den[0] += sums[i][1][threadIdx.x];
        }
    }
    const int vec0 = group * N;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int x = x0 + e * A4_MERGE_THREADS, vv = vec0 + x / D;
        if (vv >= rq.tokens * a.rep) continue;
        const int tok = vv / a.rep, head = h * a.rep + vv % a.rep;
        T *to = (T *)a.o + (a.cu ? (int64_t)(rq.first_token + tok) * a.os[2] : b * a.os[0] + tok * a.os[2]) + head * a.os[1];
        store_from(to, x % D, den[e] == 0.f ? 0.f : acc[e] / den[e]);
    }
}

constexpr int A4_MAX_CTAS_PER_SM = 8;    // what the workspace has room for

template <typename T, int D, int NT, int PARTS, bool LIST> int launch_attend4_form(Attend4Args a, cudaStream_t st)
{
    using C = A4<D, NT, PARTS>;
    auto kern = attend4_kernel<T, D, NT, PARTS, LIST>;
    // CTAs per SM, asked once per device and size of the line (threads that meet here first find the same answer)
    static std::atomic<int> known[64][3];
    const int big = a.batch <= A4_FEW ? 0 : a.batch <= A4_SOME ? 1 : 2;
    const int smem = C::total(big == 0 ? A4_FEW : big == 1 ? A4_SOME : A4_MAX_BATCH);
    int dev = 0;
    ELM_CUDA_TRY(cudaGetDevice(&dev));
    int per_sm = dev < 64 ? known[dev][big].load(std::memory_order_relaxed) : 0;
    if (per_sm == 0) {
        ELM_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::total(A4_MAX_BATCH)));
        ELM_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, A4_THREADS, smem));
        per_sm = per_sm < 1 ? 1 : (per_sm > A4_MAX_CTAS_PER_SM ? A4_MAX_CTAS_PER_SM : per_sm);
        if (dev < 64) known[dev][big].store(per_sm, std::memory_order_relaxed);
    }
    a.max_groups = (int)(((int64_t)a.n_q * a.rep + C::N - 1) / C::N);
    const int max_groups = a.max_groups;
    const int64_t problems = (int64_t)a.batch * a.pool.kv_heads * max_groups;
    if (problems > 0x7fffffff / 16) return ELM_ERR_SHAPE;
    // Short problems, so few that a cluster for each is resident at once, are done in one launch: as many CTAs as give a warp two tiles (at
    // most 16 CTAs with up to four tiles a warp); a single CTA each where they have no more than 8 tiles.
    const int tiles = (a.n_kv + A4_TILE - 1) / A4_TILE;
    for (int size = 1; size <= 16; size *= 2) {
        if (tiles > size * A4_WARPS * (size == 16 ? 4 : 2)) continue;
        // (the queries of a request may be far fewer than their bound: then CTAs by the bound would be mostly idle ones.  Rows of 200 and 1 token a
        // request, a CTA each against the line of tiles: 28 problems by the bound to an SM 45 against 50 us, 55 to an SM 53 against 50, 221 99 against 49.
        // Where all the bound's tokens are there the CTAs are the faster by 5 to 45 %, which those calls above the limit do without: 154 against 163)
        if (size == 1 && a.cu && max_groups > 1 && problems > 32 * (int64_t)device_sm_count()) continue;
        if (size > 1) {
            static std::atomic<int> resident[64][5];
            const int at = size == 2 ? 0 : size == 4 ? 1 : size == 8 ? 2 : 3;
            int clusters = dev < 64 ? resident[dev][at].load(std::memory_order_relaxed) : 0;
            if (clusters == 0) {
                // (+ 1: 0 is not known yet.  Asked with the largest line: the question sets the kernel's limit)
                clusters = resident_clusters(kern, A4_THREADS, C::total(A4_MAX_BATCH), size) + 1;
                if (dev < 64) resident[dev][at].store(clusters, std::memory_order_relaxed);
            }
            if (problems > clusters - 1) continue;
        }
        a.cluster = size;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)size;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(problems * size));
        cfg.blockDim = dim3(A4_THREADS);
        cfg.dynamicSmemBytes = (size_t)smem;
        cfg.stream = st;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        ELM_CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, a));
        count_launches(1);
        return cuda_status(cudaGetLastError());
    }
    // no more CTAs than the longest line of tiles has stretches
    const int64_t places = problems * (A4_START + (a.n_kv + A4_TILE - 1) / A4_TILE);
    const int grid = stretches(places, per_sm * device_sm_count());
    ELM_CUDA_TRY(launch_after(kern, dim3((unsigned)grid), dim3(A4_THREADS), smem, st, a));
    count_launches(1);
    // slices of 32 or 128 numbers where the problems alone are few.  Slices of 32 / of 128 / none, us for bf16 rows of 32768 each, d = 128: 1 problem
    // 14 / 15 / 29, 8 23 / 25 / 33, 16 27 / 28 / 35, 32 43 / 41 / 41, 40 49 / 45 / 47; 128 of 8192 60 / 43 / 41.  Of 96 such calls (d, types, 8 and
    // 16 vectors) the rule takes a form more than 5 % slower than the best in 8, by 14 % at most.
    constexpr int FINE = C::N * D / 32, COARSE = C::N * D / 128;
    const int slices = problems * FINE <= 2 * device_sm_count() ? FINE : problems * COARSE <= 2 * device_sm_count() ? COARSE : 1;
    auto join = slices == FINE ? attend4_merge_kernel<T, D, NT, FINE> : slices == COARSE ? attend4_merge_kernel<T, D, NT, COARSE> : attend4_merge_kernel<T, D, NT, 1>;
    const bool by_stretch = slices == 1 && problems >= grid;
    if (by_stretch && grid == 1) return cuda_status(cudaGetLastError());       // (one stretch: nothing to join)
    const dim3 join_grid(by_stretch ? (unsigned)(grid - 1) : (unsigned)problems, (unsigned)slices);
    ELM_CUDA_TRY(launch_after(join, join_grid, dim3(A4_MERGE_THREADS), line_bytes(a.batch), st, a, grid, by_stretch ? 0 : max_groups));
    count_launches(1);
    return cuda_status(cudaGetLastError());
}
template <typename T, int D, int NT, int PARTS> int launch_attend4(const Attend4Args &a, cudaStream_t st)
{
    return a.idx ? launch_attend4_form<T, D, NT, PARTS, true>(a, st) : launch_attend4_form<T, D, NT, PARTS, false>(a, st);
}

bool zeros(const int64_t (&s)[3]) { return s[0] == 0 && s[1] == 0 && s[2] == 0; }

int check(const elm_cache4_params *p, bool list, int &shift, int64_t &n_kv)
{
    if (p->dtype != ELM_F32 && p->dtype != ELM_BF16) return ELM_ERR_DTYPE;
    if (p->batch < 1 || p->batch > A4_MAX_BATCH || p->kv_heads < 1 || p->q_heads < 1 || p->q_heads % p->kv_heads != 0) return ELM_ERR_SHAPE;
    if ((int64_t)p->batch * p->q_heads > 65535 || (p->d != 64 && p->d != 128)) return ELM_ERR_SHAPE;
    if (p->n_q < 1 || p->n_tokens < 0 || p->n_kv < 0 || (list && p->n_kv < 1) || p->max_pages < 1) return ELM_ERR_SHAPE;
    shift = page_shift_of(p->page_rows);
    if (shift < 0 || !pool_fits(p->n_pages, p->page_rows, p->kv_heads)) return ELM_ERR_SHAPE;
    const int64_t capacity = (int64_t)p->max_pages << shift;
    if (capacity > 0x7fffffff - 64) return ELM_ERR_SHAPE;
    n_kv = list ? p->n_kv : (p->n_kv == 0 || p->n_kv > capacity ? capacity : p->n_kv);
    if (n_kv > 0x7fffffff - 64 || (int64_t)p->n_q * (p->q_heads / p->kv_heads) > 0x7fffffff / 2) return ELM_ERR_SHAPE;
    return ELM_OK;
}

elm_params as_attend(const elm_cache4_params *p)
{
    elm_params e = {};
    e.batch = p->batch;
    e.q_heads = p->q_heads;
    e.kv_heads = p->kv_heads;
    e.n_kv = p->n_kv;
    e.n_q = p->n_q;
    e.d = p->d;
    e.dtype = ELM_BF16;
    e.precision = ELM_PREC_FP32;
    e.delta = 0.5;
    return e;
}

// Lists met by so many queries that the tensor-core kernel of elm_attend over a gathered copy, 256 queries of a head at a time, is the faster
// way.  Both forms' times in us, as they were fitted at d = 128; measured (fitted) for 8 KV heads x 4, 2048 entries:
//   here     9 + 0.9 (A4_START + tiles) per CTA slot and problem     64 queries 31 (24), 128 44 (39), 256 71 (68), 1024 222 (246)
//   there   14 + 2.2 per block of 128 entries and wave of items                 49 (49),     51 (49),     51 (49),       51 (49)
// Of 112 calls each (1, 4, 8 and 32 KV heads, 1 to 8 query heads to one, 256 to 16384 entries, 8 to 1024 queries) the faster form is taken in 109 at
// d = 128, a form 1.12 times as slow at most in the others.  At d = 64 `here` takes 0.53 instead of 0.9 and `there` 0.9 of its time, for which the rule
// makes no difference: the second form comes too early in 8 of the 112, by 1.41 times at most (8 heads x 4, 256 entries, 256 queries: 15 against 21 us).
// With 8 queries the first form is up to 20 times as fast, with 1024 the second up to 5 times.  Its gathered copy has to fit the workspace: 552 bytes an
// entry and KV head (d = 64: 296), a twentieth of the GPU's memory at most (15 M entries), which also keeps clear of what that kernel can count.
constexpr size_t A4_MAX_COPY = (size_t)8 << 30;
bool by_tensor_cores(const elm_cache4_params *p, bool list)
{
    if (!list || p->dtype != ELM_BF16 || !zeros(p->q_stride) || !zeros(p->o_stride)) return false;
    const int sms = device_sm_count();
    const int64_t rep = p->q_heads / p->kv_heads, vectors = rep * p->n_q <= 8 ? 8 : 16;
    const double problems = (double)p->batch * p->kv_heads * ((rep * p->n_q + vectors - 1) / vectors);
    const double here = 9.0 + 0.9 * problems * (A4_START + (p->n_kv + A4_TILE - 1) / A4_TILE) / (4.0 * sms);
    const int64_t items = (int64_t)p->batch * p->q_heads * ((p->n_q + 255) / 256), waves = (items + sms - 1) / sms;
    const double there = 14.0 + 2.2 * (double)waves * ((p->n_kv + 127) / 128);
    if (there >= here) return false;
    const elm_params e = as_attend(p);
    return attend_layout(&e, p->n_kv).total <= A4_MAX_COPY;
}

size_t workspace_of(const elm_cache4_params *p, bool list)
{
    if (by_tensor_cores(p, list)) {
        const elm_params e = as_attend(p);
        return attend_layout(&e, p->n_kv).total;
    }
    const int vectors = (int64_t)p->n_q * (p->q_heads / p->kv_heads) <= 8 ? 8 : 16;
    return (size_t)2 * A4_MAX_CTAS_PER_SM * device_sm_count() * vectors * (p->d + 2) * sizeof(float);
}

}  // namespace
}  // namespace elm

using namespace elm;

extern "C" int elm_cache4_attend_workspace_bytes(const elm_cache4_params *p, int32_t with_list, size_t *bytes)
{
    if (!p || !bytes) return ELM_ERR_NULL;
    int shift;
    int64_t n_kv;
    const int rc = check(p, with_list != 0, shift, n_kv);
    if (rc != ELM_OK) return rc;
    *bytes = workspace_of(p, with_list != 0);
    return ELM_OK;
}

extern "C" int elm_cache4_attend(const void *Q, const void *rows, const int32_t *table, const int32_t *length, const int32_t *cu,
                                 const int32_t *idx, const float *w, const elm_cache4_params *p, void *O, void *workspace,
                                 size_t workspace_bytes, void *stream)
{
    if (!p) return ELM_ERR_NULL;
    const bool list = idx != nullptr;
    int shift;
    int64_t n_kv;
    const int rc = check(p, list, shift, n_kv);
    if (rc != ELM_OK) return rc;
    if (!Q || !rows || !table || !O || !workspace || (list ? !w : !length)) return ELM_ERR_NULL;
    if (list && (length || cu)) return ELM_ERR_SHAPE;                       // exactly one of the two forms
    if (((uintptr_t)Q | (uintptr_t)O | (uintptr_t)rows) & 15 || ((uintptr_t)workspace & 255)) return ELM_ERR_ALIGN;
    if (((uintptr_t)table | (uintptr_t)length | (uintptr_t)cu | (uintptr_t)idx | (uintptr_t)w) & 3) return ELM_ERR_ALIGN;
    if (workspace_bytes < workspace_of(p, list)) return ELM_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)stream;
    Attend4Args a = {};
    a.pool = Pool4{(const unsigned char *)rows, table, p->n_pages, p->max_pages, shift, p->kv_heads};
    if (by_tensor_cores(p, list)) {
        const elm_params e = as_attend(p);
        AttendWindow win;
        win.pool4 = &a.pool;
        return attend_tc((const __nv_bfloat16 *)Q, nullptr, nullptr, idx, w, p->n_kv, &e, (__nv_bfloat16 *)O, (unsigned char *)workspace, st, true, win);
    }
    a.q = Q;
    a.o = O;
    a.length = length;
    a.cu = cu;
    a.idx = idx;
    a.w = w;
    a.part = (float *)workspace;
    const int64_t d = p->d, heads = p->q_heads;
    const int64_t dense[3] = {heads * p->n_q * d, cu ? d : p->n_q * d, cu ? heads * d : d};
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = zeros(p->q_stride) ? dense[i] : p->q_stride[i];
        a.os[i] = zeros(p->o_stride) ? dense[i] : p->o_stride[i];
    }
    a.q_wide = (a.qs[0] * (int64_t)elt_bytes(p->dtype)) % 8 == 0 && (a.qs[1] * (int64_t)elt_bytes(p->dtype)) % 8 == 0 && (a.qs[2] * (int64_t)elt_bytes(p->dtype)) % 8 == 0;
    // rows of O that would be written twice
    if ((!cu && p->batch > 1 && a.os[0] == 0) || (p->q_heads > 1 && a.os[1] == 0) || ((cu ? p->n_tokens : p->n_q) > 1 && a.os[2] == 0)) return ELM_ERR_SHAPE;
    a.batch = p->batch;
    a.q_heads = p->q_heads;
    a.rep = p->q_heads / p->kv_heads;
    a.n_kv = (int32_t)n_kv;
    a.n_q = p->n_q;
    a.n_tokens = p->n_tokens;
    a.causal = p->causal;
    const bool few = (int64_t)p->n_q * a.rep <= 8;
    typedef __nv_bfloat16 bf;
    if (p->dtype == ELM_BF16) {
        if (p->d == 64) return few ? launch_attend4<bf, 64, 1, 1>(a, st) : launch_attend4<bf, 64, 2, 1>(a, st);
        return few ? launch_attend4<bf, 128, 1, 1>(a, st) : launch_attend4<bf, 128, 2, 1>(a, st);
    }
    if (p->d == 64) return few ? launch_attend4<float, 64, 1, 2>(a, st) : launch_attend4<float, 64, 2, 2>(a, st);
    return few ? launch_attend4<float, 128, 1, 2>(a, st) : launch_attend4<float, 128, 2, 2>(a, st);
}

extern "C" int elm_cache4_attend_status(const void *workspace, const elm_cache4_params *p, int32_t with_list, int32_t *status_host, void *stream)
{
    if (!workspace || !p || !status_host) return ELM_ERR_NULL;
    int shift;
    int64_t n_kv;
    const int rc = check(p, with_list != 0, shift, n_kv);
    if (rc != ELM_OK) return rc;
    if (by_tensor_cores(p, with_list != 0)) {
        const elm_params e = as_attend(p);
        return elm_attend_status(workspace, &e, p->n_kv, status_host, stream);
    }
    ELM_CUDA_TRY(cudaStreamSynchronize((cudaStream_t)stream));
    *status_host = 0;                                                       // (nothing waits in that form)
    return ELM_OK;
}
