// Pages, positions and slots of a step's new tokens from the requests' lengths, on the device (elm_page_plan), and pages given
// back (elm_page_release).
//
//   need_b = ceil((length_b + n_b) / P) - ceil(length_b / P);  request b is served iff it fits its table and the step's places and
//   need_b = 0 or need_0 + ... + need_b <= free;  its i-th new page is free[count - 1 - (need_0 + ... + need_(b-1)) - i].
// (Once the sum exceeds what is free it does for every later request that wants a page, so the requests that are served stand
// before those that are not, and the sum before each of them counts served requests only.)
//
// A few hundred numbers: bound by the launch and by one CTA's chain of reads, scans and barriers.  One CTA does the requests, 1024 at
// a time, and, in a step of few places, the places as well (256 requests: 6 us); more places go to a second launch, resident before the first has ended
// (61 prompts, 33 K places: 12 us the two).
#include "elm_common.cuh"

namespace elm {
namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_KEPT = 4096;          // requests whose places are kept in shared memory
constexpr int PLAN_PLACES = 4096;        // places the first launch fills itself
constexpr int FILL_THREADS = 256, FILL_EACH = 4;

// inclusive sum over the CTA's threads; `part` has a place for each warp, and `total` is the sum over all
__device__ __forceinline__ int64_t block_sum(int64_t x, int64_t *part, int64_t &total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();                     // (the parts of the sum before this one have been read)
    if (lane == 31) part[warp] = x;
    __syncthreads();
    int64_t p = part[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, p, o);
        if (lane >= o) p += y;
    }
    total = __shfl_sync(0xffffffffu, p, 31);
    const int64_t before = __shfl_sync(0xffffffffu, p, warp ? warp - 1 : 0);
    return x + (warp ? before : 0);
}

struct PlanArgs {
    int32_t *table;
    const int32_t *length, *n_new, *free, *free_count;
    int32_t *start_out, *length_out, *free_count_out, *cu_out, *position_out, *slot_out;
    int32_t batch, max_pages, page_shift, max_tokens, n_free;
};

// whether some pool can have the page: one whose rows' numbers pass 2^31 - 1 is none (modulo 2^32 they would be another page's)
__device__ __forceinline__ bool is_page(int32_t page, int page_shift) { return (uint32_t)page < (0x7fffffffu >> page_shift); }

// last b in [lo, hi] with cu[b] <= t (cu[lo] <= t)
template <typename Cu> __device__ __forceinline__ int request_of(const Cu &cu, int lo, int hi, int t)
{
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cu(mid) <= t) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ void fill_place(const PlanArgs &a, int t, int b, int cu_b, int start)
{
    int32_t pos = -1, slot = -1;
    if (start >= 0) {
        pos = start + (t - cu_b);
        const int32_t page = a.table[(int64_t)b * a.max_pages + (pos >> a.page_shift)];
        if (is_page(page, a.page_shift)) slot = (page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
    }
    a.position_out[t] = pos;
    a.slot_out[t] = slot;
}

__global__ void __launch_bounds__(PLAN_THREADS) page_plan_kernel(const __grid_constant__ PlanArgs a)
{
    __shared__ int64_t part[32];
    __shared__ int64_t upto[PLAN_THREADS];                     // pages wanted up to and with each request of the chunk
    __shared__ int32_t held_of[PLAN_THREADS];                  // its table entries before the step; -1: not served
    __shared__ int32_t cu[PLAN_KEPT + 1], start[PLAN_KEPT];
    cudaGridDependencySynchronize();
    const int32_t page = 1 << a.page_shift;
    int64_t tokens = 0, wanted = 0, taken = 0;
    int64_t count = *a.free_count;
    count = count < 0 ? 0 : (count > a.n_free ? a.n_free : count);
    for (int b0 = 0; b0 < a.batch; b0 += PLAN_THREADS) {
        const int b = b0 + threadIdx.x;
        const bool live = b < a.batch;
        const int32_t len = live ? a.length[b] : 0, raw = live ? a.n_new[b] : 0;
        const int32_t n = raw > 0 ? raw : 0;
        int64_t all;
        const int64_t place = tokens + block_sum(n, part, all) - n;
        tokens += all;
        const int64_t after = (int64_t)len + n;
        const bool fits = live && raw >= 0 && len >= 0 && after <= ((int64_t)a.max_pages << a.page_shift) && place + n <= a.max_tokens;
        const int64_t held = (len + (int64_t)page - 1) >> a.page_shift;
        const int64_t need = fits ? ((after + page - 1) >> a.page_shift) - held : 0;
        const int64_t sum = wanted + block_sum(need, part, all);
        const bool ok = fits && (need == 0 || sum <= count);
        int64_t served;
        block_sum(ok ? need : 0, part, served);
        upto[threadIdx.x] = sum - wanted;
        held_of[threadIdx.x] = ok ? (int32_t)held : -1;
        if (live) {
            const int32_t at = (int32_t)(place < 0x7fffffff ? place : 0x7fffffff);
            a.start_out[b] = ok ? len : -1;
            a.length_out[b] = ok ? (int32_t)after : len;
            a.cu_out[b] = at;
            if (b < PLAN_KEPT) {
                cu[b] = at;
                start[b] = ok ? len : -1;
            }
        }
        __syncthreads();
        // the pages of the requests that are served: the first `served` of those wanted by the chunk
        for (int64_t k = threadIdx.x; k < served; k += PLAN_THREADS) {
            int lo = 0, hi = PLAN_THREADS - 1;                 // first request whose sum is above k
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (upto[mid] > k) hi = mid;
                else lo = mid + 1;
            }
            const int64_t before = lo ? upto[lo - 1] : 0;
            a.table[(int64_t)(b0 + lo) * a.max_pages + held_of[lo] + (k - before)] = a.free[count - 1 - (wanted + k)];
        }
        wanted += all;
        taken += served;
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        const int32_t at = (int32_t)(tokens < 0x7fffffff ? tokens : 0x7fffffff);
        a.cu_out[a.batch] = at;
        if (a.batch <= PLAN_KEPT) cu[a.batch] = at;
        *a.free_count_out = (int32_t)(count - taken);
    }
    if (a.max_tokens > PLAN_PLACES || a.batch > PLAN_KEPT) return;       // (the second launch fills the places)
    __syncthreads();
    for (int t = threadIdx.x; t < a.max_tokens; t += PLAN_THREADS) {
        if (t < cu[a.batch]) {
            const int b = request_of([&](int i) { return cu[i]; }, 0, a.batch - 1, t);
            fill_place(a, t, b, cu[b], start[b]);
        } else {
            a.position_out[t] = -1;
            a.slot_out[t] = -1;
        }
    }
}

__global__ void __launch_bounds__(FILL_THREADS) page_fill_kernel(const __grid_constant__ PlanArgs a)
{
    constexpr int EACH = FILL_THREADS * FILL_EACH;
    __shared__ int32_t range[2];
    __shared__ int32_t cu[EACH + 1], start[EACH];
    cudaGridDependencySynchronize();
    const int t0 = blockIdx.x * EACH;
    const int t1 = min(EACH, a.max_tokens - t0) + (t0 - 1);     // (t0 + EACH may be 2^31)
    const int total = a.cu_out[a.batch];
    // the requests of the CTA's first and last place, each found by a warp, 32 ways at a time
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x & 31, end = threadIdx.x >> 5;
        const int t = end ? t1 : t0;
        int lo = 0, width = a.batch;                           // cu[lo] <= t; the answer is in [lo, lo + width)
        while (width > 1) {
            const int step = (width + 31) / 32;
            const int at = lo + lane * step;
            const unsigned low = __ballot_sync(0xffffffffu, lane * step < width && a.cu_out[at] <= t);
            const int k = 31 - __clz(low);                     // (lane 0 always counts)
            lo += k * step;
            width = min(step, width - k * step);
        }
        if (lane == 0) range[end] = lo;
    }
    __syncthreads();
    const int b0 = range[0], b1 = range[1];
    const bool kept = b1 - b0 < EACH;
    if (kept) {
        for (int i = threadIdx.x; i <= b1 - b0; i += FILL_THREADS) {
            cu[i] = a.cu_out[b0 + i];
            start[i] = a.start_out[b0 + i];
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FILL_EACH; ++i) {
        const int at = i * FILL_THREADS + threadIdx.x, t = t0 + at;
        if (at > t1 - t0) continue;
        if (t >= total) {
            a.position_out[t] = -1;
            a.slot_out[t] = -1;
        } else if (kept) {
            const int b = request_of([&](int i) { return cu[i]; }, 0, b1 - b0, t);
            fill_place(a, t, b0 + b, cu[b], start[b]);
        } else {
            const int b = request_of([&](int i) { return a.cu_out[i]; }, b0, b1, t);
            fill_place(a, t, b, a.cu_out[b], a.start_out[b]);
        }
    }
}

struct ReleaseArgs {
    int32_t *table, *length;
    const int32_t *done;
    int32_t *free, *free_count;
    int32_t batch, max_pages, page_shift, n_free;
};

__global__ void __launch_bounds__(PLAN_THREADS) page_release_kernel(const __grid_constant__ ReleaseArgs a)
{
    __shared__ int64_t part[32];
    __shared__ int64_t upto[PLAN_THREADS];
    cudaGridDependencySynchronize();
    int64_t count = *a.free_count;
    count = count < 0 ? 0 : (count > a.n_free ? a.n_free : count);
    for (int b0 = 0; b0 < a.batch; b0 += PLAN_THREADS) {
        const int b = b0 + threadIdx.x;
        const bool ends = b < a.batch && a.done[b] != 0;
        int64_t held = ends ? ((int64_t)a.length[b] + (1 << a.page_shift) - 1) >> a.page_shift : 0;
        held = held < 0 ? 0 : (held > a.max_pages ? a.max_pages : held);
        int64_t all;
        upto[threadIdx.x] = block_sum(held, part, all);
        if (ends) a.length[b] = 0;
        __syncthreads();
        for (int64_t k0 = 0; k0 < all; k0 += PLAN_THREADS) {
            const int64_t k = k0 + threadIdx.x;
            int32_t page = -1;
            if (k < all) {
                int lo = 0, hi = PLAN_THREADS - 1;
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (upto[mid] > k) hi = mid;
                    else lo = mid + 1;
                }
                int32_t *entry = a.table + (int64_t)(b0 + lo) * a.max_pages + (k - (lo ? upto[lo - 1] : 0));
                page = is_page(*entry, a.page_shift) ? *entry : -1;
                *entry = -1;
            }
            int64_t back;
            const int64_t at = count + block_sum(page >= 0, part, back) - 1;
            if (page >= 0 && at < a.n_free) a.free[at] = page;
            count = count + back < a.n_free ? count + back : a.n_free;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) *a.free_count = (int32_t)count;
}

int check(const elm_page_params *p, int &shift)
{
    if (p->batch < 1 || p->batch > 65536 || p->max_pages < 1 || p->max_tokens < 0 || p->n_free < 0) return ELM_ERR_SHAPE;
    if (p->page_rows < 16 || p->page_rows > 1024 || (p->page_rows & (p->page_rows - 1))) return ELM_ERR_SHAPE;
    if ((int64_t)p->max_pages * p->page_rows > 0x7fffffff) return ELM_ERR_SHAPE;
    for (shift = 4; (1 << shift) < p->page_rows; ++shift) {}
    return ELM_OK;
}

}  // namespace
}  // namespace elm

using namespace elm;

extern "C" int elm_page_plan(int32_t *table, const int32_t *length, const int32_t *n_new, const int32_t *free, const int32_t *free_count,
                             const elm_page_params *p, int32_t *start_out, int32_t *length_out, int32_t *free_count_out, int32_t *cu_out,
                             int32_t *position_out, int32_t *slot_out, void *stream)
{
    if (!p) return ELM_ERR_NULL;
    int shift;
    const int rc = check(p, shift);
    if (rc != ELM_OK) return rc;
    if (!table || !length || !n_new || !free_count || !start_out || !length_out || !free_count_out || !cu_out) return ELM_ERR_NULL;
    if ((p->n_free > 0 && !free) || (p->max_tokens > 0 && (!position_out || !slot_out))) return ELM_ERR_NULL;
    if (((uintptr_t)table | (uintptr_t)length | (uintptr_t)n_new | (uintptr_t)free | (uintptr_t)free_count | (uintptr_t)start_out |
         (uintptr_t)length_out | (uintptr_t)free_count_out | (uintptr_t)cu_out | (uintptr_t)position_out | (uintptr_t)slot_out) & 3)
        return ELM_ERR_ALIGN;
    cudaStream_t st = (cudaStream_t)stream;
    const PlanArgs a = {table, length, n_new, free, free_count, start_out, length_out, free_count_out, cu_out, position_out, slot_out,
                        p->batch, p->max_pages, shift, p->max_tokens, p->n_free};
    ELM_CUDA_TRY(launch_after(page_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, a));
    count_launches(1);
    if (p->max_tokens > PLAN_PLACES || (p->batch > PLAN_KEPT && p->max_tokens > 0)) {
        const int each = FILL_THREADS * FILL_EACH;
        ELM_CUDA_TRY(launch_after(page_fill_kernel, dim3((unsigned)((p->max_tokens + (int64_t)each - 1) / each)), dim3(FILL_THREADS), 0, st, a));
        count_launches(1);
    }
    return cuda_status(cudaGetLastError());
}

extern "C" int elm_page_release(int32_t *table, int32_t *length, const int32_t *done, int32_t *free, int32_t *free_count,
                                const elm_page_params *p, void *stream)
{
    if (!p) return ELM_ERR_NULL;
    int shift;
    const int rc = check(p, shift);
    if (rc != ELM_OK) return rc;
    if (!table || !length || !done || !free_count || (p->n_free > 0 && !free)) return ELM_ERR_NULL;
    if (((uintptr_t)table | (uintptr_t)length | (uintptr_t)done | (uintptr_t)free | (uintptr_t)free_count) & 3) return ELM_ERR_ALIGN;
    const ReleaseArgs a = {table, length, done, free, free_count, p->batch, p->max_pages, shift, p->n_free};
    ELM_CUDA_TRY(launch_after(page_release_kernel, dim3(1), dim3(PLAN_THREADS), 0, (cudaStream_t)stream, a));
    count_launches(1);
    return cuda_status(cudaGetLastError());
}
