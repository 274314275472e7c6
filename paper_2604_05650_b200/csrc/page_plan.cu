// Page tables of a decoding step: which free pages the requests take for their new tokens, the
// block table's new entries, and the cache slot of every new token.
//
// With lengths l_b, new tokens n_b, pages held h_b and pages of P positions:
//   need_b = max(0, ceil((l_b + n_b) / P) - h_b)     pages request b takes,
//   U_b    = sum of need over requests up to b       (in request order; the stack is popped in it),
//   slot(i of b) = page * P + pos % P,  pos = l_b + i,  page = logical page pos / P of request b.
//
// Nothing here is heavy: 4 bytes written per new token, a few words per request.  What counts is
// latency, so it is one launch: every CTA loads all requests (at most 1024, four per thread) and
// makes the two prefix sums itself in shared memory (one round of shuffles) instead of waiting for
// another CTA's, then fills its own part of the slot map and of the new table entries, finding the
// request of an index by binary search.  The lengths, held counts and the free count may be
// updated in place: they are written by the last CTA to have read them (a ticket; nobody waits).
#include "lvspec_internal.h"
#include "sm100_ptx.cuh"

namespace lvspec {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = LVSPEC_MAX_REQUESTS / kThreads;      // requests of a thread
constexpr int kSlots = 4;                                 // consecutive slots of a thread: one 16-byte store

// Index of the last entry of the ascending list a[0..n) that is <= x (a[0] <= x).
__device__ __forceinline__ int last_not_above(const int32_t *a, int n, int x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Exclusive prefix sum over the CTA of one value per thread; `total` of all.
__device__ __forceinline__ long long block_exclusive(long long x, long long *warp_sums, long long &total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long in = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, in, o);
        if (lane >= o) in += y;
    }
    if (lane == 31) warp_sums[warp] = in;
    __syncthreads();
    long long before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) before += warp_sums[w];
        total += warp_sums[w];
    }
    __syncthreads();
    return before + in - x;
}

__global__ void __launch_bounds__(kThreads) page_plan_kernel(const PagePlanParams p)
{
    __shared__ int32_t start_s[LVSPEC_MAX_REQUESTS + 1];  // first new token of each request, in the slot map
    __shared__ int32_t upto_s[LVSPEC_MAX_REQUESTS + 1];   // pages taken by the requests before each
    __shared__ int32_t len_s[LVSPEC_MAX_REQUESTS];        // positions held; -1: the request is refused
    __shared__ int32_t held_s[LVSPEC_MAX_REQUESTS];
    __shared__ long long warp_sums[kThreads / 32];
    __shared__ int s_last, s_taken, s_refused;
    const int tid = threadIdx.x;

    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    int len[kPer], add[kPer], held[kPer];
    const int n_free = min(max(*p.n_free, 0), p.n_pages);
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int b = tid * kPer + u;
        len[u] = add[u] = held[u] = 0;
        if (b < p.batch) {
            len[u] = p.kv_len[b];
            add[u] = p.n_new[b];
            held[u] = p.pages_held[b];
        }
    }
    if (tid == 0) {
        s_taken = 0;
        s_refused = 0;
    }
    __syncthreads();
    // sums in 64 bits: a request may ask for anything
    long long mine = 0, first, total;
#pragma unroll
    for (int u = 0; u < kPer; ++u) mine += max(add[u], 0);
    first = block_exclusive(mine, warp_sums, total);
    bool fits[kPer];
    int need[kPer];
    const long long capacity = (long long)p.pages_per_seq * p.page_size;
    long long at = first;
    mine = 0;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int b = tid * kPer + u;
        if (b < p.batch) start_s[b] = (int32_t)min(at, 0x7fffffffll);
        at += max(add[u], 0);
        const long long end = (long long)len[u] + add[u];
        fits[u] = b < p.batch && len[u] >= 0 && add[u] >= 0 && held[u] >= 0 && held[u] <= p.pages_per_seq &&
                  end <= capacity && at <= p.max_new;
        need[u] = fits[u] ? max(0, (int)((end + p.page_size - 1) / p.page_size) - held[u]) : 0;
        mine += need[u];
    }
    if (tid == 0) start_s[p.batch] = (int32_t)min(total, 0x7fffffffll);
    const long long n_tokens = total;
    long long upto = block_exclusive(mine, warp_sums, total);
    // all inputs of this CTA have been read (the sums are made of them): the last CTA to say so may overwrite them
    if (tid == 0) {
        s_last = 1;
        if (gridDim.x > 1) {
            __threadfence();
            s_last = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
            __threadfence();
        }
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int b = tid * kPer + u;
        if (b >= p.batch) continue;
        upto_s[b] = (int32_t)min(upto, (long long)n_free);
        upto += need[u];
        // (sums never fall: from the first request on that finds too few pages, none that needs one gets any)
        if (need[u] > 0 && upto > n_free) fits[u] = false;
        if (fits[u] && need[u] > 0) atomicMax(&s_taken, (int)upto);
        if (!fits[u]) s_refused = 1;
        len_s[b] = fits[u] ? len[u] : -1;
        held_s[b] = held[u];
    }
    __syncthreads();
    const int taken = s_taken;
    if (tid == 0) {
        upto_s[p.batch] = taken;
        if (blockIdx.x == 0 && s_refused) atomicOr(p.status, LVSPEC_DEV_REFUSED);
    }

    // new entries of the block table: the n-th page taken belongs to the request it falls to
    for (int n = blockIdx.x * kThreads + tid; n < taken; n += gridDim.x * kThreads) {
        const int b = last_not_above(upto_s, p.batch, n);
        p.block_table[(size_t)b * p.pages_per_seq + held_s[b] + n - upto_s[b]] = p.free_pages[n_free - 1 - n];
    }
    // slots
    for (long long i0 = ((long long)blockIdx.x * kThreads + tid) * kSlots; i0 < p.max_new;
         i0 += (long long)gridDim.x * kThreads * kSlots) {
        int slot[kSlots];
        int r = i0 < n_tokens ? last_not_above(start_s, p.batch, (int)i0) : p.batch;
#pragma unroll
        for (int u = 0; u < kSlots; ++u) {
            const int i = (int)i0 + u;
            while (r < p.batch && i >= start_s[r + 1]) ++r;
            slot[u] = -1;
            if (r < p.batch && len_s[r] >= 0) {
                const int pos = len_s[r] + i - start_s[r], lp = pos / p.page_size;
                const int page = lp < held_s[r] ? p.block_table[(size_t)r * p.pages_per_seq + lp]
                                                : p.free_pages[n_free - 1 - (upto_s[r] + lp - held_s[r])];
                if ((unsigned)page < (unsigned)p.n_pages) slot[u] = page * p.page_size + (pos - lp * p.page_size);
            }
        }
        if (i0 + kSlots <= p.max_new)
            *reinterpret_cast<int4 *>(p.slot_map + i0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
        else
            for (int u = 0; i0 + u < p.max_new; ++u) p.slot_map[i0 + u] = slot[u];
    }
    if (!s_last) return;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int b = tid * kPer + u;
        if (b >= p.batch) continue;
        p.new_kv_len[b] = len[u] + (fits[u] ? add[u] : 0);
        p.new_pages_held[b] = held[u] + (fits[u] ? need[u] : 0);
        p.token_start[b] = start_s[b];
    }
    if (tid == 0) {
        p.token_start[p.batch] = start_s[p.batch];
        *p.new_n_free = n_free - taken;
        *p.ticket = 0;
    }
}

}  // namespace

cudaError_t launch_page_plan(const PagePlanParams &p, int n_sm, bool pdl, cudaStream_t stream, int *launches)
{
    // one CTA does for a decoding step; a prompt's slots are spread over two CTAs per SM at most
    long long grid = ((long long)p.max_new + kThreads * kSlots - 1) / (kThreads * kSlots);
    if (grid < 1) grid = 1;
    if (grid > 2 * n_sm) grid = 2 * n_sm;
    return launch_after(page_plan_kernel, dim3((unsigned)grid), kThreads, 0, pdl, stream, launches, p);
}

}  // namespace lvspec
