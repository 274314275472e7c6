// New K and V rows into a paged E4M3 cache with one scale per block of positions and head.
//
// For the new rows of one block of positions and one head, a = the largest finite |x| among them:
//   s    = 2^ceil(log2(a / 448))          the smallest power of two with a / s <= 448
//   s    = max(s, the block's scale)      if the block has rows before the new ones; their codes
//                                         become rn(decode(code) * old / s) when s is the larger
//   code = rn_e4m3(x / s)
// A power of two loses nothing in a floating-point format (in E4M3's normal range), x / s is exact, and
// a block that is begun in one step and ends in a later one is brought to a larger scale without
// a second rounding of its normal values.
//
// Bound by memory: 2 bytes read and 1 written per element.  The rows of a block sit next to each
// other in the slot map, so the map itself says where blocks begin: a CTA takes a window of 64 tokens of
// one head of K or V and works through the blocks that begin in it, 16 rows (32 at head_dim 64) a step with
// 16-byte loads; up to 128 rows, the longest block, stay in registers between the maximum and
// the codes, so every element is read once.
#include <cuda_fp16.h>

#include "lvspec_internal.h"
#include "sm100_ptx.cuh"

namespace lvspec {
namespace {

using namespace ptx;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kWindow = 64;

// Largest finite magnitude among 8 bf16 values, as bits (they order as the values do).
__device__ __forceinline__ uint32_t finite_max(uint4 x)
{
    uint32_t m = 0;
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t lo = w[k] & 0x7FFFu, hi = (w[k] >> 16) & 0x7FFFu;
        if (lo < 0x7F80u) m = max(m, lo);
        if (hi < 0x7F80u) m = max(m, hi);
    }
    return m;
}

// 2^ceil(log2(a / 448)) for a bf16 magnitude, within 2^-100 .. 2^119
__device__ __forceinline__ float scale_of(uint32_t bf16_bits)
{
    const uint32_t f = bf16_bits << 16;
    int k = (int)(f >> 23) - 127 - 8 + ((f & 0x7FFFFFu) > 0x600000u ? 1 : 0);     // 448 = 1.75 * 2^8
    k = max(-100, min(119, k));
    return __uint_as_float((uint32_t)(127 + k) << 23);
}

__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d)
{
    return pack_e4m3x2(a, b) | (pack_e4m3x2(c, d) << 16);
}

// x / s: s is a power of two unless the caller's cache came with another scale
struct Divide {
    float s, inv;
    bool exact;
    __device__ __forceinline__ Divide(float s_) : s(s_), inv(1.0f / s_)
    {
        const uint32_t e = (__float_as_uint(s_) >> 23) & 0xFFu;
        exact = (__float_as_uint(s_) & 0x7FFFFFu) == 0 && e > 0 && e < 254;
    }
    __device__ __forceinline__ float operator()(float x) const { return exact ? x * inv : __fdiv_rn(x, s); }
};

__device__ __forceinline__ float2 decode2(uint32_t two)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

template <int D>
__global__ void __launch_bounds__(kThreads) append_fp8_kernel(const AppendFp8Params p)
{
    constexpr int kLanes = D / 8;                   // lanes of a row: 8 channels each
    constexpr int kRows = kThreads / kLanes;        // rows of a step
    constexpr int kSteps = 128 / kRows;             // steps that stay in registers
    const int tid = threadIdx.x;
    const int head = blockIdx.y;
    const bool is_v = blockIdx.z != 0;
    const uint16_t *src = (is_v ? p.v : p.k) + head * D;
    const long long stride = is_v ? p.v_stride : p.k_stride;
    uint8_t *pool = (is_v ? p.v_pool : p.k_pool) + head * p.head_stride;
    float *scales = is_v ? p.v_scale : p.k_scale;
    const long long n_slots = (long long)p.n_pages * p.page_size;
    const int w0 = blockIdx.x * kWindow;

    __shared__ uint32_t s_starts[kWindow / 32];
    __shared__ int s_end, s_begun;
    __shared__ uint32_t s_max[kWarps];

    grid_launch_dependents();
    grid_dependency_wait();
    // the block of positions of a token, over all pages; -1: the token has no slot
    auto block_of = [&](int i) {
        if (i < 0 || i >= p.n_tokens) return -1;
        const int s = p.slot_map[i];
        return s < 0 || s >= n_slots ? -1 : s >> p.block_log2;
    };
    if (tid < kWindow) {
        const int mine = block_of(w0 + tid);
        const uint32_t starts = __ballot_sync(0xffffffffu, mine >= 0 && mine != block_of(w0 + tid - 1));
        if ((tid & 31) == 0) s_starts[tid >> 5] = starts;
    }
    __syncthreads();
    const uint64_t starts = s_starts[0] | ((uint64_t)s_starts[1] << 32);
    const int row = tid / kLanes, chunk = tid % kLanes;

    for (uint64_t left = starts; left; left &= left - 1) {
        const int first = w0 + __ffsll((long long)left) - 1;
        const int block = block_of(first);
        __syncthreads();
        if (tid == 0) {
            s_end = 0x7fffffff;
            s_begun = 1 << p.block_log2;
        }
        __syncthreads();
        // the run of tokens of this block, and the first of the block's positions among them
        int end, base = first;
        do {
            const int i = base + tid;
            if (block_of(i) != block) atomicMin(&s_end, i);
            __syncthreads();
            end = s_end;
            if (i < end) atomicMin(&s_begun, p.slot_map[i] & ((1 << p.block_log2) - 1));
            __syncthreads();
            base += kThreads;
        } while (end == 0x7fffffff);
        const int begun = s_begun, n = end - first;
        const int pos0 = (block << p.block_log2) % p.page_size;                   // the block's first position in its page
        const int page = (int)(((long long)block << p.block_log2) / p.page_size);
        float *scale = scales + ((size_t)page * p.n_heads + head) * (p.page_size >> p.block_log2) + (pos0 >> p.block_log2);
        const float had = begun > 0 ? *scale : 0.f;

        uint4 x[kSteps];
        uint32_t most = 0;
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int i = u * kRows + row;
            x[u] = make_uint4(0, 0, 0, 0);
            if (i < n) x[u] = *reinterpret_cast<const uint4 *>(src + (first + i) * stride + chunk * 8);
        }
#pragma unroll
        for (int u = 0; u < kSteps; ++u) most = max(most, finite_max(x[u]));
        // (more rows than a block has positions: some slot is given twice)
        for (int i = kSteps * kRows + row; i < n; i += kRows)
            most = max(most, finite_max(*reinterpret_cast<const uint4 *>(src + (first + i) * stride + chunk * 8)));
        most = __reduce_max_sync(0xffffffffu, most);
        if ((tid & 31) == 0) s_max[tid >> 5] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWarps; ++w) most = max(most, s_max[w]);
        float now = scale_of(most);
        if (begun > 0) now = fmaxf(now, had);
        const Divide by(now);

        uint8_t *rows = pool + page * p.page_stride;
        auto put = [&](int i, uint4 v) {
            const int pos = pos0 + (p.slot_map[first + i] & ((1 << p.block_log2) - 1));
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            float f[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                f[2 * k] = by(__uint_as_float(w[k] << 16));
                f[2 * k + 1] = by(__uint_as_float(w[k] & 0xFFFF0000u));
            }
            *reinterpret_cast<uint2 *>(rows + pos * p.position_stride + chunk * 8) =
                make_uint2(codes4(f[0], f[1], f[2], f[3]), codes4(f[4], f[5], f[6], f[7]));
        };
#pragma unroll
        for (int u = 0; u < kSteps; ++u)
            if (u * kRows + row < n) put(u * kRows + row, x[u]);
        for (int i = kSteps * kRows + row; i < n; i += kRows)
            put(i, *reinterpret_cast<const uint4 *>(src + (first + i) * stride + chunk * 8));
        // older rows of a block whose scale grows
        if (begun > 0 && had != now) {
            const float ratio = __fdiv_rn(had, now);
            for (int i = row; i < begun; i += kRows) {
                uint2 *at = reinterpret_cast<uint2 *>(rows + (pos0 + i) * p.position_stride + chunk * 8);
                const uint2 c = *at;
                const float2 a = decode2(c.x), b = decode2(c.x >> 16), d = decode2(c.y), e = decode2(c.y >> 16);
                *at = make_uint2(codes4(a.x * ratio, a.y * ratio, b.x * ratio, b.y * ratio),
                                 codes4(d.x * ratio, d.y * ratio, e.x * ratio, e.y * ratio));
            }
        }
        if (tid == 0) *scale = now;
    }
}

}  // namespace

cudaError_t launch_append_fp8(const AppendFp8Params &p, int head_dim, bool pdl, cudaStream_t stream, int *launches)
{
    const dim3 grid((unsigned)((p.n_tokens + kWindow - 1) / kWindow), (unsigned)p.n_heads, 2);
    return head_dim == 128 ? launch_after(append_fp8_kernel<128>, grid, kThreads, 0, pdl, stream, launches, p)
                           : launch_after(append_fp8_kernel<64>, grid, kThreads, 0, pdl, stream, launches, p);
}

}  // namespace lvspec
