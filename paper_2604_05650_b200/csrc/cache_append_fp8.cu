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
// 2 bytes read and 1 written per element.  The rows of a block sit next to each
// other in the slot map, so the map itself says where blocks begin: a CTA takes a window of 64 tokens of
// K or V and the blocks that begin in it, for one head or several.  A prompt's window has one or two, a decoding step's eight (the
// draft tokens of as many requests): the CTA's eight warps form that many teams, which work side by side (one after the other, a
// step's blocks took 22 us instead of 6).  A thread keeps four 16-byte loads in flight, and the rows it loaded
// stay in its registers between the maximum and the codes; rows beyond those (a block of 128 shared by few warps)
// are read once more, from L2.
//
// 21600 tokens of seven prompts, 8 heads of 128, blocks of 32: 35 us for 133 MB, 3.8 TB/s.  Two thirds of the issue slots are taken
// (100 instructions for eight elements, a third of them the block's maximum and its exchange); the rest goes to the loads' latency, for
// which a head's exchange between its warps holds up the next head's.  The next
// head's rows asked for ahead, with 24 warps an SM instead of 32: 37 us.  Two, three, four, eight CTAs for the eight heads: 41,
// 35, 36, 39 us.
#include <cuda_fp16.h>

#include "lvspec_internal.h"
#include "sm100_ptx.cuh"

namespace lvspec {
namespace {

using namespace ptx;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kWindow = 64;

// Largest magnitudes among the even and among the odd of 8 bf16 values, as bits (they order as the values do).
__device__ __forceinline__ uint32_t max2(uint4 x)
{
    return __vmaxu2(__vmaxu2(x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu), __vmaxu2(x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu));
}
// The largest finite one among all
__device__ __forceinline__ uint32_t finite_max(uint4 x)
{
    const uint32_t w[4] = {x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu, x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu};
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t lo = w[k] & 0xFFFFu, hi = w[k] >> 16;
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

__device__ __forceinline__ float2 decode2(uint32_t two)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

template <int D>
__global__ void __launch_bounds__(kThreads, 4) append_fp8_kernel(const AppendFp8Params p)
{
    constexpr int kLanes = D / 8;                   // lanes of a row: 8 channels each
    constexpr int kWarpRows = 32 / kLanes;          // rows of a warp's step
    constexpr int kSteps = 4;                       // steps that stay in registers
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool is_v = blockIdx.z != 0;
    const uint16_t *all_src = is_v ? p.v : p.k;
    const long long stride = is_v ? p.v_stride : p.k_stride;
    uint8_t *all_pool = is_v ? p.v_pool : p.k_pool;
    float *scales = is_v ? p.v_scale : p.k_scale;
    const long long n_slots = (long long)p.n_pages * p.page_size;
    const int w0 = blockIdx.x * kWindow;
    const int in_block = (1 << p.block_log2) - 1;

    __shared__ uint32_t s_starts[kWindow / 32], s_breaks[kWindow / 32];
    __shared__ uint32_t s_max[2][kWarps];

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
        const bool other = mine != block_of(w0 + tid - 1);
        const uint32_t breaks = __ballot_sync(0xffffffffu, other), starts = __ballot_sync(0xffffffffu, other && mine >= 0);
        if (lane == 0) {
            s_breaks[tid >> 5] = breaks;
            s_starts[tid >> 5] = starts;
        }
    }
    __syncthreads();
    uint64_t left = s_starts[0] | ((uint64_t)s_starts[1] << 32);
    const uint64_t breaks = s_breaks[0] | ((uint64_t)s_breaks[1] << 32);
    // teams of 8, 4, 2 or 1 warps; team t takes the blocks t, t + teams, ...
    const int n_blocks = __popcll(left);
    const int team_log2 = n_blocks <= 1 ? 3 : n_blocks <= 2 ? 2 : n_blocks <= 4 ? 1 : 0;
    const int team = warp >> team_log2, teams = kWarps >> team_log2;
    const int row = ((warp & ((1 << team_log2) - 1)) * 32 + lane) / kLanes, chunk = lane % kLanes;
    const int rows_step = kWarpRows << team_log2;

    int turn = 0;                                   // of the two sets of words that the teams exchange
    for (int nth = 0; left; left &= left - 1, ++nth) {
        if (nth % teams != team) continue;
        const int at = __ffsll((long long)left) - 1, first = w0 + at;
        const int block = block_of(first);
        // the run of tokens of this block: up to the next break, which may lie behind the window
        const uint64_t later = at < 63 ? breaks >> (at + 1) : 0;
        int end = first + __ffsll((long long)later);
        if (!later) {
            uint32_t other = 0;
            for (end = w0 + kWindow; other == 0; end += 32) other = __ballot_sync(0xffffffffu, block_of(end + lane) != block);
            end += __ffs(other) - 33;
        }
        const int n = end - first;
        const int slot0 = block << p.block_log2;
        const int page = slot0 / p.page_size, pos0 = slot0 - page * p.page_size;          // the block's page, and first position in it
        // where this thread's rows go, and the first of the block's positions among all
        auto offset = [&](int i) { return p.slot_map[first + i] & in_block; };
        long long to[kSteps];
        int begun = in_block + 1;
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int i = u * rows_step + row;
            to[u] = 0;
            if (i < n) {
                const int o = offset(i);
                begun = min(begun, o);
                to[u] = (pos0 + o) * p.position_stride;
            }
        }
        for (int i = kSteps * rows_step + row; i < n; i += rows_step) begun = min(begun, offset(i));
        begun = __reduce_min_sync(0xffffffffu, (uint32_t)begun);
        const uint16_t *src0 = all_src + (first + row) * stride + chunk * 8;
        const long long step = rows_step * stride;
        uint8_t *dst0 = all_pool + page * p.page_stride + chunk * 8;
        float *scale0 = scales + (size_t)page * p.n_heads * (p.page_size >> p.block_log2) + (pos0 >> p.block_log2);

        for (int head = blockIdx.y; head < p.n_heads; head += gridDim.y, turn ^= 1) {
            const uint16_t *src = src0 + head * D;
            uint8_t *dst = dst0 + head * p.head_stride;
            float *scale = scale0 + head * (p.page_size >> p.block_log2);
            const float old = *scale;
            uint4 x[kSteps];
            uint32_t two = 0;
#pragma unroll
            for (int u = 0; u < kSteps; ++u) {
                x[u] = make_uint4(0, 0, 0, 0);
                if (u * rows_step + row < n) x[u] = *reinterpret_cast<const uint4 *>(src + u * step);
            }
#pragma unroll
            for (int u = 0; u < kSteps; ++u) two = __vmaxu2(two, max2(x[u]));
            for (int i = kSteps * rows_step + row; i < n; i += rows_step)
                two = __vmaxu2(two, max2(*reinterpret_cast<const uint4 *>(src + (i - row) * stride)));
            uint32_t most = max(two & 0xFFFFu, two >> 16);
            if (__builtin_expect(most >= 0x7F80u, 0)) {         // an infinity or a NaN among them
                most = 0;
#pragma unroll 1
                for (int i = row; i < n; i += rows_step)
                    most = max(most, finite_max(*reinterpret_cast<const uint4 *>(src + (i - row) * stride)));
            }
            most = __reduce_max_sync(0xffffffffu, most);
            if (team_log2 > 0) {
                // maximum and first position in one word: neither takes more than 16 bits
                uint32_t *words = s_max[turn] + (team << team_log2);
                if (lane == 0) words[warp & ((1 << team_log2) - 1)] = (most << 16) | (uint32_t)(in_block + 1 - begun);
                asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(32 << team_log2) : "memory");
                const uint32_t m = words[lane & ((1 << team_log2) - 1)];
                most = __reduce_max_sync(0xffffffffu, m >> 16);
                begun = in_block + 1 - (int)__reduce_max_sync(0xffffffffu, m & 0xFFFFu);
            }
            float now = scale_of(most);
            const float had = begun > 0 ? old : 0.f;
            if (begun > 0) now = fmaxf(now, had);
            // x / scale is x times a power of two, unless the caller's cache came with another scale
            const uint32_t e = (__float_as_uint(now) >> 23) & 0xFFu;
            const bool exact = (__float_as_uint(now) & 0x7FFFFFu) == 0 && e > 0 && e < 254;
            const float inv = __uint_as_float((254u - e) << 23);
            const uint64_t inv2 = pack_f32x2(__float_as_uint(inv), __float_as_uint(inv));
            auto put = [&](long long to, uint4 v) {
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
                uint32_t c[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float a, b;
                    unpack_f32x2(mul_f32x2(pack_f32x2(w[k] << 16, w[k] & 0xFFFF0000u), inv2), a, b);
                    c[k] = pack_e4m3x2(a, b);
                }
                *reinterpret_cast<uint2 *>(dst + to) = make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
            };
            if (__builtin_expect(exact, 1)) {
#pragma unroll
                for (int u = 0; u < kSteps; ++u)
                    if (u * rows_step + row < n) put(to[u], x[u]);
                for (int i = kSteps * rows_step + row; i < n; i += rows_step)
                    put((pos0 + offset(i)) * p.position_stride, *reinterpret_cast<const uint4 *>(src + (i - row) * stride));
            } else {
#pragma unroll 1
                for (int i = row; i < n; i += rows_step)
#pragma unroll 1
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t w = reinterpret_cast<const uint32_t *>(src + (i - row) * stride)[k];
                        *reinterpret_cast<uint16_t *>(dst + (pos0 + offset(i)) * p.position_stride + 2 * k) =
                            (uint16_t)pack_e4m3x2(__fdiv_rn(__uint_as_float(w << 16), now), __fdiv_rn(__uint_as_float(w & 0xFFFF0000u), now));
                    }
            }
            // older rows of a block whose scale grows
            if (begun > 0 && had != now) {
                const float ratio = __fdiv_rn(had, now);
                for (int i = row; i < begun; i += rows_step) {
                    uint2 *to = reinterpret_cast<uint2 *>(dst + (pos0 + i) * p.position_stride);
                    const uint2 c = *to;
                    const float2 a = decode2(c.x), b = decode2(c.x >> 16), d = decode2(c.y), e = decode2(c.y >> 16);
                    *to = make_uint2(codes4(a.x * ratio, a.y * ratio, b.x * ratio, b.y * ratio),
                                     codes4(d.x * ratio, d.y * ratio, e.x * ratio, e.y * ratio));
                }
            }
            if (row == 0 && chunk == 0) *scale = now;
        }
    }
}

}  // namespace

cudaError_t launch_append_fp8(const AppendFp8Params &p, int head_dim, int n_sm, bool pdl, cudaStream_t stream, int *launches)
{
    // a CTA for each head where tokens are few; a prompt's windows fill the device with CTAs that go through several heads (what
    // they find out about the slots then counts for all)
    const int windows = (p.n_tokens + kWindow - 1) / kWindow;
    int heads = (10 * n_sm + 2 * windows - 1) / (2 * windows);
    if (heads > p.n_heads) heads = p.n_heads;
    const dim3 grid((unsigned)windows, (unsigned)heads, 2);
    return head_dim == 128 ? launch_after(append_fp8_kernel<128>, grid, kThreads, 0, pdl, stream, launches, p)
                           : launch_after(append_fp8_kernel<64>, grid, kThreads, 0, pdl, stream, launches, p);
}

}  // namespace lvspec
