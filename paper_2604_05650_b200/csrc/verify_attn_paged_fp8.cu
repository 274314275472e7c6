// Verification attention on a paged E4M3 cache with a scale for each block of positions and head:
// TMA + tcgen05 kernel (head_dim 128 or 64), lengths and spans on the device.
//
//   k_j = ks[block of j] * decode(kc_j),  v_j likewise
//   s_j = <q, k_j> / sqrt(D) for the positions the query sees, p = softmax(s)
//   out = sum_j p_j v_j,   mass = sum of p_j over the visual span
//
// As in the kernel for the other caches the few query rows of a KV head are the small side, so the products
// are taken transposed, 128 cache positions a tile:
//   S^T[pos, n] = K codes . Q^T         kind::f8f6f4, the codes as they are; q split into two E4M3 terms
//                                       (leading four significant bits and the next four: exact for bf16)
//   O^T[ch, n] += V codes^T . P^T       kind::f16
// Every TMEM lane of S^T is one position, so a block's scale is one number per thread: the K scale goes
// into the factor that the scores are multiplied with anyway, the V scale onto the probability.
// A probability that carries a scale can neither be kept in 8 bits (E4M3 spans 17 binades; a sink position
// that holds most of a row's mass would push all others out) nor be summed by the tensor core for the
// denominator.  So P^T is fp16, the sums l and the visual sums are taken in fp32 by the softmax threads
// (each adds up its own position's column values over the tiles; the 128 lanes are summed when the stream
// enters or leaves the visual span, and at its end), and V is brought to fp16 (exact) on its way:
// four warps read the 8-bit tile transposed (ldmatrix b8), convert and store it to tensor memory, from
// where the product takes its A operand.  That keeps the 32 KB of fp16 out of shared memory, whose bandwidth is
// the next bound after HBM: per tile 16 + 32 KB for K (written, read for either term of q), 16 + 16 for V.
//
// The reference exponent of a row is the score of its segment's first position, 2^3 below it; it moves
// (a tile's maximum over the lanes, accumulators rescaled) when a score passes 2^14.  fp16 then holds a
// probability with eleven bits down to 2^17 below the first position's, and down to 2^27 with fewer.  V scales are
// taken relative to 2^(k0): four times the power of two below the segment's first one, moved with the reference.
//
// Work is laid out on the device, from the lengths: the tiles of all (sequence, KV head) pairs in a row are cut into
// equal shares, one per SM, either at multiples of the share within each pair (no CTA has two pairs) or straight
// through (a CTA may end one pair and begin the next).  A captured launch so follows lengths that change, and a batch of
// different lengths keeps all SMs busy.  Partials of pairs that several CTAs share are merged by a second, small
// kernel; a pair that one CTA has to itself is finished there.
#include <cuda.h>
#include <cuda_bf16.h>

#include <type_traits>

#include "lvspec_internal.h"
#include "sm100_ptx.cuh"

namespace lvspec {
namespace {

using namespace ptx;

constexpr int kTilePos = 128;
constexpr int kGroups = 2;                  // softmax groups of four warps, each on its share of the columns
constexpr int kConvertWarp0 = 4, kSoftmaxWarp0 = 8;
constexpr int kSoftmaxThreads = 128 * kGroups;
constexpr int kThreads = 32 * kSoftmaxWarp0 + kSoftmaxThreads;
constexpr int kMergeWarps = 8;
constexpr int kBufs = 2;                    // S^T, P^T and V^T buffers each
constexpr float kFirst = 3.f;               // log2 of the probability of a segment's first position
constexpr float kGuard = 14.f;              // log2 units above the reference before it moves
constexpr int kFlatGain = 3;                // tiles a straight cut has to save to be taken

// ---- work ---------------------------------------------------------------------------
// Tiles of all (sequence, head) pairs one after the other; CTA c has the tiles [c * share, (c + 1) * share) of
// that line.  With `aligned` every pair is padded to a multiple of the share.
struct Line {
    int32_t start[LVSPEC_MAX_BATCH + 1];    // of each sequence's first pair
    int32_t len[LVSPEC_MAX_BATCH];          // positions; 0 for a sequence without any
    int32_t share, aligned;
};

__device__ __forceinline__ int tiles_of(int len) { return (len + kTilePos - 1) / kTilePos; }
__device__ __forceinline__ int padded(const Line &w, int tiles)
{
    return w.aligned ? (tiles + w.share - 1) / w.share * w.share : tiles;
}

// One warp.  True when a length lies outside 0..max_len (the sequence then counts as empty).
__device__ __forceinline__ bool make_line(Line &w, const PagedFp8Params &p)
{
    constexpr int kPer = LVSPEC_MAX_BATCH / 32;
    const int lane = threadIdx.x & 31;
    int tiles[kPer], total = 0, longest = 0;
    bool bad = false;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int b = u * 32 + lane;
        int len = b < p.B ? p.kv_len[b] : 0;
        if (len < 0 || len > p.max_len) {
            bad = true;
            len = 0;
        }
        if (b < p.B) w.len[b] = len;
        tiles[u] = tiles_of(len);
        total += tiles[u];
        longest = max(longest, tiles[u]);
    }
    total = __reduce_add_sync(0xffffffffu, total) * p.Hkv;
    longest = __reduce_max_sync(0xffffffffu, longest);
    const int flat = max(1, (total + p.n_cta - 1) / p.n_cta);
    int share = flat, aligned = 0;
    // cutting within pairs is taken if it costs a few tiles at most: a second pair in a CTA costs as much
    for (int t = flat; t <= flat + kFlatGain && !aligned; ++t) {
        int ctas = 0;
#pragma unroll
        for (int u = 0; u < kPer; ++u)
            if (u * 32 < p.B) ctas += (tiles[u] + t - 1) / t;
        if (__reduce_add_sync(0xffffffffu, ctas) * p.Hkv <= p.n_cta) {
            share = t;
            aligned = 1;
        }
    }
    int before = 0;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        if (u * 32 >= p.B) break;
        int mine = (aligned ? (tiles[u] + share - 1) / share * share : tiles[u]) * p.Hkv, in = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, in, o);
            if (lane >= o) in += y;
        }
        if (u * 32 + lane < p.B) w.start[u * 32 + lane] = before + in - mine;
        before += __shfl_sync(0xffffffffu, in, 31);
    }
    if (lane == 0) {
        w.start[p.B] = before;
        w.share = share;
        w.aligned = aligned;
    }
    return __any_sync(0xffffffffu, bad);
}

// The pieces of a CTA's share: tiles [t0, t0 + T) of one pair each.
struct Segment {
    int b, head, t0, T, tiles, len;
    bool first, last;                       // begins / ends its pair
};
struct Walk {
    const Line &w;
    const int n_seq;
    int at, end, b;
    __device__ __forceinline__ Walk(const Line &w_, int n_seq_, int cta) : w(w_), n_seq(n_seq_), b(0)
    {
        at = cta * w.share;
        end = min(at + w.share, w.start[n_seq]);
        int hi = n_seq;
        while (hi - b > 1) {
            const int mid = (b + hi) >> 1;
            if (w.start[mid] <= at) b = mid;
            else hi = mid;
        }
    }
    __device__ __forceinline__ bool next(Segment &s)
    {
        if (at >= end) return false;
        while (at >= w.start[b + 1]) ++b;
        s.b = b;
        s.len = w.len[b];
        s.tiles = tiles_of(s.len);
        const int each = padded(w, s.tiles), off = at - w.start[b];
        s.head = off / each;
        s.t0 = off - s.head * each;
        const int stop = min(end, w.start[b] + (s.head + 1) * each);
        s.T = min(s.tiles - s.t0, stop - at);
        s.first = s.t0 == 0;
        s.last = s.t0 + s.T == s.tiles;
        at = stop;
        return true;
    }
};
// Partial results of a CTA: of the pair it goes on with, and of the pair it begins and does not end.
__device__ __forceinline__ int part_slot(int cta, bool first) { return 2 * cta + (first ? 1 : 0); }

// ---- shared memory --------------------------------------------------------------------
struct Smem {
    uint32_t k, v, q, p, m, tmx, sums, bars, misc, line, total;
    int ks, vs;                             // K and V slots
};
constexpr int kBarsFixed = 6 * kBufs + 3;
Smem smem_map(int D, int NP, int ks, int vs)
{
    Smem s;
    uint32_t o = 0;
    s.ks = ks;
    s.vs = vs;
    s.k = o;    o += ks * kTilePos * D;
    s.v = o;    o += vs * kTilePos * D;
    s.q = o;    o += 2 * NP * D;
    s.p = o;    o += kBufs * NP * 256;
    s.m = o;    o += NP * 4;
    s.tmx = o;  o += 4 * NP * 4;
    s.sums = o; o += 2 * 4 * NP * 4;
    s.bars = o; o += 8 * (2 * ks + 2 * vs + kBarsFixed);
    s.misc = o; o += 64;                    // TMEM address, abort flag, per-warp maxima
    s.line = o; o += (sizeof(Line) + 15) & ~15u;
    s.total = o;
    return s;
}

struct KernelParams {
    PagedFp8Params a;
    Smem sm;
    int NP, tmem_cols;
    uint32_t group_magic;
};

struct Ring {
    int idx = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next(int n)
    {
        if (++idx == n) {
            idx = 0;
            parity ^= 1u;
        }
    }
};

__device__ __forceinline__ bool wait_unconditional(uint32_t bar, uint32_t parity)
{
    // used while tearing down: time-bounded, ignores the abort flag
    const uint64_t t0 = global_timer_ns();
    while (!mbar_try_wait(bar, parity))
        if (global_timer_ns() - t0 > 1000000000ull) return false;
    return true;
}
__device__ __forceinline__ void named_sync(int id, int threads)
{
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
__device__ __forceinline__ bool group_any(int id, bool pred)
{
    uint32_t out;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 q, %2, 0;\n\t"
        "bar.red.or.pred p, %1, 128, q;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(out) : "r"(id), "r"((uint32_t)pred) : "memory");
    return out != 0;
}

// The columns (query rows g * G + hg) that see a position with tail index t = pos - (len - gamma):
// a range [lo, lo + n), as in draft_query_sees.
struct Seen {
    int lo;
    uint32_t n;
    __device__ __forceinline__ bool operator()(int col) const { return (uint32_t)(col - lo) < n; }
};
__device__ __forceinline__ Seen seen_by(int t, int G, int gamma, int branch_len)
{
    Seen s = {0, t < 0 ? 0xFFFFFFFFu : 0u};
    if (t >= 0 && t < gamma) {
        s.lo = t * G;
        s.n = (uint32_t)((t / branch_len + 1) * branch_len * G - s.lo);
    }
    return s;
}

// Where the positions of consecutive tiles sit: logical page and offset in it.  A page holds whole
// tiles, or a tile holds whole pages (16, 32 or 64 positions).
struct PageWalk {
    int page, off;
    __device__ __forceinline__ PageWalk(const PagedFp8Params &p, int tile, int row)
    {
        const int pos = tile * kTilePos + row;
        page = pos / p.page_size;
        off = pos - page * p.page_size;
    }
    __device__ __forceinline__ void next_tile(const PagedFp8Params &p)
    {
        if (p.page_size < kTilePos) page += kTilePos / p.page_size;
        else if ((off += kTilePos) >= p.page_size) {
            off -= p.page_size;
            ++page;
        }
    }
};

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// four E4M3 codes -> two packed fp16 pairs
__device__ __forceinline__ void decode4(uint32_t codes, uint32_t &lo, uint32_t &hi)
{
    asm("{\n\t.reg .b16 a, b;\n\t"
        "mov.b32 {a, b}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi) : "r"(codes));
}
// Two 16 x 16 blocks of bytes, transposed: lane t gets of row t / 4 (and t / 4 + 8) the four
// bytes 4 (t % 4) .. + 3, where a row of the result is a column of the block.
__device__ __forceinline__ void ldmatrix_b8_x2(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// 16 lanes x 64 columns: lane t's registers 4 i .. 4 i + 3 are row t / 4, columns 8 i + 2 (t % 4) and the next,
// then row t / 4 + 8.
__device__ __forceinline__ void tmem_st_16x256b_x8(uint32_t taddr, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.16x256b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem desc]
__device__ __forceinline__ void mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ constexpr uint32_t make_idesc_f16(uint32_t M, uint32_t N, uint32_t b_mn)
{
    return (1u << 4) | (b_mn << 16) | ((N >> 3) << 17) | ((M >> 4) << 24);     // fp32 accumulators; format code 0 = fp16
}
constexpr uint32_t kSwizzle64B = 4;

// Sum of each of eight values over the warp: lane t with t % 4 == 0 gets that of value t / 4 (bits 4, 3, 2
// of the lane, highest first).  Nine shuffles where eight plain sums take forty.
__device__ __forceinline__ float sum8(const float (&v)[8], int lane)
{
    float a[4], b[2], c;
    const bool h16 = lane & 16, h8 = lane & 8, h4 = lane & 4;
#pragma unroll
    for (int k = 0; k < 4; ++k) a[k] = (h16 ? v[k + 4] : v[k]) + __shfl_xor_sync(0xffffffffu, h16 ? v[k] : v[k + 4], 16);
#pragma unroll
    for (int k = 0; k < 2; ++k) b[k] = (h8 ? a[k + 2] : a[k]) + __shfl_xor_sync(0xffffffffu, h8 ? a[k] : a[k + 2], 8);
    c = (h4 ? b[1] : b[0]) + __shfl_xor_sync(0xffffffffu, h4 ? b[0] : b[1], 4);
    c += __shfl_xor_sync(0xffffffffu, c, 2);
    c += __shfl_xor_sync(0xffffffffu, c, 1);
    return c;
}

__device__ __forceinline__ int div_by(int x, int d, uint32_t m)
{
    if (m == 0u) return x;
    const int q = (int)__umulhi((uint32_t)x, m);
    return q * d > x ? q - 1 : q;
}

// kC: chunks of eight columns a softmax group has at most
template <int kC>
__global__ void __launch_bounds__(kThreads, 1)
attn_paged_fp8_kernel(const KernelParams P, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v)
{
    extern __shared__ uint8_t smem_raw[];
    const PagedFp8Params &p = P.a;
    const Smem &sm = P.sm;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int D = p.D, NP = P.NP, M = p.M, G = p.G, gamma = p.gamma;
    const int n8 = (M + 7) >> 3;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *gbase = smem_raw + (base - smem_u32(smem_raw));
    float *m_s = reinterpret_cast<float *>(gbase + sm.m);
    float *tmx_s = reinterpret_cast<float *>(gbase + sm.tmx);
    float *sums_s = reinterpret_cast<float *>(gbase + sm.sums);      // [outside, inside the span][warp of the group][NP]
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(gbase + sm.misc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(gbase + sm.misc + 4);
    volatile uint32_t *wmax_s = reinterpret_cast<volatile uint32_t *>(gbase + sm.misc + 16);
    Line &line = *reinterpret_cast<Line *>(gbase + sm.line);
    const uint32_t slot_bytes = kTilePos * D;

    const uint32_t bar0 = base + sm.bars;
    auto k_full = [&](int s) { return bar0 + 8 * s; };
    auto k_empty = [&](int s) { return bar0 + 8 * (sm.ks + s); };
    auto v_full = [&](int s) { return bar0 + 8 * (2 * sm.ks + s); };
    auto v_empty = [&](int s) { return bar0 + 8 * (2 * sm.ks + sm.vs + s); };
    const uint32_t bar1 = bar0 + 8 * (2 * sm.ks + 2 * sm.vs);
    auto s_full = [&](int s) { return bar1 + 8 * s; };
    auto s_free = [&](int s) { return bar1 + 8 * (kBufs + s); };
    auto p_full = [&](int s) { return bar1 + 8 * (2 * kBufs + s); };
    auto vt_full = [&](int s) { return bar1 + 8 * (3 * kBufs + s); };
    auto pv_done = [&](int s) { return bar1 + 8 * (4 * kBufs + s); };      // frees the P^T and the V^T buffer
    const uint32_t q_full = bar1 + 8 * 5 * kBufs, o_free = q_full + 8, drain_qk = q_full + 16, drain_pv = q_full + 24;

    if (warp == 3 && lane < 2) prefetch_tensormap(lane ? &tmap_v : &tmap_k);
    if (warp == 0) {
        const int n_bars = 2 * sm.ks + 2 * sm.vs + kBarsFixed;
        for (int i = lane; i < n_bars; i += 32) {
            const int j = i - 2 * (sm.ks + sm.vs);
            uint32_t count = 1;
            if (j < 0) count = i >= 2 * sm.ks + sm.vs ? D / 32 : 1;                 // v_empty: the converting warps
            else if (j >= kBufs && j < 3 * kBufs) count = 4 * kGroups;              // s_free, p_full
            else if (j >= 3 * kBufs && j < 4 * kBufs) count = D / 32;               // vt_full
            else if (j == 5 * kBufs || j == 5 * kBufs + 1) count = 4 * kGroups;     // q_full, o_free
            mbar_init(bar0 + 8 * i, count);
        }
        if (lane == 0) *abort_flag = 0;
        fence_proxy_async_smem();
        grid_dependency_wait();
        grid_launch_dependents();
        const bool bad = make_line(line, p);
        if (bad && blockIdx.x == 0 && lane == 0) atomicOr(p.status, LVSPEC_DEV_BAD_LENGTH);
    } else {
        if (warp == 1) {
            tmem_alloc(base + sm.misc, (uint32_t)P.tmem_cols);
            tmem_relinquish();
        }
        // columns beyond the last chunk stay zero (at most one chunk per P^T buffer)
        if (warp >= kSoftmaxWarp0 && n8 * 8 < NP) {
            const int i = tid - 32 * kSoftmaxWarp0;      // 0..255: buffer, position
            static_assert(kBufs * 128 == kSoftmaxThreads, "one 16-byte chunk a thread");
            *reinterpret_cast<uint4 *>(gbase + sm.p + (i >> 7) * (NP * 256) + n8 * 2048 + (i & 127) * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
        }
        grid_dependency_wait();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const uint32_t tm_v = tmem, tm_s = tmem + kBufs * 64, tm_o = tm_s + kBufs * NP;

    Walk walk(line, p.B, blockIdx.x);
    Segment seg;

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer
        const uint64_t policy = l2_evict_first_policy();
        Ring kr, vr;
        const int boxes = p.page_size < kTilePos ? kTilePos / p.page_size : 1;
        const uint32_t box_bytes = slot_bytes / boxes;
        int n = 0;                                     // tiles asked for
        bool ok = true;
        while (ok && walk.next(seg)) {
            const int32_t *row = p.block_table + (size_t)seg.b * p.pages_per_seq;
            const int n_live = (seg.len + p.page_size - 1) / p.page_size;
            // 32 entries of the block table at a time, the next 32 on their way
            auto entries = [&](int first) {
                int e = p.n_pages;                     // outside the pool: reads as zeros
                if (first + lane < n_live) e = row[first + lane];
                return (unsigned)e < (unsigned)p.n_pages ? e : p.n_pages;
            };
            PageWalk at(p, seg.t0, 0);
            int have = at.page & ~31, cur = entries(have), nxt = entries(have + 32);
            for (int j = 0; ok && j < seg.T; ++j, ++n) {
                if ((at.page & ~31) != have) {
                    have += 32;
                    cur = nxt;
                    nxt = entries(have + 32);
                }
                const int page = __shfl_sync(0xffffffffu, cur, (at.page + (lane < boxes ? lane : 0)) & 31);
                if (n >= sm.ks) ok = mbar_wait(k_empty(kr.idx), kr.parity ^ 1u, abort_flag);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                const uint32_t kd = base + sm.k + kr.idx * slot_bytes, vd = base + sm.v + vr.idx * slot_bytes;
                if (lane == 0) mbar_arrive_expect_tx(k_full(kr.idx), slot_bytes);
                __syncwarp();
                if (lane < boxes) tma_load_4d_hint(kd + lane * box_bytes, &tmap_k, k_full(kr.idx), 0, at.off, seg.head, page, policy);
                if (n >= sm.vs) ok = mbar_wait(v_empty(vr.idx), vr.parity ^ 1u, abort_flag);
                if (!__all_sync(0xffffffffu, ok)) {
                    ok = false;
                    kr.next(sm.ks);
                    break;
                }
                if (lane == 0) mbar_arrive_expect_tx(v_full(vr.idx), slot_bytes);
                __syncwarp();
                if (lane < boxes) tma_load_4d_hint(vd + lane * box_bytes, &tmap_v, v_full(vr.idx), 0, at.off, seg.head, page, policy);
                kr.next(sm.ks);
                vr.next(sm.vs);
                at.next_tile(p);
            }
        }
        if (*abort_flag) {
            // copies still in flight end (bounded) before the CTA leaves: the last round of either ring
            for (int j = 0; j < sm.ks; ++j) wait_unconditional(k_full(j), j < kr.idx ? kr.parity : kr.parity ^ 1u);
            for (int j = 0; j < sm.vs; ++j) wait_unconditional(v_full(j), j < vr.idx ? vr.parity : vr.parity ^ 1u);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ K.Q^T issuer
        const uint32_t idesc = make_idesc_e4m3(128, NP, 0, 0);
        const uint32_t swz = D == 128 ? kSwizzle128B : kSwizzle64B;
        const uint64_t kd0 = make_smem_desc(base + sm.k, 16, 8 * D, swz), qd0 = make_smem_desc(base + sm.q, 16, 8 * D, swz);
        const int steps = D / 32;
        Ring kr, sr, qr;
        int n = 0;
        bool ok = true;
        while (ok && walk.next(seg)) {
            ok = mbar_wait(q_full, qr.parity, abort_flag);
            qr.next(1);
            for (int j = 0; ok && j < seg.T; ++j, ++n) {
                ok = mbar_wait(k_full(kr.idx), kr.parity, abort_flag);
                if (n >= kBufs) ok = mbar_wait(s_free(sr.idx), sr.parity ^ 1u, abort_flag) && ok;
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t kd = kd0 + (uint64_t)(kr.idx * (slot_bytes >> 4));
                    // q's leading bits, then the rest
                    for (int t = 0; t < 2; ++t)
                        for (int c = 0; c < steps; ++c)
                            mma_f8_ss(tm_s + sr.idx * NP, kd + 2 * c, qd0 + (uint64_t)(t * (NP * D >> 4) + 2 * c), idesc, t + c > 0);
                    mma_commit(s_full(sr.idx));
                    mma_commit(k_empty(kr.idx));
                }
                __syncwarp();
                kr.next(sm.ks);
                sr.next(kBufs);
            }
        }
        if (elect_one()) {
            mma_commit(drain_qk);
            wait_unconditional(drain_qk, 0);
        }
        __syncwarp();
    } else if (warp == 2) {
        // ------------------------------------------------------------ P.V issuer
        const uint32_t idesc = make_idesc_f16(128, NP, 1);
        const uint64_t pd0 = make_smem_desc(base + sm.p, 128, 2048, kSwizzleNone);
        Ring br, orr;
        int n_seg = 0;
        bool ok = true;
        while (ok && walk.next(seg)) {
            if (n_seg++ > 0) {
                ok = mbar_wait(o_free, orr.parity, abort_flag);     // the accumulators of the segment before have been read
                orr.next(1);
            }
            for (int j = 0; ok && j < seg.T; ++j) {
                ok = mbar_wait(vt_full(br.idx), br.parity, abort_flag) && ok;
                ok = mbar_wait(p_full(br.idx), br.parity, abort_flag) && ok;
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t pd = pd0 + (uint64_t)(br.idx * (NP * 256 >> 4));
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        mma_f16_ts(tm_o, tm_v + br.idx * 64 + c * 8, pd + (uint64_t)(c * 16), idesc, j + c > 0);
                    mma_commit(pv_done(br.idx));
                }
                __syncwarp();
                br.next(kBufs);
            }
        }
        if (elect_one()) {
            mma_commit(drain_pv);
            wait_unconditional(drain_pv, 0);
        }
        __syncwarp();
    } else if (warp >= kConvertWarp0 && warp < kSoftmaxWarp0) {
        // ------------------------------------------------- V codes to fp16 in tensor memory
        const int wq = warp & 3;                       // channels 32 wq .. + 31 = TMEM lanes
        Ring vr, br;
        int n = 0;
        bool ok = 32 * wq < D;
        while (ok && walk.next(seg)) {
            for (int j = 0; ok && j < seg.T; ++j, ++n) {
                ok = mbar_wait(v_full(vr.idx), vr.parity, abort_flag);
                if (n >= kBufs) ok = mbar_wait(pv_done(br.idx), br.parity ^ 1u, abort_flag) && ok;
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const int live = seg.len - (seg.t0 + j) * kTilePos;      // positions of this tile below the length
                const uint32_t tile = base + sm.v + vr.idx * slot_bytes;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t w[32];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int pos = u * 32 + lane, chunk = wq * 2 + h;
                        const int phase = D == 128 ? pos & 7 : (pos >> 1) & 3;
                        uint32_t r[4];
                        ldmatrix_b8_x2(tile + pos * D + ((chunk ^ phase) << 4), r);
                        if (live < kTilePos) {
                            // what lies behind the sequence is not the cache's: it may be anything, NaN among it
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const int left = live - (u * 32 + (k >> 1) * 16 + (lane & 3) * 4);
                                if (left < 4) r[k] &= left <= 0 ? 0u : 0xFFFFFFFFu >> (8 * (4 - left));
                            }
                        }
                        // matrix m of this pair holds registers 2 m (row) and 2 m + 1 (row + 8)
#pragma unroll
                        for (int k = 0; k < 4; ++k) decode4(r[k], w[u * 8 + k * 2], w[u * 8 + k * 2 + 1]);
                    }
                    if (h == 1) {
                        __syncwarp();
                        if (lane == 0) mbar_arrive(v_empty(vr.idx));
                    }
                    tmem_st_16x256b_x8(tm_v + br.idx * 64 + ((uint32_t)(wq * 32 + h * 16) << 16), w);
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(vt_full(br.idx));
                vr.next(sm.vs);
                br.next(kBufs);
            }
        }
    } else if (warp >= kSoftmaxWarp0) {
        // ------------------------------------------------------------ softmax
        const int grp = (warp - kSoftmaxWarp0) >> 2, bar_id = 1 + grp;
        const int wq = warp & 3, row = wq * 32 + lane;          // TMEM lane: position of the tile, channel of the output
        const int stid = tid - 32 * kSoftmaxWarp0;
        const uint32_t lane_addr = (uint32_t)(wq * 32) << 16;
        const int c_lo = grp == 0 ? 0 : (n8 + 1) / 2, n_c = grp == 0 ? (n8 + 1) / 2 : n8 / 2, col0 = c_lo * 8;
        float *my_sums = sums_s + wq * NP + col0;
        Ring sr, br, done;
        int n = 0;
        // No wait ends a loop here: a warp that left would leave its group at a barrier.  After a wait has run out all
        // others end at once, and what is computed then is void.
        while (walk.next(seg)) {
            const int L = seg.len;
            const int vis0 = p.span[2 * seg.b], vis1 = p.span[2 * seg.b + 1];
            const int32_t *table = p.block_table + (size_t)seg.b * p.pages_per_seq;
            // ---- scales, asked for ahead: the table's entry two tiles, the scale one tile
            PageWalk at(p, seg.t0, row);
            int pos_e = seg.t0 * kTilePos + row;
            auto entry = [&]() {
                const int e = pos_e < L ? table[at.page] : -1;
                pos_e += kTilePos;
                return (unsigned)e < (unsigned)p.n_pages ? e : -1;
            };
            auto scales = [&](int e, int off, float &k, float &v) {
                k = v = 0.f;
                if (e < 0) return;
                const size_t i = ((size_t)e * p.Hkv + seg.head) * p.blocks_per_page + (off >> p.block_log2);
                k = p.k_scale[i];
                v = p.v_scale[i];
            };
            int e_next = entry(), off_next = at.off;
            float ks, vs, ks_next, vs_next;
            scales(e_next, off_next, ks_next, vs_next);
            at.next_tile(p);
            e_next = entry();
            off_next = at.off;

            // ---- q as two E4M3 operand tiles
            float scale;
            {
                const int per_row = D / 8, n_chunks = NP * per_row;
                constexpr int kMine = (kC * 16 * 16 + kSoftmaxThreads - 1) / kSoftmaxThreads;   // 16-byte chunks of a thread
                uint4 qv[kMine];
                uint32_t amax = 0;
#pragma unroll
                for (int u = 0; u < kMine; ++u) {
                    const int ch = stid + u * kSoftmaxThreads;
                    qv[u] = make_uint4(0, 0, 0, 0);
                    if (ch < n_chunks) {
                        const int r = D == 128 ? ch >> 4 : ch >> 3, c = ch & (per_row - 1);
                        if (r < M) {
                            const int g = div_by(r, G, P.group_magic), hg = r - g * G;
                            qv[u] = *reinterpret_cast<const uint4 *>(
                                p.q + (((size_t)seg.b * gamma + g) * p.Hq + seg.head * G + hg) * D + c * 8);
                        }
                        const uint32_t w[4] = {qv[u].x, qv[u].y, qv[u].z, qv[u].w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) amax = max(amax, max(w[k] & 0x7FFFu, (w[k] >> 16) & 0x7FFFu));
                    }
                }
                amax = __reduce_max_sync(0xffffffffu, amax);
                // (a segment's first barrier: nobody still reads the last one's maxima, its epilogue lies between)
                if (lane == 0) wmax_s[warp - kSoftmaxWarp0] = amax;
                named_sync(1 + kGroups, kSoftmaxThreads);
#pragma unroll
                for (int u = 0; u < 4 * kGroups; ++u) amax = max(amax, wmax_s[u]);
                // the power of two that brings the largest magnitude into [128, 256); NaN or Inf in q: none, the result is NaN
                int shift = 0;
                if (amax > 0 && amax < 0x7F80u) shift = 7 - ((int)(amax >> 7) - 127);
                shift = max(-100, min(100, shift));
                const float up = __uint_as_float((uint32_t)(127 + shift) << 23);
                scale = p.scale_log2 * __uint_as_float((uint32_t)(127 - shift) << 23);
#pragma unroll
                for (int u = 0; u < kMine; ++u) {
                    const int ch = stid + u * kSoftmaxThreads;
                    if (ch >= n_chunks) continue;
                    const int r = D == 128 ? ch >> 4 : ch >> 3, c = ch & (per_row - 1);
                    const uint32_t w[4] = {qv[u].x, qv[u].y, qv[u].z, qv[u].w};
                    uint32_t hd[4], rs[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float x0 = __uint_as_float(w[k] << 16) * up, x1 = __uint_as_float(w[k] & 0xFFFF0000u) * up;
                        const float h0 = e4m3_head(x0), h1 = e4m3_head(x1);
                        hd[k] = pack_e4m3x2(h0, h1);
                        rs[k] = pack_e4m3x2(x0 - h0, x1 - h1);
                    }
                    const int phase = D == 128 ? r & 7 : (r >> 1) & 3;
                    const uint32_t off = r * D + (((c >> 1) ^ phase) << 4) + ((c & 1) << 3);
                    *reinterpret_cast<uint2 *>(gbase + sm.q + off) = make_uint2(hd[0] | (hd[1] << 16), hd[2] | (hd[3] << 16));
                    *reinterpret_cast<uint2 *>(gbase + sm.q + NP * D + off) = make_uint2(rs[0] | (rs[1] << 16), rs[2] | (rs[3] << 16));
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(q_full);
            }

            float l[kC * 8];
#pragma unroll
            for (int k = 0; k < kC * 8; ++k) l[k] = 0.f;
            for (int c = lane; c < n_c * 8; c += 32) my_sums[c] = my_sums[4 * NP + c] = 0.f;
            int l_cat = -1;                             // whose sums l holds: 0 outside, 1 inside the span, -1 none
            int k0 = 0;                                 // V scales are taken relative to 2^k0
            float inv_k0 = 1.f;

            // adds this thread's values to the sums of their kind, over the warp
            auto flush = [&](int cat, bool mine) {
#pragma unroll
                for (int c = 0; c < kC; ++c) {
                    if (c >= n_c) break;
                    float v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = mine ? l[c * 8 + k] : 0.f;
                    const float t = sum8(v, lane);
                    if ((lane & 3) == 0) my_sums[cat * 4 * NP + c * 8 + ((lane >> 4) & 1) * 4 + ((lane >> 3) & 1) * 2 + ((lane >> 2) & 1)] += t;
                }
                __syncwarp();
            };

            for (int j = 0; j < seg.T; ++j, ++n) {
                const int pos0 = (seg.t0 + j) * kTilePos, pos = pos0 + row;
                ks = ks_next;
                vs = vs_next;
                scales(e_next, off_next, ks_next, vs_next);
                at.next_tile(p);
                e_next = entry();
                off_next = at.off;
                const bool tail = pos0 + kTilePos > L - gamma;        // some query does not see some position
                const Seen seen = seen_by(pos - (L - gamma), G, gamma, p.branch_len);
                const float ck = scale * ks;

                mbar_wait(s_full(sr.idx), sr.parity, abort_flag);
                __syncwarp();
                tc_fence_after();
                uint32_t raw[kC][8];
#pragma unroll
                for (int c = 0; c < kC; ++c)
                    if (c < n_c) tmem_ld_x8(tm_s + sr.idx * NP + lane_addr + col0 + c * 8, raw[c]);
                tmem_wait_ld();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(s_free(sr.idx));
                sr.next(kBufs);
                float x[kC * 8];

                if (j == 0) {
                    // the first position's scores set the references
                    if (row == 0) {
#pragma unroll
                        for (int c = 0; c < kC; ++c)
                            if (c < n_c)
#pragma unroll
                                for (int k = 0; k < 8; ++k) {
                                    const float y = __uint_as_float(raw[c][k]) * ck;
                                    m_s[col0 + c * 8 + k] = fabsf(y) < INFINITY ? y - kFirst : 0.f;
                                }
                        const uint32_t e = (__float_as_uint(vs) >> 23) & 0xFFu;
                        wmax_s[8 + grp] = e > 0 && e < 255 ? e : 127;
                    }
                    named_sync(bar_id, 128);
                    k0 = (int)wmax_s[8 + grp] - 127 + 2;
                    inv_k0 = ldexpf(1.f, -k0);
                }
                float vsr = vs * inv_k0;
                float gmax = -INFINITY;
#pragma unroll
                for (int c = 0; c < kC; ++c)
                    if (c < n_c) {
                        const float4 ma = *reinterpret_cast<const float4 *>(m_s + col0 + c * 8);
                        const float4 mb = *reinterpret_cast<const float4 *>(m_s + col0 + c * 8 + 4);
                        const float mm[8] = {ma.x, ma.y, ma.z, ma.w, mb.x, mb.y, mb.z, mb.w};
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            float y = fmaf(__uint_as_float(raw[c][k]), ck, -mm[k]);
                            if (tail) y = seen(col0 + c * 8 + k) ? y : -INFINITY;
                            x[c * 8 + k] = y;
                            gmax = fmaxf(gmax, y);
                        }
                    }
                // (a first tile in the draft slots: its first position need not be one that every query sees)
                if (group_any(bar_id, gmax > kGuard || fabsf(vsr) > 2.f || (j == 0 && tail))) {
                    // ---- references up to this tile's maxima
                    uint32_t e = (__float_as_uint(vs) >> 23) & 0xFFu;
                    if (e == 255u) e = 0u;
                    e = __reduce_max_sync(0xffffffffu, e);
#pragma unroll
                    for (int c = 0; c < kC; ++c)
                        if (c < n_c)
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const float y = warp_max_f32(x[c * 8 + k]);
                                if (lane == 0) tmx_s[wq * NP + col0 + c * 8 + k] = y;
                            }
                    if (lane == 0) wmax_s[warp - kSoftmaxWarp0] = e;
                    named_sync(bar_id, 128);
#pragma unroll
                    for (int u = 0; u < 4; ++u) e = max(e, wmax_s[grp * 4 + u]);
                    const int k_new = (int)e - 127 > k0 ? (int)e - 127 + 2 : k0;
                    const float fk = j > 0 ? ldexpf(1.f, max(k0 - k_new, -200)) : 1.f;
                    if (j > 0) {
                        // (the products of the tile before have ended)
                        mbar_wait(pv_done(done.idx), done.parity, abort_flag);
                        __syncwarp();
                        tc_fence_after();
                    }
#pragma unroll
                    for (int c = 0; c < kC; ++c)
                        if (c < n_c) {
                            uint32_t o[8];
                            if (j > 0) {
                                tmem_ld_x8(tm_o + lane_addr + col0 + c * 8, o);
                                tmem_wait_ld();
                            }
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const int col = col0 + c * 8 + k;
                                const float top = fmaxf(fmaxf(tmx_s[col], tmx_s[NP + col]), fmaxf(tmx_s[2 * NP + col], tmx_s[3 * NP + col]));
                                const bool moves = j == 0 ? top > -INFINITY : top > kGuard;
                                const float up = moves ? top - kFirst : 0.f;
                                x[c * 8 + k] -= up;
                                const float f = ex2(-up);
                                if (moves) l[c * 8 + k] *= f;
                                if (j > 0) o[k] = __float_as_uint(__uint_as_float(o[k]) * (f * fk));
                            }
                            if (j > 0) tmem_st_x8(tm_o + lane_addr + col0 + c * 8, o);
                        }
                    if (j > 0) tmem_wait_st();
                    tc_fence_before();
                    // the warp's own sums, and (one warp of the group) the references
                    for (int c = lane; c < n_c * 8; c += 32) {
                        const int col = col0 + c;
                        const float top = fmaxf(fmaxf(tmx_s[col], tmx_s[NP + col]), fmaxf(tmx_s[2 * NP + col], tmx_s[3 * NP + col]));
                        const bool moves = j == 0 ? top > -INFINITY : top > kGuard;
                        if (moves) {
                            const float f = ex2(kFirst - top);
                            my_sums[c] *= f;
                            my_sums[4 * NP + c] *= f;
                            if (wq == 0) m_s[col] += top - kFirst;
                        }
                    }
                    k0 = k_new;
                    inv_k0 = ldexpf(1.f, -k0);
                    vsr = vs * inv_k0;
                    named_sync(bar_id, 128);
                }

                // ---- probabilities
                const int cat = pos0 >= vis0 && pos0 + kTilePos <= vis1 ? 1 : pos0 + kTilePos <= vis0 || pos0 >= vis1 ? 0 : 2;
                if (cat != l_cat) {
                    if (l_cat >= 0) {
                        flush(l_cat, true);
#pragma unroll
                        for (int k = 0; k < kC * 8; ++k) l[k] = 0.f;
                    }
                    l_cat = cat;
                }
                if (n >= kBufs) mbar_wait(pv_done(br.idx), br.parity ^ 1u, abort_flag);
                uint8_t *prow = gbase + sm.p + br.idx * (NP * 256) + c_lo * 2048 + row * 16;
#pragma unroll
                for (int c = 0; c < kC; ++c)
                    if (c < n_c) {
                        float e[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            e[k] = ex2(x[c * 8 + k]);
                            l[c * 8 + k] += e[k];
                        }
                        *reinterpret_cast<uint4 *>(prow + c * 2048) =
                            make_uint4(pack_f16x2(e[0] * vsr, e[1] * vsr), pack_f16x2(e[2] * vsr, e[3] * vsr),
                                       pack_f16x2(e[4] * vsr, e[5] * vsr), pack_f16x2(e[6] * vsr, e[7] * vsr));
                    }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full(br.idx));
                done = br;
                br.next(kBufs);
                if (cat == 2) {
                    const bool in = pos >= vis0 && pos < vis1;
                    flush(1, in);
                    flush(0, !in);
#pragma unroll
                    for (int k = 0; k < kC * 8; ++k) l[k] = 0.f;
                    l_cat = -1;
                }
            }
            if (l_cat >= 0) flush(l_cat, true);
            mbar_wait(pv_done(done.idx), done.parity, abort_flag);
            __syncwarp();
            tc_fence_after();
            named_sync(bar_id, 128);                    // the group's sums are there

            // ---- results: whole, or this CTA's part of them
            const bool whole = seg.first && seg.last;
            const float vk = ldexpf(1.f, k0 / 2), vk2 = ldexpf(1.f, k0 - k0 / 2);
            const int slot = part_slot(blockIdx.x, seg.first);
            float *part_o = p.part_o + (size_t)slot * M * D;
            float *part_stat = p.part_stat + (size_t)slot * M * 4;
#pragma unroll 1
            for (int c = 0; c < n_c; ++c) {
                uint32_t o[8];
                tmem_ld_x8(tm_o + lane_addr + col0 + c * 8, o);
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int col = col0 + c * 8 + k;
                    if (col >= M) break;
                    const float *t = sums_s + col;
                    const float in = t[4 * NP] + t[5 * NP] + t[6 * NP] + t[7 * NP];
                    const float all = t[0] + t[NP] + t[2 * NP] + t[3 * NP] + in;
                    const float v = __uint_as_float(o[k]) * vk * vk2;
                    if (whole) {
                        const int g = div_by(col, G, P.group_magic), hg = col - g * G;
                        const size_t at_row = ((size_t)seg.b * gamma + g) * p.Hq + seg.head * G + hg;
                        const float inv = all == 0.f ? 0.f : 1.f / all;       // a query that sees nothing gives zeros
                        if (row < D) p.out[at_row * D + row] = (uint16_t)(pack_bf16x2(all == 0.f ? 0.f : v * inv, 0.f) & 0xFFFFu);
                        if (row == 0) p.mass[at_row] = in * inv;
                    } else {
                        if (row < D) part_o[(size_t)col * D + row] = v;
                        if (row == 0) *reinterpret_cast<float4 *>(part_stat + col * 4) = make_float4(m_s[col], all, in, 0.f);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(o_free);
            named_sync(1 + kGroups, kSoftmaxThreads);   // sums, references and q may be written anew
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, (uint32_t)P.tmem_cols);
    if (tid == 0 && *abort_flag) atomicOr(p.status, LVSPEC_DEV_WAIT_EXPIRED);
}

// Merges the parts of pairs that several CTAs share: one warp per query row.  With m, l and the unnormalised O of
// each part, w = 2^(m - max m): out = sum w O / sum w l, mass = sum w l_vis / sum w l, summed in the CTAs' order.
// Rows of empty sequences are written as zeros here.
template <int D>
__global__ void __launch_bounds__(32 * kMergeWarps) merge_paged_fp8_kernel(const PagedFp8Params p, const uint32_t group_magic)
{
    __shared__ Line line;
    constexpr int kEach = D / 32;
    using Vec = typename std::conditional<D == 128, float4, float2>::type;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    grid_launch_dependents();
    grid_dependency_wait();
    if (warp == 0) make_line(line, p);
    __syncthreads();
    const int row = blockIdx.x * kMergeWarps + warp;
    if (row >= p.B * p.gamma * p.Hq) return;
    const int b = row / (p.gamma * p.Hq), r = row - b * p.gamma * p.Hq, g = r / p.Hq, h = r - g * p.Hq;
    const int head = div_by(h, p.G, group_magic), col = g * p.G + h - head * p.G;
    uint16_t *out = p.out + (size_t)row * D + lane * kEach;
    const int tiles = tiles_of(line.len[b]);
    float acc[kEach] = {};
    float inv = 0.f, mass = 0.f;
    if (tiles > 0) {
        const int first = line.start[b] + head * padded(line, tiles);
        const int c0 = first / line.share, c1 = (first + tiles - 1) / line.share;
        if (c0 == c1) return;                           // that CTA has finished the pair itself
        auto stat = [&](int c) { return *reinterpret_cast<const float4 *>(p.part_stat + ((size_t)part_slot(c, c == c0) * p.M + col) * 4); };
        float top = -INFINITY;
        for (int c = c0 + lane; c <= c1; c += 32) {
            const float4 s = stat(c);
            if (s.y != 0.f) top = fmaxf(top, s.x);
        }
        top = warp_max_f32(top);
        float total = 0.f, vis = 0.f;
        for (int cb = c0; cb <= c1; cb += 32) {
            float w = 0.f, wl = 0.f, wv = 0.f;
            if (cb + lane <= c1) {
                const float4 s = stat(cb + lane);
                if (s.y != 0.f) w = ex2(s.x - top);     // (a part that the row sees nothing of counts for nothing)
                wl = w * s.y;
                wv = w * s.z;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                wl += __shfl_xor_sync(0xffffffffu, wl, o);
                wv += __shfl_xor_sync(0xffffffffu, wv, o);
            }
            total += wl;
            vis += wv;
            const int n = min(32, c1 - cb + 1);
#pragma unroll 4
            for (int u = 0; u < n; ++u) {
                const float wu = __shfl_sync(0xffffffffu, w, u);
                if (wu == 0.f) continue;
                const Vec v = *reinterpret_cast<const Vec *>(p.part_o + ((size_t)part_slot(cb + u, cb + u == c0) * p.M + col) * D + lane * kEach);
                const float *f = reinterpret_cast<const float *>(&v);
#pragma unroll
                for (int k = 0; k < kEach; ++k) acc[k] = fmaf(wu, f[k], acc[k]);
            }
        }
        inv = total == 0.f ? 0.f : 1.f / total;
        mass = vis * inv;
    }
#pragma unroll
    for (int k = 0; k < kEach; k += 2)
        *reinterpret_cast<uint32_t *>(out + k) = pack_bf16x2(acc[k] * inv, acc[k + 1] * inv);
    if (lane == 0) p.mass[row] = mass;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// A page pool as [pages][heads][positions][channels]; a box is a tile of one page and head, or all of a shorter page.
bool make_pool_map(CUtensorMap *map, const uint8_t *pool, const PagedFp8Params &p)
{
    static EncodeTiledFn fn = nullptr;
    if (!fn) {
        void *sym = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            return false;
        fn = reinterpret_cast<EncodeTiledFn>(sym);
    }
    const cuuint64_t dims[4] = {(cuuint64_t)p.D, (cuuint64_t)p.page_size, (cuuint64_t)p.Hkv, (cuuint64_t)p.n_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)p.position_stride, (cuuint64_t)p.head_stride, (cuuint64_t)p.page_stride};
    const cuuint32_t box[4] = {(cuuint32_t)p.D, (cuuint32_t)(p.page_size < kTilePos ? p.page_size : kTilePos), 1, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<uint8_t *>(pool), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, p.D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kC>
cudaError_t launch_attention(const KernelParams &P, const CUtensorMap &tk, const CUtensorMap &tv, cudaStream_t stream, int *launches)
{
    const size_t smem = P.sm.total + 1024;
    cudaError_t e = cudaFuncSetAttribute(attn_paged_fp8_kernel<kC>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch_after(attn_paged_fp8_kernel<kC>, dim3((unsigned)P.a.n_cta), kThreads, smem, P.a.pdl != 0, stream, launches, P, tk, tv);
}

}  // namespace

size_t paged_fp8_scratch_bytes(int n_cta, int M, int D) { return (size_t)2 * n_cta * M * (D + 4) * sizeof(float); }

cudaError_t launch_attn_paged_fp8(const PagedFp8Params &p, const uint8_t *k_pool, const uint8_t *v_pool, cudaStream_t stream,
                                  int *launches)
{
    KernelParams P;
    P.a = p;
    P.NP = (p.M + 15) & ~15;
    int cols = 32;
    while (cols < kBufs * 64 + (kBufs + 1) * P.NP) cols *= 2;
    P.tmem_cols = cols;
    P.group_magic = p.G > 1 ? 0xFFFFFFFFu / (uint32_t)p.G + 1u : 0u;
    // as many slots as shared memory holds, K's one more where the count is odd (its tile is used first)
    int slots = 12;
    do P.sm = smem_map(p.D, P.NP, (slots + 1) / 2, slots / 2);
    while (P.sm.total + 1024 > 227 * 1024 && --slots > 2);
    CUtensorMap tk, tv;
    if (!make_pool_map(&tk, k_pool, p) || !make_pool_map(&tv, v_pool, p)) return cudaErrorInvalidValue;
    cudaError_t e;
    switch ((((p.M + 7) / 8) + 1) / 2) {
        case 1: e = launch_attention<1>(P, tk, tv, stream, launches); break;
        case 2: e = launch_attention<2>(P, tk, tv, stream, launches); break;
        case 3: e = launch_attention<3>(P, tk, tv, stream, launches); break;
        case 4: e = launch_attention<4>(P, tk, tv, stream, launches); break;
        case 5: e = launch_attention<5>(P, tk, tv, stream, launches); break;
        case 6: e = launch_attention<6>(P, tk, tv, stream, launches); break;
        default: e = launch_attention<8>(P, tk, tv, stream, launches); break;
    }
    if (e != cudaSuccess) return e;
    const int rows = p.B * p.gamma * p.Hq;
    const dim3 grid((unsigned)((rows + kMergeWarps - 1) / kMergeWarps));
    return p.D == 128 ? launch_after(merge_paged_fp8_kernel<128>, grid, 32 * kMergeWarps, 0, p.pdl != 0, stream, launches, p, P.group_magic)
                      : launch_after(merge_paged_fp8_kernel<64>, grid, 32 * kMergeWarps, 0, p.pdl != 0, stream, launches, p, P.group_magic);
}

}  // namespace lvspec
