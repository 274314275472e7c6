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
// The tiles of a segment (a CTA's share of one sequence and head) go to two streams in turn, each with its own softmax group of
// four warps, references, sums and accumulators of O, put together when the segment ends: while one group works on a tile the
// other's products run.  From 97 rows on tensor memory holds one stream, whose two groups share out the columns.  A tile's chain is
// wait for S^T, pass, vote, P^T there, next K.Q^T: at 80 rows 4150 cycles, 930 of them the wait and 2460 the pass (the
// special-function unit needs 640), the mean over a call's tiles; at 40 rows 2600, 150 and 1800.  That chain, not HBM, bounds all but
// the longest launches of few rows.
//
// The reference exponent of a row is taken from the stream's first tile: its largest probability there becomes 2^6.  It moves (the
// tile's pass is taken back, a maximum over the lanes, accumulators rescaled, the pass made again) when a score passes 2^14.  fp16 then
// holds a probability with eleven bits down to 2^-20 of the first tile's largest, and down to 2^-30 with fewer.  V scales are
// taken relative to 2^(k0): four times the power of two below the largest of that tile, moved with the references.
//
// Work is laid out on the device, from the lengths: the tiles of all (sequence, KV head) pairs in a row are cut into
// equal shares, one per SM, either at multiples of the share within each pair (no CTA has two pairs) or straight
// through (a CTA may end one pair and begin the next).  A captured launch so follows lengths that change, and a batch of
// different lengths keeps all SMs busy.  Partials of pairs that several CTAs share are merged by a second, small
// kernel; a pair that one CTA has to itself is finished there.
//
// Measured, us a call (merge included): 8 heads x 131071 positions x 2 sequences, 20 rows 102 (537 MB, 5.3 TB/s); 14 sequences of
// 16000 to 32003, 80 rows 245 (75 tiles a stream on the busiest SM, 376 000 cycles with the segments' ends, at the 1.8 GHz that the
// power cap leaves); 32768 positions, 40 rows 28; 8 x 16384 ragged, 7 rows 27; 333 positions 11 (launches and cold code: a CTA's first
// product is ready 6 us after its lengths).
#include <cuda_bf16.h>

#include <type_traits>

#include "lvspec_internal.h"
#include "sm100_ptx.cuh"
#include "tensor_map.h"

namespace lvspec {
namespace {

using namespace ptx;

constexpr int kTilePos = 128;
constexpr int kVBufs = 2;                   // V^T buffers in tensor memory, and sets of four warps that fill them
constexpr int kConvertWarp0 = 4, kSoftmaxWarp0 = kConvertWarp0 + 4 * kVBufs;
constexpr int kGroups = 2;                  // softmax groups, of four warps each
constexpr int kThreads = 32 * kSoftmaxWarp0 + 128 * kGroups;
// Registers of a thread at launch, and what the softmax warps are given when the others have given up theirs (kIssueRegs for the
// four warps that issue, kConvertRegs for those that convert).
constexpr int kIssueRegs = 40, kConvertRegs = 48, kLaunchRegs = 96, kSoftmaxRegs = 168;
static_assert(32 * (kConvertWarp0 * kIssueRegs + 4 * kVBufs * kConvertRegs + 4 * kGroups * kSoftmaxRegs) <= kThreads * kLaunchRegs &&
                  kThreads * kLaunchRegs <= 65536,
              "a share of the registers that is not there is waited for without end");
// chunks of columns that the registers hold beside the sums
__host__ __device__ constexpr int block_of(int chunks)
{
    const int room = (kSoftmaxRegs - 36) / 8 - chunks;
    return room >= chunks ? chunks : room >= (chunks + 1) / 2 ? (chunks + 1) / 2 : room >= 2 ? 2 : 1;
}
constexpr int kMergeWarps = 8;
constexpr int kMaxBufs = 4;                 // S^T buffers and P^T buffers, at most
constexpr float kFirst = 6.f;               // log2 of the largest probability of a stream's first tile
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

// ceil(x / d) for x < 2^30 with m = 2^32 / d + 1 (0 for d = 1): the product is one too large at most
__device__ __forceinline__ int ceil_div(int x, int d, uint32_t m)
{
    const int y = x + d - 1;
    if (m == 0u) return x;
    const int q = (int)__umulhi((uint32_t)y, m);
    return q * d > y ? q - 1 : q;
}
__device__ __forceinline__ uint32_t magic_of(uint32_t d) { return d > 1 ? 0xFFFFFFFFu / d + 1u : 0u; }

// One warp.  True when a length lies outside 0..max_len (the sequence then counts as empty).
__device__ __forceinline__ bool make_line(Line &w, const int32_t *kv_len, int B, int Hkv, int max_len, int n_cta)
{
    const int lane = threadIdx.x & 31;
    int total = 0;
    bool bad = false;
#pragma unroll 1
    for (int b = lane; b < B; b += 32) {
        int len = kv_len[b];
        if (len < 0 || len > max_len) {
            bad = true;
            len = 0;
        }
        w.len[b] = len;
        total += tiles_of(len);
    }
    total = __reduce_add_sync(0xffffffffu, total) * Hkv;
    const int flat = max(1, (total + n_cta - 1) / n_cta);
    int share = flat, aligned = 0;
    uint32_t magic = 0;
    // cutting within pairs is taken if it costs a few tiles at most: a second pair in a CTA costs as much
#pragma unroll 1
    for (int t = flat; t <= flat + kFlatGain; ++t) {
        magic = magic_of(t);
        int ctas = 0;
#pragma unroll 1
        for (int b = lane; b < B; b += 32) ctas += ceil_div(tiles_of(w.len[b]), t, magic);
        if (__reduce_add_sync(0xffffffffu, ctas) * Hkv <= n_cta) {
            share = t;
            aligned = 1;
            break;
        }
    }
    int before = 0;
#pragma unroll 1
    for (int b0 = 0; b0 < B; b0 += 32) {
        const int b = b0 + lane, tiles = b < B ? tiles_of(w.len[b]) : 0;
        const int mine = (aligned ? ceil_div(tiles, share, magic) * share : tiles) * Hkv;
        int in = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, in, o);
            if (lane >= o) in += y;
        }
        if (b < B) w.start[b] = before + in - mine;
        before += __shfl_sync(0xffffffffu, in, 31);
    }
    if (lane == 0) {
        w.start[B] = before;
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
    int at, end, b;
    __device__ __forceinline__ Walk(const Line &w, int n_seq, int cta) : b(0)
    {
        at = cta * w.share;
        end = min(at + w.share, w.start[n_seq]);
    }
};
__device__ __forceinline__ bool next_segment(const Line &w, Walk &walk, Segment &s)
{
    if (walk.at >= walk.end) return false;
    int b = walk.b;
    while (walk.at >= w.start[b + 1]) ++b;
    s.b = walk.b = b;
    s.len = w.len[b];
    s.tiles = tiles_of(s.len);
    const int each = padded(w, s.tiles), off = walk.at - w.start[b];
    s.head = off / each;
    s.t0 = off - s.head * each;
    const int stop = min(walk.end, w.start[b] + (s.head + 1) * each);
    s.T = min(s.tiles - s.t0, stop - walk.at);
    s.first = s.t0 == 0;
    s.last = s.t0 + s.T == s.tiles;
    walk.at = stop;
    return true;
}
// Partial results of a CTA: of the pair it goes on with, and of the pair it begins and does not end.
__device__ __forceinline__ int part_slot(int cta, bool first) { return 2 * cta + (first ? 1 : 0); }

// ---- shared memory --------------------------------------------------------------------
struct Smem {
    uint32_t k, v, q, p, nm, tmx, fac, sums, rows, scale, nan, bars, misc, seg, line, total;
    int ks, vs;                             // K and V slots
    int s_log2, p_log2;                     // S^T and P^T buffers
};
constexpr int kBarsFixed = 3 * kMaxBufs + 2 * kVBufs + 4;
Smem smem_map(int D, int NP, int streams, int ks, int vs, int s_log2, int p_log2)
{
    Smem s;
    uint32_t o = 0;
    s.ks = ks;
    s.vs = vs;
    s.s_log2 = s_log2;
    s.p_log2 = p_log2;
    s.k = o;    o += ks * kTilePos * D;
    s.v = o;    o += vs * kTilePos * D;
    s.q = o;    o += 2 * NP * D;
    s.p = o;    o += (NP * 256) << p_log2;
    s.nm = o;   o += streams * NP * 4;            // [stream][NP]: minus the reference exponents
    s.tmx = o;  o += streams * 4 * NP * 4;  // [stream][warp of the group][NP]: a tile's maxima
    s.fac = o;  o += streams * NP * 4;      // [stream][NP]: what a move multiplies by; the streams' weights at the end
    s.sums = o; o += streams * 2 * 4 * NP * 4;   // [stream][all, inside the span][warp of the group][NP]
    s.rows = o; o += NP * 4;
    s.scale = o; o += kMaxBufs * 16 * 4;    // [S^T buffer][K, V][block of the tile]
    s.nan = o; o += kVBufs * 4 * 4 * 4;
    s.bars = o; o += 8 * (2 * ks + 2 * vs + kBarsFixed);
    s.misc = o; o += 128;                   // TMEM address, abort flag, words of the softmax warps and groups
    s.seg = o; o += (sizeof(Segment) + 15) & ~15u;
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
// tile n's place in a ring of 2^log2 buffers, and the parity of its round
__device__ __forceinline__ int place(int n, int log2) { return n & ((1 << log2) - 1); }
__device__ __forceinline__ uint32_t round_of(int n, int log2) { return (uint32_t)(n >> log2) & 1u; }

// Bounded wait (about two seconds, then the CTA's abort flag is raised): as mbar_wait, in fewer instructions.
__device__ __forceinline__ uint32_t timer_lo()
{
    uint32_t t;
    asm volatile("mov.u32 %0, %globaltimer_lo;" : "=r"(t));
    return t;
}
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int *abort_flag)
{
    if (mbar_try_wait(bar, parity)) return true;
    const uint32_t t0 = timer_lo();
    while (!mbar_try_wait(bar, parity)) {
        if (*abort_flag) return false;
        if (timer_lo() - t0 > 2000000000u) *abort_flag = 1;
    }
    return true;
}
// 2^k, k within -126 .. 127
__device__ __forceinline__ float pow2(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

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
// 16 lanes x 32 columns: lane t's registers 4 i .. 4 i + 3 are row t / 4, columns 8 i + 2 (t % 4) and the next,
// then row t / 4 + 8.
__device__ __forceinline__ void tmem_st_16x256b_x4(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// Takes registers from (gives them to) the pool that the block was launched with.
template <int kRegs>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs) : "memory"); }
template <int kRegs>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs)); }
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

// Sum of each of eight values over the warp's lanes: lanes with lane % 4 == 0 get that of value number (bits 4, 3, 2 of the
// lane, the highest first).  Nine shuffles where plain sums take forty.
__device__ __forceinline__ float warp_sums(const float *v, int lane)
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

__device__ __forceinline__ uint64_t pair(float lo, float hi) { return pack_f32x2(__float_as_uint(lo), __float_as_uint(hi)); }
__device__ __forceinline__ void tmem_ld_x16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld_x32(uint32_t taddr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
        "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
          "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
          "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// A view of the references (minus them) in shared memory that the compiler may read ahead of the stores to P^T, which it could not
// tell apart otherwise: a warp then waits for a chunk's stores before it asks for the next one's references, 200 cycles a
// chunk instead of the 64 that its exponentials take.  Made anew (here) whenever the references may have changed.
struct References {
    uint32_t at;
    __device__ __forceinline__ explicit References(const float *nm)
    {
        asm volatile("mov.u32 %0, %1;" : "=r"(at) : "r"(smem_u32(nm)) : "memory");
    }
    __device__ __forceinline__ void get8(int first, uint64_t (&n2)[4]) const
    {
        asm("ld.shared.v2.u64 {%0, %1}, [%2];" : "=l"(n2[0]), "=l"(n2[1]) : "r"(at + 4 * first));
        asm("ld.shared.v2.u64 {%0, %1}, [%2];" : "=l"(n2[2]), "=l"(n2[3]) : "r"(at + 4 * first + 16));
    }
};

// Scaled scores x of eight columns, from `first` on of the group's: score * ck + (minus the reference)
template <bool kMask>
__device__ __forceinline__ void scores8(const uint32_t *raw, References nm, int first, float ck, Seen seen, int col, float (&x)[8])
{
    const uint64_t c2 = pair(ck, ck);
    uint64_t n2[4];
    nm.get8(first, n2);
#pragma unroll
    for (int k = 0; k < 4; ++k) unpack_f32x2(fma_f32x2(pack_f32x2(raw[2 * k], raw[2 * k + 1]), c2, n2[k]), x[2 * k], x[2 * k + 1]);
    if (kMask)
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = seen(col + k) ? x[k] : -INFINITY;
}

// Eight columns of one position: probabilities into P^T and (times sign, s2) the sums.
template <bool kMask>
__device__ __forceinline__ void softmax8(const uint32_t *raw, References nm, int first, float ck, Seen seen, int col, uint64_t v2,
                                         uint64_t s2, float &top, float *l, uint8_t *to)
{
    float x[8];
    scores8<kMask>(raw, nm, first, ck, seen, col, x);
    top = max3(max3(top, x[0], x[1]), max3(x[2], x[3], x[4]), max3(x[5], x[6], x[7]));
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = ex2(x[k]);
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint64_t e2 = pair(x[2 * k], x[2 * k + 1]);
        unpack_f32x2(fma_f32x2(s2, e2, pair(l[2 * k], l[2 * k + 1])), l[2 * k], l[2 * k + 1]);
        float a, b;
        unpack_f32x2(mul_f32x2(e2, v2), a, b);
        if (kMask) {                    // (v2 is NaN where the cache is: a query that does not see the position takes nothing of it)
            a = x[2 * k] == 0.f ? 0.f : a;
            b = x[2 * k + 1] == 0.f ? 0.f : b;
        }
        w[k] = pack_f16x2(a, b);
    }
    *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
}

// kN chunks of eight columns, asked for in as few instructions as it takes.
template <int kN>
__device__ __forceinline__ void tmem_ld_chunks(uint32_t taddr, uint32_t *r)
{
    if constexpr (kN >= 4) {
        tmem_ld_x32(taddr, *reinterpret_cast<uint32_t(*)[32]>(r));
        if constexpr (kN > 4) tmem_ld_chunks<kN - 4>(taddr + 32, r + 32);
    } else if constexpr (kN >= 2) {
        tmem_ld_x16(taddr, *reinterpret_cast<uint32_t(*)[16]>(r));
        if constexpr (kN > 2) tmem_ld_chunks<kN - 2>(taddr + 16, r + 16);
    } else {
        tmem_ld_x8(taddr, *reinterpret_cast<uint32_t(*)[8]>(r));
    }
}

// One tile, one position, kC chunks of eight columns, kBlock of them at a time (asking tensor memory and waiting for it takes
// 170 cycles, whatever the number of columns; 16 columns' work takes 330): probabilities into P^T and (times sign) the sums;
// returns the largest scaled score.
template <int kC, int kBlock, bool kMask>
__device__ __forceinline__ float softmax_pass(uint32_t s_addr, const float *nm_s, float ck, float vsr, Seen seen, int col0,
                                              uint8_t *prow, float sign, float (&l)[kC * 8])
{
    float top = -INFINITY;
    const References nm(nm_s);
    const uint64_t v2 = pair(vsr, vsr), s2 = pair(sign, sign);
#pragma unroll
    for (int b = 0; b < kC; b += kBlock) {
        uint32_t raw[8 * kBlock];
        if (b + kBlock <= kC) tmem_ld_chunks<kBlock>(s_addr + b * 8, raw);
        else tmem_ld_chunks<kC % kBlock == 0 ? 1 : kC % kBlock>(s_addr + b * 8, raw);
        tmem_wait_ld();
#pragma unroll
        for (int u = 0; u < kBlock; ++u)
            if (b + u < kC)
                softmax8<kMask>(raw + u * 8, nm, (b + u) * 8, ck, seen, col0 + (b + u) * 8, v2, s2, top, l + (b + u) * 8,
                                prow + (b + u) * 2048);
    }
    return top;
}

__device__ __forceinline__ int div_by(int x, int d, uint32_t m)
{
    if (m == 0u) return x;
    const int q = (int)__umulhi((uint32_t)x, m);
    return q * d > x ? q - 1 : q;
}

// The tiles of a segment go to kStreams streams in turn, each with its own references, sums and accumulators of O, put together when
// the segment ends; the groups of a stream (kGroups / kStreams) share out the columns, kC chunks of eight to a group.
template <int kStreams, int kC>
__global__ void __launch_bounds__(kThreads, 1)
attn_paged_fp8_kernel(const KernelParams P, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v)
{
    constexpr int kSoftmaxThreads = 128 * kGroups;
    extern __shared__ uint8_t smem_raw[];
    const PagedFp8Params &p = P.a;
    const Smem &sm = P.sm;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int D = p.D, NP = P.NP, M = p.M, G = p.G, gamma = p.gamma;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *gbase = smem_raw + (base - smem_u32(smem_raw));
    float *nm_s = reinterpret_cast<float *>(gbase + sm.nm), *fac_s = reinterpret_cast<float *>(gbase + sm.fac);
    float *sums_s = reinterpret_cast<float *>(gbase + sm.sums);
    float *scale_s = reinterpret_cast<float *>(gbase + sm.scale);
    int *row_s = reinterpret_cast<int *>(gbase + sm.rows);           // output row of each column
    uint32_t *nan_s = reinterpret_cast<uint32_t *>(gbase + sm.nan);  // [V^T buffer][converting warp][32 positions]: V is NaN there
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(gbase + sm.misc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(gbase + sm.misc + 4);
    volatile uint32_t *wmax_s = reinterpret_cast<volatile uint32_t *>(gbase + sm.misc + 16);
    Line &line = *reinterpret_cast<Line *>(gbase + sm.line);
    volatile Segment &seg_s = *reinterpret_cast<volatile Segment *>(gbase + sm.seg);     // the softmax warps'
    const uint32_t slot_bytes = kTilePos * D;

    const uint32_t bar0 = base + sm.bars;
    auto k_full = [&](int s) { return bar0 + 8 * s; };
    auto k_empty = [&](int s) { return bar0 + 8 * (sm.ks + s); };
    auto v_full = [&](int s) { return bar0 + 8 * (2 * sm.ks + s); };
    auto v_empty = [&](int s) { return bar0 + 8 * (2 * sm.ks + sm.vs + s); };
    const uint32_t bar1 = bar0 + 8 * (2 * sm.ks + 2 * sm.vs);
    auto s_full = [&](int n) { return bar1 + 8 * place(n, sm.s_log2); };       // the product, and the tile's scales
    auto p_full = [&](int n) { return bar1 + 8 * (kMaxBufs + place(n, sm.p_log2)); };      // P^T there, S^T read
    auto pv_done = [&](int n) { return bar1 + 8 * (2 * kMaxBufs + place(n, sm.p_log2)); };
    const uint32_t bar2 = bar1 + 8 * 3 * kMaxBufs;
    auto vt_full = [&](int s) { return bar2 + 8 * s; };
    auto vt_free = [&](int s) { return bar2 + 8 * (kVBufs + s); };
    const uint32_t q_full = bar2 + 8 * 2 * kVBufs, o_free = q_full + 8, drain_qk = q_full + 16, drain_pv = q_full + 24;
    constexpr int kShare = kGroups / kStreams;              // groups that work on a tile

    if (warp == 3 && lane < 2) prefetch_tensormap(lane ? &tmap_v : &tmap_k);
    if (warp == 0) {
        const int n_bars = 2 * sm.ks + 2 * sm.vs + kBarsFixed;
        for (int i = lane; i < n_bars; i += 32) {
            const int j = i - 2 * (sm.ks + sm.vs);
            uint32_t count = 1;
            if (j < 0) count = i >= 2 * sm.ks + sm.vs ? D / 32 : 1;                             // v_empty: the converting warps
            else if (j < kMaxBufs) count = 2;                                                   // s_full: the products, the scales
            else if (j < 2 * kMaxBufs) count = kShare;                                          // p_full: one thread of a group
            else if (j >= 3 * kMaxBufs && j < 3 * kMaxBufs + kVBufs) count = D / 32;            // vt_full
            else if (j == 3 * kMaxBufs + 2 * kVBufs || j == 3 * kMaxBufs + 2 * kVBufs + 1) count = 4 * kGroups;     // q_full, o_free
            mbar_init(bar0 + 8 * i, count);
        }
        if (lane == 0) *abort_flag = 0;
        nan_s[lane] = 0;                        // (warps without channels never write theirs)
        fence_proxy_async_smem();
        grid_dependency_wait();
        grid_launch_dependents();
        const bool bad = make_line(line, p.kv_len, p.B, p.Hkv, p.max_len, p.n_cta);
        if (blockIdx.x == 0) {
            if (bad && lane == 0) atomicOr(p.status, LVSPEC_DEV_BAD_LENGTH);
            // (the merge looks it up instead of working it out again)
            __syncwarp();
            if (lane < 2) p.line[lane] = lane ? line.aligned : line.share;
            for (int b = lane; b < p.B; b += 32) *reinterpret_cast<int2 *>(p.line + 2 + 2 * b) = make_int2(line.start[b], line.len[b]);
        }
    } else {
        if (warp == 1) {
            tmem_alloc(base + sm.misc, (uint32_t)P.tmem_cols);
            tmem_relinquish();
        }
        // an odd number of chunks, and the product takes an even one: the last stays zero
        if (8 * kC * kShare < NP && warp >= kSoftmaxWarp0) {
            for (int i = tid - 32 * kSoftmaxWarp0; i < 128 << sm.p_log2; i += kSoftmaxThreads)
                *reinterpret_cast<uint4 *>(gbase + sm.p + (i >> 7) * (NP * 256) + kC * kShare * 2048 + (i & 127) * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
        }
        grid_dependency_wait();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const uint32_t tm_v = tmem, tm_o = tmem + kVBufs * 64, tm_s = tm_o + kStreams * NP;

    Walk walk(line, p.B, blockIdx.x);
    Segment seg;

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer
        fewer_registers<kIssueRegs>();
        const uint64_t policy = l2_evict_first_policy();
        Ring kr, vr;
        const int boxes = p.page_size < kTilePos ? kTilePos / p.page_size : 1;
        const uint32_t box_bytes = slot_bytes / boxes;
        int n = 0;                                     // tiles asked for
        bool ok = true;
        while (ok && next_segment(line, walk, seg)) {
            const int32_t *row = p.block_table + (size_t)seg.b * p.pages_per_seq;
            const int n_live = (seg.len - 1) / p.page_size + 1;           // (a page may be nearly 2^31 long)
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
                if (n >= sm.ks) ok = wait(k_empty(kr.idx), kr.parity ^ 1u, abort_flag);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                const uint32_t kd = base + sm.k + kr.idx * slot_bytes, vd = base + sm.v + vr.idx * slot_bytes;
                if (lane == 0) mbar_arrive_expect_tx(k_full(kr.idx), slot_bytes);
                __syncwarp();
                if (lane < boxes) tma_load_4d_hint(kd + lane * box_bytes, &tmap_k, k_full(kr.idx), 0, at.off, seg.head, page, policy);
                if (n >= sm.vs) ok = wait(v_empty(vr.idx), vr.parity ^ 1u, abort_flag);
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
        fewer_registers<kIssueRegs>();
        const uint32_t idesc = make_idesc_e4m3(128, NP, 0, 0);
        const uint32_t swz = D == 128 ? kSwizzle128B : kSwizzle64B;
        const uint64_t kd0 = make_smem_desc(base + sm.k, 16, 8 * D, swz), qd0 = make_smem_desc(base + sm.q, 16, 8 * D, swz);
        const uint32_t rest = (uint32_t)(NP * D) >> 4;
        Ring kr, qr;
        int n = 0;
        bool ok = true;
        while (ok && next_segment(line, walk, seg)) {
            ok = wait(q_full, qr.parity, abort_flag);
            qr.next(1);
            for (int j = 0; ok && j < seg.T; ++j, ++n) {
                ok = wait(k_full(kr.idx), kr.parity, abort_flag);
                // S^T's buffer has been read, and (so that the softmax need not ask) the tile's P^T buffer
                const int s_before = n - (1 << sm.s_log2);
                if (s_before >= 0) ok = wait(p_full(s_before), round_of(s_before, sm.p_log2), abort_flag) && ok;
                if (n >> sm.p_log2) ok = wait(pv_done(n), round_of(n, sm.p_log2) ^ 1u, abort_flag) && ok;
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t kd = kd0 + (uint64_t)(kr.idx * (slot_bytes >> 4));
                    const uint32_t d = tm_s + place(n, sm.s_log2) * NP;
                    // q's leading bits, then the rest
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (c < 2 || D == 128) mma_f8_ss(d, kd + 2 * c, qd0 + 2 * c, idesc, c > 0);
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (c < 2 || D == 128) mma_f8_ss(d, kd + 2 * c, qd0 + (rest + 2 * c), idesc, 1);
                    mma_commit(s_full(n));
                    mma_commit(k_empty(kr.idx));
                }
                __syncwarp();
                kr.next(sm.ks);
            }
        }
        if (elect_one()) {
            mma_commit(drain_qk);
            wait_unconditional(drain_qk, 0);
        }
        __syncwarp();
    } else if (warp == 2) {
        // ------------------------------------------------------------ P.V issuer
        fewer_registers<kIssueRegs>();
        const uint32_t idesc = make_idesc_f16(128, NP, 1);
        const uint64_t pd0 = make_smem_desc(base + sm.p, 128, 2048, kSwizzleNone);
        Ring vr, orr;
        int n = 0;
        bool ok = true;
        while (ok && next_segment(line, walk, seg)) {
            if (n > 0) {
                ok = wait(o_free, orr.parity, abort_flag);     // the accumulators of the segment before have been read
                orr.next(1);
            }
            for (int j = 0, stream = 0; ok && j < seg.T; ++j, ++n) {
                ok = wait(vt_full(vr.idx), vr.parity, abort_flag) && ok;
                ok = wait(p_full(n), round_of(n, sm.p_log2), abort_flag) && ok;
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t pd = pd0 + (uint64_t)(place(n, sm.p_log2) * (NP * 256 >> 4));
                    const uint32_t d = tm_o + stream * NP;
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        mma_f16_ts(d, tm_v + vr.idx * 64 + c * 8, pd + (uint64_t)(c * 16), idesc, j >= kStreams || c > 0);
                    mma_commit(vt_free(vr.idx));
                    mma_commit(pv_done(n));
                }
                __syncwarp();
                vr.next(kVBufs);
                if (++stream == kStreams) stream = 0;
            }
        }
        if (elect_one()) {
            mma_commit(drain_pv);
            wait_unconditional(drain_pv, 0);
        }
        __syncwarp();
    } else if (warp >= kConvertWarp0 && warp < kSoftmaxWarp0) {
        // ------------------------------------------------- V codes to fp16 in tensor memory
        fewer_registers<kConvertRegs>();
        const int wq = warp & 3;                       // channels 32 wq .. + 31 = TMEM lanes
        const int set = (warp - kConvertWarp0) >> 2;   // tiles set, set + kVBufs, ... into V^T buffer `set`
        Ring vr;
        for (int i = 0; i < set; ++i) vr.next(sm.vs);
        uint32_t parity = 0;
        int n = 0;
        bool ok = 32 * wq < D;
        while (ok && next_segment(line, walk, seg)) {
            int j = (set - n) & (kVBufs - 1);
            n += seg.T;
#pragma unroll 1
            for (; j < seg.T; j += kVBufs) {
                // The buffer first (at once for the set's first tile): once the products of the tile two before have ended, every earlier tile has
                // been converted, so that the V slot's barrier cannot still be in the round before (with three slots that
                // round is the other set's, and loads may land in any order).
                ok = wait(vt_free(set), parity ^ 1u, abort_flag);
                ok = wait(v_full(vr.idx), vr.parity, abort_flag) && ok;
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const int live = seg.len - (seg.t0 + j) * kTilePos;      // positions of this tile below the length
                const int drafts = gamma > 1 ? live - gamma : kTilePos;  // the first that not all queries see
                uint32_t nan_at[2] = {0, 0};
                const uint32_t tile = base + sm.v + vr.idx * slot_bytes;
                // 16 channels x 64 positions a turn
                const uint32_t from = tile + lane * D, to = tm_v + set * 64 + ((uint32_t)(wq * 32) << 16);
                const int phase = D == 128 ? lane & 7 : (lane >> 1) & 3;
#pragma unroll 1
                for (int h = 0; h < 4; ++h) {
                    const int chunk = wq * 2 + (h & 1), half = h >> 1;
                    uint32_t r[2][4], w[16];
#pragma unroll
                    for (int u = 0; u < 2; ++u) ldmatrix_b8_x2(from + (half * 2 + u) * 32 * D + ((chunk ^ phase) << 4), r[u]);
                    if (__builtin_expect(min(live, drafts) < kTilePos, 0)) {
                        // What lies behind the sequence is not the cache's: it may be anything, NaN among it.  A NaN in a draft slot must
                        // not reach the queries that do not see it, and a zero probability times NaN would: it becomes zero here, and the
                        // softmax is told of the position.
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const int at = half * 64 + u * 32 + (k >> 1) * 16 + (lane & 3) * 4;
                                const int left = max(0, min(4, live - at)), before = max(0, min(4, drafts - at));
                                r[u][k] &= (uint32_t)((1ull << (8 * left)) - 1ull);
                                const uint32_t nan = __vcmpeq4(r[u][k] & 0x7F7F7F7Fu, 0x7F7F7F7Fu) & ~(uint32_t)((1ull << (8 * before)) - 1ull);
                                r[u][k] &= ~nan;
                                const uint32_t bits = (nan & 1u) | (nan >> 7 & 2u) | (nan >> 14 & 4u) | (nan >> 21 & 8u);
                                nan_at[u] |= bits << (at & 31);
                            }
                        if (h & 1) {
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                const uint32_t all = __reduce_or_sync(0xffffffffu, nan_at[u]);
                                if (lane == 0) nan_s[(set * 4 + wq) * 4 + half * 2 + u] = all;
                                nan_at[u] = 0;
                            }
                        }
                    }
                    // matrix m of a pair holds registers 2 m (row) and 2 m + 1 (row + 8)
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int k = 0; k < 4; ++k) decode4(r[u][k], w[u * 8 + k * 2], w[u * 8 + k * 2 + 1]);
                    tmem_st_16x256b_x4(to + half * 32 + ((uint32_t)((h & 1) * 16) << 16), w);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(v_empty(vr.idx));
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(vt_full(set));
                for (int i = 0; i < kVBufs; ++i) vr.next(sm.vs);
                parity ^= 1u;
            }
        }
    } else if (warp == 3) {
        // ------------------------------------------------- the blocks' scales, from global to shared memory
        fewer_registers<kIssueRegs>();
        // lanes 0..7 the K scales of a tile's blocks, 16..23 the V scales
        const int blk = lane & 15, in_tile = blk << p.block_log2;
        const float *from = lane < 16 ? p.k_scale : p.v_scale;
        int n = 0;
        bool ok = true;
        while (ok && next_segment(line, walk, seg)) {
            const int32_t *row = p.block_table + (size_t)seg.b * p.pages_per_seq;
            PageWalk at(p, seg.t0, min(in_tile, kTilePos - 1));
            int pos = seg.t0 * kTilePos + in_tile;
            const int stop = min(seg.len, (seg.t0 + seg.T) * kTilePos);
            // entry of the block table three tiles ahead, the scale itself two
            int e = -1, off = 0;
            float v0 = 0.f, v1 = 0.f;
#pragma unroll 1
            for (int j = -3; ok && j < seg.T; ++j) {
                if (j >= 0) {
                    const int before = n - (1 << sm.s_log2);
                    if (before >= 0) ok = wait(p_full(before), round_of(before, sm.p_log2), abort_flag);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    if (blk < 8) scale_s[place(n, sm.s_log2) * 16 + (lane >> 4) * 8 + blk] = v0;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(s_full(n));
                    ++n;
                }
                v0 = v1;
                v1 = e < 0 ? 0.f : from[((size_t)e * p.Hkv + seg.head) * p.blocks_per_page + (off >> p.block_log2)];
                e = in_tile < kTilePos && pos < stop ? row[at.page] : -1;
                if ((unsigned)e >= (unsigned)p.n_pages) e = -1;
                off = at.off;
                at.next_tile(p);
                pos += kTilePos;
            }
        }
    } else if (warp >= kSoftmaxWarp0) {
        // ------------------------------------------------------------ softmax
        more_registers<kSoftmaxRegs>();
        const int grp = (warp - kSoftmaxWarp0) >> 2, bar_id = 1 + grp;
        constexpr int kAll = 1 + kGroups;                       // barrier of all softmax threads
        constexpr int kBlock = block_of(kC);
        const int stream = grp / kShare, part = grp % kShare;
        const int wq = warp & 3, row = wq * 32 + lane;          // TMEM lane: position of the tile, channel of the output
        const int stid = tid - 32 * kSoftmaxWarp0, gtid = stid & 127;
        const uint32_t lane_addr = (uint32_t)(wq * 32) << 16;
        // this group's chunks of columns
        const int c_lo = part * kC, col0 = c_lo * 8;
        float *nm = nm_s + stream * NP + col0, *fac = fac_s + stream * NP + col0;
        float *tmx = reinterpret_cast<float *>(gbase + sm.tmx) + stream * 4 * NP + col0;
        float *my_sums = sums_s + (stream * 8 + wq) * NP + col0;            // + 4 NP: inside the span
        int n0 = 0;                                             // tiles of the segments before
        // No wait ends a loop here: a warp that left would leave its group at a barrier.  After a wait has run out all
        // others end at once, and what is computed then is void.
        while (true) {
            // one thread steps, the others read: what a segment is about is looked up again when it ends, not kept
            if (stid == 0) {
                if (!next_segment(line, walk, seg)) seg.T = 0;
                seg_s.b = seg.b;
                seg_s.head = seg.head;
                seg_s.t0 = seg.t0;
                seg_s.T = seg.T;
                seg_s.len = seg.len;
                seg_s.first = seg.first;
                seg_s.last = seg.last;
            }
            named_sync(kAll, kSoftmaxThreads);
            seg.T = seg_s.T;
            if (seg.T == 0) break;
            seg.b = seg_s.b;
            seg.head = seg_s.head;
            seg.t0 = seg_s.t0;
            const int L = seg_s.len;
            const int vis0 = p.span[2 * seg.b], vis1 = p.span[2 * seg.b + 1];

            // ---- q as two E4M3 operand tiles
            float scale;
            {
                const int per_log2 = D == 128 ? 4 : 3, n_chunks = NP << per_log2;          // chunks of eight channels
                const uint16_t *q = p.q + ((size_t)seg.b * gamma * p.Hq + seg.head * G) * D;
                auto load = [&](int ch) {
                    const int r = ch >> per_log2, c = ch & ((1 << per_log2) - 1);
                    if (ch >= n_chunks || r >= M) return make_uint4(0, 0, 0, 0);
                    const int g = div_by(r, G, P.group_magic), hg = r - g * G;
                    return *reinterpret_cast<const uint4 *>(q + ((size_t)g * p.Hq + hg) * D + c * 8);
                };
                // a thread's first two chunks (all of them up to 64 rows) stay in registers
                uint4 qv[2] = {load(stid), load(stid + kSoftmaxThreads)};
                uint32_t amax = 0;
                auto largest = [&](uint4 x) {
                    // (of either half, as integers: without their signs bf16 values order as their bits do)
                    const uint32_t a = __vmaxu2(__vmaxu2(x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu), __vmaxu2(x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu));
                    amax = max(amax, max(a & 0xFFFFu, a >> 16));
                };
                largest(qv[0]);
                largest(qv[1]);
#pragma unroll 1
                for (int ch = stid + 2 * kSoftmaxThreads; ch < n_chunks; ch += kSoftmaxThreads) largest(load(ch));
                amax = __reduce_max_sync(0xffffffffu, amax);
                if (lane == 0) wmax_s[warp - kSoftmaxWarp0] = amax;
                named_sync(kAll, kSoftmaxThreads);
                amax = __reduce_max_sync(0xffffffffu, lane < 4 * kGroups ? wmax_s[lane] : 0u);
                if (__builtin_expect(amax >= 0x7F80u, 0)) {
                    // NaN or Inf: its row's results are NaN, and the others are scaled by what is finite
                    amax = 0;
#pragma unroll 1
                    for (int ch = stid; ch < n_chunks; ch += kSoftmaxThreads) {
                        const uint4 x = load(ch);
                        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const uint32_t a = (w[k >> 1] >> (16 * (k & 1))) & 0x7FFFu;
                            if (a < 0x7F80u) amax = max(amax, a);
                        }
                    }
                    amax = __reduce_max_sync(0xffffffffu, amax);
                    named_sync(kAll, kSoftmaxThreads);
                    if (lane == 0) wmax_s[warp - kSoftmaxWarp0] = amax;
                    named_sync(kAll, kSoftmaxThreads);
                    amax = __reduce_max_sync(0xffffffffu, lane < 4 * kGroups ? wmax_s[lane] : 0u);
                }
                // the power of two that brings the largest magnitude into [128, 256); bf16's own range keeps it above 2^-121, and a
                // largest magnitude below 2^-119 is brought as far as one power goes
                int shift = 0;
                if (amax > 0) shift = min(126, 7 - ((int)(amax >> 7) - 127));
                const float up = pow2(shift);
                scale = p.scale_log2 * pow2(-shift);
#pragma unroll 1
                for (int ch = stid, u = 0; ch < n_chunks; ch += kSoftmaxThreads, ++u) {
                    const uint4 x = u == 0 ? qv[0] : u == 1 ? qv[1] : load(ch);
                    const int r = ch >> per_log2, c = ch & ((1 << per_log2) - 1);
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
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
            for (int c = lane; c < kC * 8; c += 32) my_sums[c] = my_sums[4 * NP + c] = 0.f;
            bool l_in = false;                          // l holds sums of positions inside the span
            int k0 = 0;                                 // V scales are taken relative to 2^k0
            float inv_k0 = 1.f;

            // adds what the threads hold to the warp's sums
            auto add_to_sums = [&](int c, float t, bool all, bool in) {
                if (lane & 3) return;
                float *at = my_sums + c * 8 + ((lane >> 4) & 1) * 4 + ((lane >> 3) & 1) * 2 + ((lane >> 2) & 1);
                if (all) *at += t;
                if (in) at[4 * NP] += t;
            };
            const int j_first = stream;
            int last = -1;                              // this stream's last tile
#pragma unroll 1
            for (int j = j_first;; j += kStreams) {
                // sums of one kind at a time: a tile inside the span, or another (what one of both has inside is added below)
                const int pos0 = (seg.t0 + j) * kTilePos, pos = pos0 + row;
                const bool inside = pos0 >= vis0 && pos0 + kTilePos <= vis1;
                if (__builtin_expect(inside != l_in || j >= seg.T, 0)) {
#pragma unroll
                    for (int c = 0; c < kC; ++c)
                        add_to_sums(c, warp_sums(l + c * 8, lane), true, l_in);
#pragma unroll
                    for (int k = 0; k < kC * 8; ++k) l[k] = 0.f;
                    __syncwarp();
                    l_in = inside;
                    if (j >= seg.T) break;
                }
                const int n = n0 + j;
                const bool tail = pos0 + kTilePos > L - gamma;        // some query does not see some position
                const bool begins = j == j_first;
                const uint32_t s_addr = tm_s + place(n, sm.s_log2) * NP + lane_addr + col0;

                wait(s_full(n), round_of(n, sm.s_log2), abort_flag);
                __syncwarp();
                tc_fence_after();
                const float *sc = scale_s + place(n, sm.s_log2) * 16 + (row >> p.block_log2);
                const float ck = scale * sc[0];
                float vs = sc[8];
                const int ve = (int)((__float_as_uint(vs) >> 23) & 0xFFu) - 127;
                if (__builtin_expect(begins, 0)) {
                    // the first tile's maxima set the references (below)
                    if (gtid < kC * 8) nm[gtid] = 0.f;
                    named_sync(bar_id, 128);
                }
                if (__builtin_expect(tail, 0) && gamma > 1) {
                    // is V NaN in this draft slot?
                    // The V^T buffer's round must be this tile's or the one before it for the wait to tell them apart: the products of the
                    // tile that had the buffer before have ended, and the next to have it waits for this tile's.
                    if (n >= kVBufs) wait(pv_done(n - kVBufs), round_of(n - kVBufs, sm.p_log2), abort_flag);
                    wait(vt_full(n & (kVBufs - 1)), (uint32_t)(n / kVBufs) & 1u, abort_flag);
                    __syncwarp();
                    const uint32_t *at = nan_s + (n & (kVBufs - 1)) * 16 + wq;
                    if (((at[0] | at[4] | at[8] | at[12]) >> lane) & 1u) vs = __int_as_float(0x7FFFFFFF);
                }
                uint8_t *prow = gbase + sm.p + place(n, sm.p_log2) * (NP * 256) + c_lo * 2048 + row * 16;
                const Seen seen = tail ? seen_by(pos - (L - gamma), G, gamma, p.branch_len) : Seen{0, 0xFFFFFFFFu};
                // A stream's first tile sets its references: to the tile's maxima, 2^kFirst below the largest probability.  They move when
                // a score of a later tile passes the guard or a V scale is large against 2^k0: the tile's pass is taken back and made
                // again.
                bool move = begins, back = false;
#pragma unroll 1
                for (int turn = 0;;) {
                    if (!move) {
                        const float vsr = vs * inv_k0, sign = back ? -1.f : 1.f;
                        const float top = __builtin_expect(!tail, 1)
                                              ? softmax_pass<kC, kBlock, false>(s_addr, nm, ck, vsr, seen, col0, prow, sign, l)
                                              : softmax_pass<kC, kBlock, true>(s_addr, nm, ck, vsr, seen, col0, prow, sign, l);
                        if (!back) {
                            // (all of the group's P^T is on its way to the tensor core when the vote is over)
                            tc_fence_before();
                            fence_proxy_async_smem();
                            if (__builtin_expect(!group_any(bar_id, top > kGuard || (ve > k0 && ve < 100)) || turn == 3, 1)) break;
                            back = true;
                            ++turn;
                            continue;
                        }
                    }
                    // ---- references up to this tile's maxima over the lanes (the sums are without this tile)
                    int e = __reduce_max_sync(0xffffffffu, ve < 128 ? min(ve, 100) : -127);
                    const References refs(nm);
#pragma unroll 1
                    for (int c = 0; c < kC; ++c) {
                        uint32_t r[8];
                        tmem_ld_x8(s_addr + c * 8, r);
                        tmem_wait_ld();
                        float x[8];
                        scores8<true>(r, refs, c * 8, ck, seen, col0 + c * 8, x);
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float y = warp_max_f32(x[k]);
                            if (lane == 0) tmx[wq * NP + c * 8 + k] = y;
                        }
                    }
                    if (lane == 0) wmax_s[warp - kSoftmaxWarp0] = (uint32_t)(e + 127);
                    named_sync(bar_id, 128);
                    e = max(-100, (int)__reduce_max_sync(0xffffffffu, wmax_s[grp * 4 + (lane & 3)]) - 127);
                    const int k_new = begins && turn == 0 ? e + 2 : e > k0 ? e + 2 : k0;
                    if (gtid < kC * 8) {
                        const float t = fmaxf(fmaxf(tmx[gtid], tmx[NP + gtid]), fmaxf(tmx[2 * NP + gtid], tmx[3 * NP + gtid]));
                        const float up = (begins ? t > -INFINITY : t > kGuard) ? t - kFirst : 0.f;
                        nm[gtid] -= up;
                        fac[gtid] = ex2(-up);
                    }
                    named_sync(bar_id, 128);
                    if (!begins) {
                        const float fk = pow2(max(k0 - k_new, -126));
#pragma unroll
                        for (int k = 0; k < kC * 8; ++k) {
                            // (NaN: the tile had brought an infinity, against which what was there before does not count)
                            l[k] = l[k] == l[k] ? l[k] * fac[k] : 0.f;
                        }
                        // (the products of the stream's last tile have ended; the next are those of this one)
                        wait(pv_done(last), round_of(last, sm.p_log2), abort_flag);
                        __syncwarp();
                        tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < kC; ++c) {
                            const uint32_t o_addr = tm_o + stream * NP + lane_addr + col0 + c * 8;
                            uint32_t o[8];
                            tmem_ld_x8(o_addr, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int k = 0; k < 8; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * (fac[c * 8 + k] * fk));
                            tmem_st_x8(o_addr, o);
                        }
                        tmem_wait_st();
                        for (int c = lane; c < kC * 8; c += 32) {
                            my_sums[c] *= fac[c];
                            my_sums[4 * NP + c] *= fac[c];
                        }
                        __syncwarp();
                    } else if (turn > 0) {
#pragma unroll
                        for (int k = 0; k < kC * 8; ++k) l[k] = 0.f;
                    }
                    k0 = k_new;
                    inv_k0 = pow2(-k0);
                    move = back = false;
                }
                if (__builtin_expect(!inside && pos0 + kTilePos > vis0 && pos0 < vis1, 0)) {
                    const bool in = pos >= vis0 && pos < vis1;
#pragma unroll 1
                    for (int c = 0; c < kC; ++c) {
                        uint32_t r[8];
                        tmem_ld_x8(s_addr + c * 8, r);
                        tmem_wait_ld();
                        float x[8];
                        scores8<true>(r, References(nm), c * 8, ck, seen, col0 + c * 8, x);
#pragma unroll
                        for (int k = 0; k < 8; ++k) x[k] = in ? ex2(x[k]) : 0.f;
                        add_to_sums(c, warp_sums(x, lane), false, true);
                    }
                    tc_fence_before();
                    named_sync(bar_id, 128);            // (S^T has been read once more)
                }
                if (gtid == 0) mbar_arrive(p_full(n));
                last = n;
            }
            n0 += seg.T;
            if (last >= 0) wait(pv_done(last), round_of(last, sm.p_log2), abort_flag);
            __syncwarp();
            tc_fence_after();
            if (gtid == 0) wmax_s[4 * kGroups + grp] = (uint32_t)(k0 + 1024);
            named_sync(kAll, kSoftmaxThreads);             // all sums are there

            // ---- a row's weights: each stream's part of the sum, in fac_s
            seg.b = seg_s.b;
            seg.head = seg_s.head;
            const bool whole = seg_s.first && seg_s.last;
            const int slot = part_slot(blockIdx.x, seg_s.first);
            float *part_o = p.part_o + (size_t)slot * M * D;
            if (stid < M) {
                const int col = stid;
                float all[kStreams], in[kStreams], m[kStreams], top = -INFINITY;
#pragma unroll
                for (int u = 0; u < kStreams; ++u) {
                    const float *t = sums_s + u * 8 * NP + col;
                    in[u] = t[4 * NP] + t[5 * NP] + t[6 * NP] + t[7 * NP];
                    all[u] = t[0] + t[NP] + t[2 * NP] + t[3 * NP];
                    m[u] = -nm_s[u * NP + col];
                    if (all[u] != 0.f) top = fmaxf(top, m[u]);
                }
                float total = 0.f, vis = 0.f, w[kStreams];
#pragma unroll
                for (int u = 0; u < kStreams; ++u) {
                    w[u] = all[u] != 0.f ? ex2(m[u] - top) : 0.f;     // (a stream without tiles, or that the row sees nothing of)
                    if (w[u] != 0.f) {
                        total = fmaf(w[u], all[u], total);
                        vis = fmaf(w[u], in[u], vis);
                    }
                }
                const float inv = total == 0.f ? 0.f : 1.f / total;   // a query that sees nothing gives zeros
#pragma unroll
                for (int u = 0; u < kStreams; ++u) {
                    const int g_of = u * kShare + col / (8 * kC);       // the group of this stream that has the column
                    fac_s[u * NP + col] = (whole ? w[u] * inv : w[u]) * pow2((int)wmax_s[4 * kGroups + g_of] - 1024);
                }
                const int g = div_by(col, G, P.group_magic), hg = col - g * G;
                const int out_row = (seg.b * gamma + g) * p.Hq + seg.head * G + hg;
                row_s[col] = out_row;
                if (whole) {
                    p.mass[out_row] = vis * inv;
                } else {
                    *reinterpret_cast<float4 *>(p.part_stat + ((size_t)slot * M + col) * 4) = make_float4(top, total, vis, 0.f);
                }
            }
            named_sync(kAll, kSoftmaxThreads);
            // ---- results: whole, or this CTA's part of them; the chunks of columns go to the groups in turn
            if (row < D) {
#pragma unroll 1
                for (int c = grp; c * 8 < M; c += kGroups) {
                    float v[8] = {};
#pragma unroll
                    for (int u = 0; u < kStreams; ++u) {
                        uint32_t o[8];
                        tmem_ld_x8(tm_o + u * NP + lane_addr + c * 8, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float w = fac_s[u * NP + c * 8 + k];
                            v[k] = w != 0.f ? fmaf(w, __uint_as_float(o[k]), v[k]) : v[k];
                        }
                    }
                    if (whole) {
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (c * 8 + k < M) p.out[(size_t)row_s[c * 8 + k] * D + row] = (uint16_t)(pack_bf16x2(v[k], 0.f) & 0xFFFFu);
                    } else {
                        float *to = part_o + c * 8 * D + row;
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (c * 8 + k < M) to[k * D] = v[k];
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(o_free);
            named_sync(kAll, kSoftmaxThreads);             // sums, references and q may be written anew
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
// Rows of empty sequences are written as zeros here.  All latency (40 rows of 8 heads, 19 parts each: 3.1 MB from L2): the first
// sixteen parts are asked for together with the statistics that say what they weigh.
template <int D>
__global__ void __launch_bounds__(32 * kMergeWarps) merge_paged_fp8_kernel(const PagedFp8Params p, const uint32_t group_magic)
{
    constexpr int kEach = D / 32, kAhead = 16;
    using Vec = typename std::conditional<D == 128, float4, float2>::type;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int row = blockIdx.x * kMergeWarps + warp;
    const int b = row / (p.gamma * p.Hq), r = row - b * p.gamma * p.Hq, g = r / p.Hq, h = r - g * p.Hq;
    const int head = div_by(h, p.G, group_magic), col = g * p.G + h - head * p.G;
    grid_launch_dependents();
    grid_dependency_wait();
    if (b >= p.B) return;
    const int2 cut = *reinterpret_cast<const int2 *>(p.line), seq = *reinterpret_cast<const int2 *>(p.line + 2 + 2 * b);
    const int share = cut.x, tiles = tiles_of(seq.y);
    float acc[kEach] = {};
    float total = 0.f, vis = 0.f;
    if (tiles > 0) {
        const int first = seq.x + head * (cut.y ? (tiles + share - 1) / share * share : tiles);
        const int c0 = first / share, n = (first + tiles - 1) / share - c0 + 1;
        if (n == 1) return;                             // that CTA has finished the pair itself
        auto at = [&](int u) { return (size_t)part_slot(c0 + u, u == 0) * p.M + col; };
        auto values = [&](int u) { return *reinterpret_cast<const Vec *>(p.part_o + at(u) * D + lane * kEach); };
        auto stat = [&](int u) { return u < n ? *reinterpret_cast<const float4 *>(p.part_stat + at(u) * 4) : make_float4(0.f, 0.f, 0.f, 0.f); };
        const float4 mine = stat(lane);
        Vec v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (u < n) v[u] = values(u);
        float top = mine.y != 0.f ? mine.x : -INFINITY;
        for (int u = 32 + lane; u < n; u += 32) {
            const float4 s = stat(u);
            if (s.y != 0.f) top = fmaxf(top, s.x);
        }
        top = warp_max_f32(top);
        float wl = 0.f, wv = 0.f;
        for (int u0 = 0; u0 < n; u0 += 32) {
            const float4 s = u0 == 0 ? mine : stat(u0 + lane);
            const float w = s.y != 0.f ? ex2(s.x - top) : 0.f;      // (a part that the row sees nothing of counts for nothing)
            wl = fmaf(w, s.y, wl);
            wv = fmaf(w, s.z, wv);
            for (int u1 = 0; u1 < 32 && u0 + u1 < n; u1 += kAhead) {
                if (u0 + u1 > 0)
#pragma unroll
                    for (int u = 0; u < kAhead; ++u)
                        if (u0 + u1 + u < n) v[u] = values(u0 + u1 + u);
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const float wu = __shfl_sync(0xffffffffu, w, u1 + u);
                    if (wu == 0.f) continue;            // (beyond the last part too)
                    const float *f = reinterpret_cast<const float *>(&v[u]);
#pragma unroll
                    for (int k = 0; k < kEach; ++k) acc[k] = fmaf(wu, f[k], acc[k]);
                }
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            wl += __shfl_xor_sync(0xffffffffu, wl, o);
            wv += __shfl_xor_sync(0xffffffffu, wv, o);
        }
        total = wl;
        vis = wv;
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    uint16_t *out = p.out + (size_t)row * D + lane * kEach;
#pragma unroll
    for (int k = 0; k < kEach; k += 2)
        *reinterpret_cast<uint32_t *>(out + k) = pack_bf16x2(acc[k] * inv, acc[k + 1] * inv);
    if (lane == 0) p.mass[row] = vis * inv;
}

// A page pool as [pages][heads][positions][channels]; a box is a tile of one page and head, or all of a shorter page.
bool make_pool_map(CUtensorMap *map, const uint8_t *pool, const PagedFp8Params &p)
{
    const EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)p.D, (cuuint64_t)p.page_size, (cuuint64_t)p.Hkv, (cuuint64_t)p.n_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)p.position_stride, (cuuint64_t)p.head_stride, (cuuint64_t)p.page_stride};
    const cuuint32_t box[4] = {(cuuint32_t)p.D, (cuuint32_t)(p.page_size < kTilePos ? p.page_size : kTilePos), 1, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<uint8_t *>(pool), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, p.D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kStreams, int kC>
cudaError_t launch_attention(const KernelParams &P, const CUtensorMap &tk, const CUtensorMap &tv, cudaStream_t stream, int *launches)
{
    const auto kernel = attn_paged_fp8_kernel<kStreams, kC>;
    const size_t smem = P.sm.total + 1024;
    cudaError_t e = allow_shared_memory(kernel);
    if (e != cudaSuccess) return e;
    return launch_after(kernel, dim3((unsigned)P.a.n_cta), kThreads, smem, P.a.pdl != 0, stream, launches, P, tk, tv);
}

}  // namespace

size_t paged_fp8_scratch_bytes(int n_cta, int M, int D)
{
    return (size_t)2 * n_cta * M * (D + 4) * sizeof(float) + (2 + 2 * LVSPEC_MAX_BATCH) * sizeof(int32_t);
}

cudaError_t launch_attn_paged_fp8(const PagedFp8Params &p, const uint8_t *k_pool, const uint8_t *v_pool, cudaStream_t stream,
                                  int *launches)
{
    KernelParams P;
    P.a = p;
    const int n8 = p.M > 96 ? (p.M + 15) / 16 * 2 : (p.M + 7) / 8;      // chunks of eight columns
    P.NP = (n8 + 1) / 2 * 16;
    // Two streams where tensor memory holds the accumulators of both beside 2 x 64 columns of V^T and two S^T buffers.  (Four streams up
    // to 32 rows and three up to 48, of a group each, with fewer registers a thread: 16 sequences of 9500 to 32000 positions, 8 heads,
    // 8 rows 113 us against 112, 32 rows 127 against 118, 40 rows 152 against 141, 48 rows 145 against 141.)
    const int streams = P.NP <= 96 ? 2 : 1;
    const int s_log2 = kVBufs * 64 + (streams + 4) * P.NP <= 512 ? 2 : 1, p_log2 = P.NP <= 96 ? 2 : 1;
    // (a group's wait for its S^T buffer's next round must find the round before ended)
    if (streams > 1 << s_log2) return cudaErrorInvalidValue;
    int cols = 32;
    while (cols < kVBufs * 64 + (streams + (1 << s_log2)) * P.NP) cols *= 2;
    P.tmem_cols = cols;
    P.group_magic = p.G > 1 ? 0xFFFFFFFFu / (uint32_t)p.G + 1u : 0u;
    // as many slots as shared memory holds, K's one more where the count is odd (its tile is used first)
    int slots = 12;
    do P.sm = smem_map(p.D, P.NP, streams, (slots + 1) / 2, slots / 2, s_log2, p_log2);
    while (P.sm.total + 1024 > 227 * 1024 && --slots > 4);
    if (P.sm.total + 1024 > 227 * 1024) return cudaErrorInvalidValue;        // (six at 128 rows)
    CUtensorMap tk, tv;
    if (!make_pool_map(&tk, k_pool, p) || !make_pool_map(&tv, v_pool, p)) return cudaErrorInvalidValue;
    cudaError_t e;
    switch (n8) {
        case 1: e = launch_attention<2, 1>(P, tk, tv, stream, launches); break;
        case 2: e = launch_attention<2, 2>(P, tk, tv, stream, launches); break;
        case 3: e = launch_attention<2, 3>(P, tk, tv, stream, launches); break;
        case 4: e = launch_attention<2, 4>(P, tk, tv, stream, launches); break;
        case 5: e = launch_attention<2, 5>(P, tk, tv, stream, launches); break;
        case 6: e = launch_attention<2, 6>(P, tk, tv, stream, launches); break;
        case 7: e = launch_attention<2, 7>(P, tk, tv, stream, launches); break;
        case 8: e = launch_attention<2, 8>(P, tk, tv, stream, launches); break;
        case 9: e = launch_attention<2, 9>(P, tk, tv, stream, launches); break;
        case 10: e = launch_attention<2, 10>(P, tk, tv, stream, launches); break;
        case 11: e = launch_attention<2, 11>(P, tk, tv, stream, launches); break;
        case 12: e = launch_attention<2, 12>(P, tk, tv, stream, launches); break;
        case 14: e = launch_attention<1, 7>(P, tk, tv, stream, launches); break;
        default: e = launch_attention<1, 8>(P, tk, tv, stream, launches); break;
    }
    if (e != cudaSuccess) return e;
    const int rows = p.B * p.gamma * p.Hq;
    const dim3 grid((unsigned)((rows + kMergeWarps - 1) / kMergeWarps));
    return p.D == 128 ? launch_after(merge_paged_fp8_kernel<128>, grid, 32 * kMergeWarps, 0, p.pdl != 0, stream, launches, p, P.group_magic)
                      : launch_after(merge_paged_fp8_kernel<64>, grid, 32 * kMergeWarps, 0, p.pdl != 0, stream, launches, p, P.group_magic);
}

}  // namespace lvspec
