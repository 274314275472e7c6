// Sampling from logits by temperature, top-k, top-p and min-p, from one given uniform number per row.
//
// With M the row's largest logit and T the temperature, token i has weight w_i = exp((l_i - M) / T).  In the
// order of falling logits (equal ones by rising index) every filter keeps a prefix: top-k its first k, top-p the
// shortest prefix of those with at least the share p of their weight, min-p the logits at or above
// M + T ln(min_p).  Of what the shortest prefix keeps, taken in index order again, the token is the first whose
// running sum exceeds u times the whole.
//
// Weights are integers, 2^40 for the largest: log2(e) (l_i - M) / T with its rounding errors carried, 2^x of its fraction to 2^-22.
// Sums of integers do not depend on their order, so a row gives the same token however it is cut up.
//
// A row is read once, by a cluster of up to eight CTAs that keep it in their shared memory (a vocabulary of 152 K is 76 KB
// each, two CTAs an SM) and pass sums on through distributed shared memory.  A boundary is found without sorting: a histogram over
// (M - l) in steps of T / 64 or T / 128, then the tokens of the bin that holds the boundary are ranked by comparing all with all (more
// than 160 by the CTAs together); a bin with more than 1024 tokens (equal or nearly equal logits, or the last one, which has no end) is
// cut into bins of the logits' bit patterns until it fits or holds a single value.  Top-p's bin is chosen by the bins' counts and the weights of their
// middles; it is ranked together with the bins beside it by exact sums, or put right step by step if it is not among them.  Once a
// boundary's bin is known each warp lists its tokens up to it, and what follows goes over the lists.
//
// Not HBM bounds it: with many rows a row's load (a CTA has nothing else to do meanwhile, and an SM one other CTA), and for all the
// exchanges, a cluster barrier each (two without top-k and top-p, five or six with one of them, seven to nine with both, four
// more for each cut of a bin), and the passes over shared memory.
// 128 rows of 152064 in fp32, us: greedy 41, no filter 67, min-p 47, top-k 76, top-p 0.9 145, 0.99 at T = 1.2 248; one row: 6, 9, 8,
// 13, 22, 38.  At T = 0.1 top-k 50 ends in the last bin, where most of the row is: with top-p 0.9 198 us and 28 (117 and 20 at
// T = 0.8).  With the bins beside the boundary's only, large vocabularies take 10 % less and rows with few tokens a bin, which then
// settle step by step, three times as long (2 rows of 3422, top-k and top-p: 52 us instead of 17).  Sixteen CTAs a row, three an SM,
// take 50 to 90 % longer with 32 rows or more, and win with few: the barrier's cost against the passes'.
#include <cfloat>

#include "lvspec_internal.h"
#include "sm100_ptx.cuh"

namespace lvspec {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048;
constexpr int kCandidates = 1024;       // tokens that are ranked directly
constexpr int kRankAlone = 160;         // up to so many each CTA ranks all, beyond they share the work
constexpr int kListed = 2 * kBins / kWarps;         // tokens in a warp's list
constexpr int kMaxCluster = 16;
typedef unsigned long long u64;

// ---- cluster -----------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// Shared memory of another CTA may be written once that CTA is known to run: each says so as it starts, and waits for the others
// ahead of its first store to them.  (Nothing else is handed over by this.)
__device__ __forceinline__ void cluster_here() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_all_here() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_address(uint32_t smem, uint32_t rank)
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem), "r"(rank));
    return a;
}
__device__ __forceinline__ void st_peer(uint32_t a, u64 x) { asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(x) : "memory"); }
__device__ __forceinline__ uint32_t add_peer(uint32_t a, uint32_t x)
{
    uint32_t old;
    asm volatile("atom.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(old) : "r"(a), "r"(x) : "memory");
    return old;
}
__device__ __forceinline__ u64 ld_peer(uint32_t a)
{
    u64 x;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(x) : "r"(a) : "memory");
    return x;
}

// Order of logits as that of unsigned integers, and back.
__device__ __forceinline__ uint32_t key_of(float l)
{
    const uint32_t b = __float_as_uint(l);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }

// 2^40 2^(n + f) rounded down, n the low bits of t = n + 1.5 * 2^23: 2^f's 24 bits shifted into place.
__device__ __forceinline__ u64 weight_of(float t, float f)
{
    const uint32_t e = __float_as_uint(ptx::ex2(f));
    const uint32_t m = (e & 0x7FFFFFu) | 0x800000u;
    const int down = 127 - (int)(e >> 23) - (int)(__float_as_uint(t) - 0x4B400000u);        // m << 17 >> down
    u64 w;
    asm("shr.u64 %0, %1, %2;" : "=l"(w) : "l"((u64)m << 17), "r"(down));        // (nothing is left of shifts by 64 and more)
    return w;
}
constexpr float kNearestInt = 12582912.f;           // 1.5 * 2^23: added and taken off again it rounds to an integer
// For any top and T, c = log2(e) / T (its two halves): of fp32 numbers neither 1 / T nor the difference passes the range of fp64.
__device__ __noinline__ u64 weight_anywhere(float l, float top, int c_hi, int c_lo)
{
    const double c = __hiloint2double(c_hi, c_lo);
    if (!(l > -INFINITY)) return 0;             // (nothing even where T is infinite)
    const double y = ((double)l - (double)top) * c;
    if (!(y > -42.0)) return 0;
    const double n = rint(y);
    return weight_of((float)n + kNearestInt, (float)(y - n));
}
struct Weight {
    float top;                  // the row's largest logit, finite
    float per, per_rest;        // log2(e) / T in two parts
    float lowest;               // logits below this count as it: their weight is nothing
    float at_top, at_top_rest;  // top log2(e) / T in two parts; where T is not usual the halves of log2(e) / T as a double
    bool usual;
    __device__ __forceinline__ void set(float top_, float T)
    {
        top = top_;
        const double c = 1.4426950408889634 / (double)T, ct = c * (double)top;
        per = (float)c;
        per_rest = (float)(c - (double)per);            // (of use where 1 / T is in the range of fp32)
        lowest = top - 45.f * T;                    // 2^40 exp(-45) is below 1
        // The first part has so few bits that it is still exact with an integer down to -66 added.
        usual = fabs(ct) < 1048576.0 && T > 1e-30f && T < 1e30f;
        double grain = 1.52587890625e-05;
        while (usual && fabs(ct) >= 16777216.0 * grain - 66.0) grain *= 2;
        at_top = (float)(rint(ct / grain) * grain);
        at_top_rest = (float)(ct - (double)at_top);
        if (!usual) {
            at_top = __int_as_float(__double2hiint(c));
            at_top_rest = __int_as_float(__double2loint(c));
        }
    }
    // floor(2^40 exp((l - top) / T)), 2^x of the fraction good to 2^-22
    __device__ __forceinline__ u64 operator()(float l) const
    {
        if (__builtin_expect(!usual, 0)) return weight_anywhere(l, top, __float_as_int(at_top), __float_as_int(at_top_rest));
        l = fmaxf(l, lowest);
        const float t = fmaf(l, per, -at_top) + kNearestInt;
        const float f = fmaf(l, per, -(at_top + (t - kNearestInt))) + fmaf(l, per_rest, -at_top_rest);
        return weight_of(t, f);
    }
};

// A place in the order of falling logits, equal ones by rising index.
struct Place {
    uint32_t key;
    int index;
    __device__ __forceinline__ bool reaches(uint32_t k, int i) const { return k > key || (k == key && i <= index); }
};

struct Shared {
    u64 box[2][kMaxCluster][4];         // what the CTAs tell one another, two rounds by turns
    u64 warp_val[3][kWarps];
    union {
        uint32_t bins[kBins];           // a histogram of this CTA's tokens
        uint16_t list[kWarps][kListed]; // later the places of those that may be kept, each warp's in its order
    };
    uint32_t all_bins[kBins];           // the histogram of the whole row, for as long as the row is worked on
    union {
        struct {
            u64 cand[kCandidates], cand_weight[kCandidates];    // key and index of a bin's tokens; their weights
        };
        struct {
            uint32_t cut[kBins], all_cut[kBins];                // while a bin has too many: histograms of it, likewise
        };
    };
    u64 cum;
    int bin, around[4], n_cand, answer, row;
    u64 place, found;                   // a place as one word (key above, index below); is there one
};

struct Row {
    Shared &s;
    const float *v;                     // this CTA's logits, v[0 .. n); before and behind them, to 16-byte borders, -inf
    int n, first, pad;                  // first: the index of v[0]; pad: logits from the first border to v[0]
    int g0, g1;                         // the warp's share of them: groups of four from the first border
    int listed;                         // tokens in the warp's list; -1: it has none, passes go over its share
    int n_cta, rank, turn;
    Weight weight;
    float bins_per, bin_step;           // bins to a logit's difference, and its inverse

    __device__ __forceinline__ Row(Shared &s_) : s(s_), listed(-1), turn(0) {}

    // f(logit, its place in v) for the warp's logits (-inf among them), or those of its list
    template <typename F>
    __device__ __forceinline__ void for_each(F f) const
    {
        const int lane = threadIdx.x & 31;
        if (listed >= 0) {
            const uint16_t *list = s.list[threadIdx.x >> 5];
#pragma unroll 1
            for (int e = lane; e < listed; e += 32) {
                const int i = list[e];
                f(v[i], i);
            }
            return;
        }
        const float4 *g4 = reinterpret_cast<const float4 *>(v - pad);
#pragma unroll 1
        for (int g = g0 + lane; g < g1; g += 32) {
            const float4 x = g4[g];
            const float l[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) f(l[k], g * 4 + k - pad);
        }
    }
    // Lists the warp's logits from `least` on, in their order.  A warp with more than it has room for goes on without a list.  (The
    // bins are the lists' memory: no CTA may need them any more.)
    __device__ void make_list(float least)
    {
        if (!(least > -INFINITY)) return;
        const int lane = threadIdx.x & 31;
        uint16_t *list = s.list[threadIdx.x >> 5];
        const float4 *g4 = reinterpret_cast<const float4 *>(v - pad);
        const uint32_t below = (1u << lane) - 1u;
        int m = 0;
#pragma unroll 1
        for (int g = g0; g < g1; g += 32) {
            const float4 x = g + lane < g1 ? g4[g + lane] : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            const float l[4] = {x.x, x.y, x.z, x.w};
            if (!__any_sync(0xffffffffu, fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])) >= least)) continue;
            int at = m, all = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t has = __ballot_sync(0xffffffffu, l[k] >= least);
                at += __popc(has & below);
                all += __popc(has);
            }
            if (m + all > kListed) return;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (l[k] >= least) list[at++] = (uint16_t)((g + lane) * 4 + k - pad);
            m += all;
        }
        __syncwarp();
        listed = m;
    }
    // No logit of bins 0 .. bin is below this.
    __device__ __forceinline__ float least_of(int bin) const { return bin < kBins - 1 ? weight.top - (float)(bin + 1) * bin_step : -INFINITY; }

    // Sums (op 0), or largest values (op 1), of kN numbers per thread over the row; every CTA's in box[slot].
    template <int kN>
    __device__ int gather(u64 a, u64 b, u64 c, int op)
    {
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
        u64 x[3] = {a, b, c};
#pragma unroll
        for (int k = 0; k < kN; ++k) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const u64 y = __shfl_xor_sync(0xffffffffu, x[k], o);
                x[k] = op ? (y > x[k] ? y : x[k]) : x[k] + y;
            }
            if (lane == 0) s.warp_val[k][warp] = x[k];
        }
        __syncthreads();
        const int slot = turn & 1;
        ++turn;
        if (warp == 0) {
#pragma unroll
            for (int k = 0; k < kN; ++k) {
                u64 t = lane < kWarps ? s.warp_val[k][lane] : 0;
#pragma unroll
                for (int o = kWarps / 2; o > 0; o >>= 1) {
                    const u64 y = __shfl_xor_sync(0xffffffffu, t, o);
                    t = op ? (y > t ? y : t) : t + y;
                }
                if (lane < n_cta) st_peer(peer_address(ptx::smem_u32(&s.box[slot][rank][k]), lane), t);
            }
        }
        cluster_sync();
        return slot;
    }
    __device__ u64 of_all(int slot, int k, int op)
    {
        u64 t = 0;
        int r = 0;
        for (; r + 4 <= n_cta; r += 4) {
            u64 y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = s.box[slot][r + j][k];
#pragma unroll
            for (int j = 0; j < 4; ++j) t = op ? (y[j] > t ? y[j] : t) : t + y[j];
        }
        for (; r < n_cta; ++r) {
            const u64 y = s.box[slot][r][k];
            t = op ? (y > t ? y : t) : t + y;
        }
        return t;
    }
    // The nearest bin to (top - l) bins_per; it falls as l rises, whatever the rounding.  Counting and looking for a bin's tokens
    // have to round alike, so the product and the sum are written as operations that the compiler may not join into one.
    __device__ __forceinline__ float in_bins(float l) const { return __fmul_rn(weight.top - l, bins_per); }
    __device__ __forceinline__ int nearest_bin(float t) const
    {
        return (int)(__float_as_uint(__fadd_rn(t, kNearestInt)) - 0x4B400000u);         // (the integer is in the low bits)
    }
    __device__ __forceinline__ int bin_of(float l) const { return nearest_bin(fminf(in_bins(l), (float)(kBins - 1))); }
    // Counts a logit in its bin; those of the last one (they have no end: most of a peaked row is there, and all at one counter would
    // wait for one another) in `in_last`.
    __device__ __forceinline__ void count(float l, uint32_t &in_last)
    {
        const float t = in_bins(l);
        if (t < (float)(kBins - 1) - 0.75f)
            asm volatile("red.shared.add.u32 [%0], 1;" ::"r"(ptx::smem_u32(s.bins) + 4u * (uint32_t)nearest_bin(t)) : "memory");
        else if (l > -INFINITY) {
            const int b = bin_of(l);
            if (b < kBins - 1) atomicAdd(&s.bins[b], 1u);
            else ++in_last;
        }
    }
    // Weight of a logit in the middle of a bin (none for the last, which has no end)
    __device__ __forceinline__ u64 bin_weight(int b) const { return b < kBins - 1 ? weight(weight.top - b * bin_step) : 0; }
    // Bins of the whole row from those of the CTAs (which a cluster barrier has seen done): each CTA adds up its share and hands it
    // to all.
    template <bool kCut>
    __device__ void share_bins()
    {
        const uint32_t *bins = kCut ? s.cut : s.bins;
        uint32_t *all_bins = kCut ? s.all_cut : s.all_bins;
        const int per = kBins / n_cta;
        for (int i = threadIdx.x; i < per / 2; i += kThreads) {
            const int bin = rank * per + 2 * i;
            u64 c = 0;                  // two 32-bit counters side by side: neither overflows
            int r = 0;
            for (; r + 4 <= n_cta; r += 4) {
                u64 y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = ld_peer(peer_address(ptx::smem_u32(&bins[bin]), r + j));
                c += (y[0] + y[1]) + (y[2] + y[3]);
            }
            for (; r < n_cta; ++r) c += ld_peer(peer_address(ptx::smem_u32(&bins[bin]), r));
            for (r = 0; r < n_cta; ++r) st_peer(peer_address(ptx::smem_u32(&all_bins[bin]), r), c);
        }
        cluster_sync();
    }
    __device__ void clear_bins(uint32_t *bins)
    {
        for (int i = threadIdx.x; i < kBins; i += kThreads) bins[i] = 0;
        __syncthreads();
    }
    // First bin at which the running sum, of tokens or (`each`: weight of a token of a bin) of weights, reaches `want`; kBins if none
    // does.  The sum before it.  s.around: the first bins that reach these sums.
    template <bool kCut, typename Each>
    __device__ int bin_reaching(u64 want, u64 &before, Each each, u64 s0 = 0, u64 s1 = 0, u64 s2 = 0, u64 s3 = 0)
    {
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
        constexpr int kEach = kBins / kThreads;
        u64 a[kEach], mine = 0;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const uint32_t c = (kCut ? s.all_cut : s.all_bins)[tid * kEach + k];
            a[k] = c ? c * each(tid * kEach + k) : 0;
            mine += a[k];
        }
        u64 in = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const u64 y = __shfl_up_sync(0xffffffffu, in, o);
            if (lane >= o) in += y;
        }
        if (lane == 31) s.warp_val[0][warp] = in;
        if (tid < 5) (tid < 4 ? s.around[tid] : s.bin) = kBins;
        __syncthreads();
        u64 at = in - mine;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) at += w < warp ? s.warp_val[0][w] : 0;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            if (at < want && at + a[k] >= want) {
                s.bin = tid * kEach + k;
                s.cum = at;
            }
            if (at < s0 && at + a[k] >= s0) s.around[0] = tid * kEach + k;
            if (at < s1 && at + a[k] >= s1) s.around[1] = tid * kEach + k;
            if (at < s2 && at + a[k] >= s2) s.around[2] = tid * kEach + k;
            if (at < s3 && at + a[k] >= s3) s.around[3] = tid * kEach + k;
            at += a[k];
        }
        __syncthreads();
        const int bin = s.bin;
        before = s.cum;
        __syncthreads();
        return bin;
    }

    // Puts a bin right by exact sums of the row's weights: the one in which the running sum over the bins reaches `need`.  `bin_at`
    // says which bin of 0..kBins - 1 a logit is in (-1: none); the lists, if any, hold bins up to `b_listed`.  `before`: the sum of the
    // bins before it; `count`: its tokens.
    template <typename BinAt>
    __device__ int settle(int b, int b_listed, u64 need, u64 &before, u64 &count, BinAt bin_at)
    {
        if (b >= kBins) b = kBins - 1;
        int lo = 0, hi = kBins - 1;
        for (int turn_no = 0;; ++turn_no) {
            if (b > b_listed) listed = -1;
            u64 above = 0, inside = 0, tokens = 0;
            for_each([&](float l, int) {
                const int bb = bin_at(l);
                if (bb < 0 || bb > b || !(l > -INFINITY)) return;
                const u64 w = weight(l);
                if (bb < b) above += w;
                else {
                    inside += w;
                    ++tokens;
                }
            });
            const int slot = gather<3>(above, inside, tokens, 0);
            const u64 a = of_all(slot, 0, 0), in = of_all(slot, 1, 0);
            before = a;
            count = of_all(slot, 2, 0);
            if (a >= need && b > lo) hi = b - 1;
            else if (a + in < need && b < hi) lo = b + 1;
            else return b;
            // (the bin chosen by the bins' middles is off by one if at all; otherwise the range is halved)
            b = turn_no < 2 ? (a >= need ? b - 1 : b + 1) : (lo + hi) / 2;
        }
    }

    // Gives a token of the candidates to all CTAs; places are handed out by the first.
    __device__ __forceinline__ void put_candidate(float l, int i, u64 w)
    {
        const uint32_t at = add_peer(peer_address(ptx::smem_u32(&s.n_cand), 0), 1u);
        if (at >= kCandidates) return;          // (never: they have been counted)
        const u64 word = ((u64)key_of(l) << 32) | (0xFFFFFFFFu - (uint32_t)(first + i));
        for (int r = 0; r < n_cta; ++r) {
            st_peer(peer_address(ptx::smem_u32(&s.cand[at]), r), word);
            st_peer(peer_address(ptx::smem_u32(&s.cand_weight[at]), r), w);
        }
    }
    // The one of m candidates at which the running sum in their order reaches `need`; false if none does.  (A cluster barrier
    // has seen them there.)
    __device__ bool rank_candidates(int m, u64 need, Place &place)
    {
        const int tid = threadIdx.x;
        if (tid == 0) s.n_cand = 0;
        // larger words come first; lanes side by side share a candidate's comparisons
        const bool shared = m > kRankAlone && n_cta > 1;
        const int by = shared ? n_cta : 1, c_of = shared ? rank : 0, own = (m - c_of + by - 1) / by;
        int side = 1;
        while (side < 32 && side * 2 * own <= kThreads) side *= 2;
        for (int c0 = 0; c0 < own; c0 += kThreads / side) {
            const int c = (c0 + tid / side) * by + c_of;
            const u64 mine = c < m ? s.cand[c] : 0;
            u64 sum = 0;
            if (c < m) {
#pragma unroll 4
                for (int j = tid % side; j < m; j += side)
                    if (s.cand[j] > mine) sum += s.cand_weight[j];
            }
            for (int o = side / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (c < m && tid % side == 0 && sum < need && sum + s.cand_weight[c] >= need) {
                if (!shared) {
                    s.place = mine;
                    s.found = 1;
                } else {
                    for (int r = 0; r < n_cta; ++r) {
                        st_peer(peer_address(ptx::smem_u32(&s.place), r), mine);
                        st_peer(peer_address(ptx::smem_u32(&s.found), r), 1);
                    }
                }
            }
        }
        if (shared) cluster_sync();
        else __syncthreads();
        const bool found = s.found != 0;
        if (found) {
            place.key = (uint32_t)(s.place >> 32);
            place.index = (int)(0xFFFFFFFFu - (uint32_t)s.place);
        }
        __syncthreads();
        if (tid == 0) s.found = 0;              // (a cluster barrier comes before the next candidates)
        return found;
    }

    // The last token of the prefix: of the `total` tokens of bin `bin` of (M - l), the one at which the count (by_mass = false) or
    // the sum of weights reaches `need`, counted from the bin's first.
    __device__ Place resolve(int bin, bool by_mass, u64 need, u64 total)
    {
        const int tid = threadIdx.x, lane = tid & 31;
        uint32_t lo = key_of(-INFINITY) + 1, hi = 0xFFFFFFFFu;             // keys of the bin
        auto in_bin = [&](float l, uint32_t &k) {
            k = key_of(l);
            return bin_of(l) == bin && k >= lo && k <= hi;
        };
        for (;;) {
            if (total <= kCandidates) {
                for_each([&](float l, int i) {
                    uint32_t k;
                    if (in_bin(l, k)) put_candidate(l, i, by_mass ? weight(l) : 1);
                });
                cluster_sync();
                Place p = {0u, 0x7fffffff};
                rank_candidates((int)total, need, p);
                return p;
            }
            u64 most = 0, least = 0, count = 0;
            for_each([&](float l, int) {
                uint32_t k;
                if (!in_bin(l, k)) return;
                most = max((u64)k, most);
                least = max((u64)(0xFFFFFFFFu - k), least);
                ++count;
            });
            int slot = gather<2>(most, least, 0, 1);
            const uint32_t k_hi = (uint32_t)of_all(slot, 0, 1), k_lo = 0xFFFFFFFFu - (uint32_t)of_all(slot, 1, 1);
            if (k_hi == k_lo) {
                // ---- one value: the place among equals is a matter of index
                const u64 each = by_mass ? weight(logit_of(k_hi)) : 1;
                u64 nth = each ? (need + each - 1) / each : 1;              // counted from 1
                if (nth > total) nth = total;
                if (nth < 1) nth = 1;
                slot = gather<1>(count, 0, 0, 0);
                u64 before = 0;
                for (int r = 0; r < rank; ++r) before += s.box[slot][r][0];
                const u64 here = s.box[slot][rank][0];
                if (tid == 0) s.answer = -1;
                __syncthreads();
                if (nth > before && nth <= before + here && tid < 32) {
                    u64 left = nth - before;
                    for (int i0 = 0; i0 < n; i0 += 32) {
                        const bool is = i0 + lane < n && key_of(v[i0 + lane]) == k_hi;
                        const uint32_t which = __ballot_sync(0xffffffffu, is);
                        if ((u64)__popc(which) >= left) {
                            const int at = __fns(which, 0, (int)left);
                            if (lane == 0) s.answer = first + i0 + at;
                            break;
                        }
                        left -= __popc(which);
                    }
                }
                __syncthreads();
                slot = gather<1>(tid == 0 ? (u64)(s.answer + 1) : 0, 0, 0, 1);
                Place p;
                p.key = k_hi;
                p.index = (int)of_all(slot, 0, 1) - 1;
                return p;
            }
            // ---- bins of the keys, in the candidates' place: the row's own histogram and the lists are needed again
            int shift = 0;
            while (((k_hi - k_lo) >> shift) >= (uint32_t)kBins) ++shift;
            lo = k_lo;
            hi = k_hi;
            auto key_bin = [&](float l) {
                uint32_t k;
                return in_bin(l, k) ? (int)((k_hi - k) >> shift) : -1;
            };
            clear_bins(s.cut);
            for_each([&](float l, int) {
                const int b = key_bin(l);
                if (b >= 0) atomicAdd(&s.cut[b], 1u);
            });
            cluster_sync();
            share_bins<true>();
            u64 at = 0;
            int b;
            if (by_mass) {
                b = bin_reaching<true>(need, at, [&](int k) { return weight(logit_of(k_hi - ((uint32_t)k << shift))); });
                b = settle(b, kBins, need, at, total, key_bin);
            } else {
                b = bin_reaching<true>(need, at, [](int) { return 1ull; });
                total = s.all_cut[b];
                cluster_sync();                 // (all have read them: the next candidates go there)
            }
            need -= at;
            const uint32_t top_key = k_hi - ((uint32_t)b << shift);
            hi = top_key;
            lo = max(k_lo, top_key - min(top_key, (1u << shift) - 1u));
        }
    }
};

template <bool kBf16>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const SampleParams p)
{
    extern __shared__ __align__(16) uint8_t smem_raw[];
    Shared &s = *reinterpret_cast<Shared *>(smem_raw);
    float *values = reinterpret_cast<float *>(smem_raw + ((sizeof(Shared) + 15) & ~size_t(15)));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    Row r(s);
    r.n_cta = p.cluster;
    r.rank = (int)cluster_rank();
    int row = blockIdx.x / p.cluster;

    cluster_here();
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    if (p.by_cost) {
        // more rows than run at once: those that take longest first (by their filters, then by index)
        const bool is = tid < p.rows;
        const float t = is && p.temperature ? p.temperature[tid] : 1.f, tp = is && p.top_p ? p.top_p[tid] : 1.f;
        const int k = is && p.top_k ? p.top_k[tid] : 0;
        const float mp = is && p.min_p ? p.min_p[tid] : 0.f;
        const bool has_k = k > 0 && k < p.vocab, has_p = tp < 1.f;
        const int kind = !(t > 0.f) ? 4 : has_k && has_p ? 1 : has_p ? 0 : has_k ? 2 : mp > 0.f ? 4 : 3;
        uint32_t same = 0;
        u64 counts = 0;                 // 12 bits for each kind
#pragma unroll
        for (int c = 0; c < 5; ++c) {
            const uint32_t has = __ballot_sync(0xffffffffu, is && kind == c);
            counts |= (u64)__popc(has) << (12 * c);
            if (kind == c) same = has;
        }
        if (lane == 0) s.warp_val[0][warp] = counts;
        __syncthreads();
        u64 all = 0, before = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            all += s.warp_val[0][w];
            before += w < warp ? s.warp_val[0][w] : 0;
        }
        int at = (int)(before >> (12 * kind) & 0xFFF) + __popc(same & ((1u << lane) - 1u));
#pragma unroll
        for (int c = 0; c < 4; ++c) at += c < kind ? (int)(all >> (12 * c) & 0xFFF) : 0;
        if (is && at == row) s.row = tid;
        __syncthreads();
        row = s.row;
    }
    const float T = p.temperature ? p.temperature[row] : 1.f;
    const int top_k = p.top_k ? p.top_k[row] : 0;
    const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f;
    float u = p.uniform[row];
    u = u > 0.f ? fminf(u, 0.99999994f) : 0.f;

    // ---- this CTA's logits [c0, c1) into shared memory, 16 bytes at a time where the row's alignment has them
    constexpr int kVec = kBf16 ? 8 : 4;
    const int per = ((p.vocab + p.cluster - 1) / p.cluster + kVec - 1) / kVec * kVec;
    const int c0 = min(p.vocab, r.rank * per), c1 = min(p.vocab, c0 + per);
    const size_t esz = kBf16 ? 2 : 4;
    const char *from = static_cast<const char *>(p.logits) + ((size_t)row * p.row_stride + c0) * esz;
    const int pad = (int)((reinterpret_cast<uintptr_t>(from) & 15u) / esz);          // elements before the first 16-byte group's
    r.v = values + pad;
    r.pad = pad;
    r.n = c1 - c0;
    r.first = c0;
    bool nan_seen = false;
    float best = -INFINITY;
    auto take = [&](float x) {
        // NaN ranks as -inf; -0 and 0 are one value
        if (x != x) {
            nan_seen = true;
            x = -INFINITY;
        }
        best = fmaxf(best, x);
        return x + 0.f;
    };
    const int groups = (pad + r.n + kVec - 1) / kVec;
    constexpr int kAhead = 5;           // 16-byte loads of a thread in flight
    for (int g0 = tid; g0 < groups; g0 += kAhead * kThreads) {
        uint4 w[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const int e = (g0 + a * kThreads) * kVec - pad;         // place in the chunk
            if (e >= 0 && e + kVec <= r.n) w[a] = *reinterpret_cast<const uint4 *>(from + (long long)e * (long long)esz);
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const int g = g0 + a * kThreads, e = g * kVec - pad;
            if (g >= groups) break;
            const bool whole = e >= 0 && e + kVec <= r.n;
            const uint32_t ww[4] = {w[a].x, w[a].y, w[a].z, w[a].w};
            float x[kVec];
#pragma unroll
            for (int k = 0; k < kVec; ++k) {
                x[k] = -INFINITY;
                if (whole)
                    x[k] = kBf16 ? __uint_as_float(k & 1 ? ww[k / 2] & 0xFFFF0000u : ww[k / 2] << 16) : __uint_as_float(ww[k % 4]);
                else if (e + k >= 0 && e + k < r.n)
                    x[k] = kBf16 ? __uint_as_float((uint32_t) reinterpret_cast<const uint16_t *>(from)[e + k] << 16)
                                 : reinterpret_cast<const float *>(from)[e + k];
                if (whole || (e + k >= 0 && e + k < r.n)) x[k] = take(x[k]);
            }
#pragma unroll
            for (int k = 0; k < kVec; k += 4)
                *reinterpret_cast<float4 *>(values + g * kVec + k) = make_float4(x[k], x[k + 1], x[k + 2], x[k + 3]);
        }
    }
    if (nan_seen) atomicOr(p.status, LVSPEC_DEV_NAN_LOGIT);
    if (tid == 0) s.n_cand = 0, s.found = 0;
    r.clear_bins(s.bins);
    const int n4 = (pad + r.n + 3) / 4, share = (n4 + kWarps - 1) / kWarps;
    r.g0 = min(warp * share, n4);
    r.g1 = min(r.g0 + share, n4);
    cluster_all_here();
    const float top = logit_of((uint32_t)r.of_all(r.gather<1>(key_of(best + 0.f), 0, 0, 1), 0, 1));
    if (!(T > 0.f) || !(top > -INFINITY)) {
        // greedy: the lowest index with the largest logit; a row with nothing above -inf gives token 0
        u64 at = 0;
        r.for_each([&](float l, int i) {
            if (l == top) at = max(at, (u64)(0xFFFFFFFFu - (uint32_t)(c0 + i)));
        });
        at = r.of_all(r.gather<1>(at, 0, 0, 1), 0, 1);
        if (r.rank == 0 && tid == 0) {
            p.tokens[row] = at ? (int)(0xFFFFFFFFu - (uint32_t)at) : 0;
            if (p.probs) p.probs[row] = 1.f;
        }
        return;
    }
    r.weight.set(fminf(top, FLT_MAX), T);
    if (top > FLT_MAX) {
        // infinite logits: as the largest finite number they keep all the weight among them (unless that number is there too, or T
        // so large that others count beside it)
        for (int i = tid; i < r.n; i += kThreads)
            if (values[pad + i] > FLT_MAX) values[pad + i] = FLT_MAX;
        __syncthreads();
    }
    // steps of T / 64 (32 T in all; what lies beyond weighs nothing), or, for a boundary by weight alone, T / 128: fewer tokens to rank
    r.bins_per = fmaxf(fminf((top_k > 0 ? 64.f : 128.f) / T, 3.0e38f), 1.0e-37f);
    r.bin_step = 1.f / r.bins_per;

    // ---- the shortest prefix that the filters keep
    Place place = {0u, 0x7fffffff};                     // everything
    const bool by_p = top_p < 1.f;
    bool by_k = top_k > 0 && top_k < p.vocab, filtered = false;
    if (by_k || by_p) {
        const bool weigh = !by_k;       // (with top-k it is only known later what counts)
        u64 whole = 0;
        uint32_t in_last = 0;
        if (weigh)
            r.for_each([&](float l, int) {
                r.count(l, in_last);
                whole += r.weight(l);
            });
        else
            r.for_each([&](float l, int) { r.count(l, in_last); });
        in_last = __reduce_add_sync(0xffffffffu, in_last);
        if (lane == 0 && in_last) atomicAdd(&s.bins[kBins - 1], in_last);
        if (weigh) whole = r.of_all(r.gather<1>(whole, 0, 0, 0), 0, 0);
        else cluster_sync();
        r.share_bins<false>();
        int b_listed = kBins;
        u64 before = 0;
        if (by_k) {
            const int b = r.bin_reaching<false>((u64)top_k, before, [](int) { return 1ull; });
            if (b < kBins) {            // (otherwise fewer logits above -inf than that: no filter)
                b_listed = b;
                r.make_list(r.least_of(b));
                place = r.resolve(b, false, (u64)top_k - before, s.all_bins[b]);
                filtered = true;
            }
        }
        if (by_p) {
            // of the weight that top-k leaves top-p keeps a share
            if (by_k) {
                whole = 0;
                r.for_each([&](float l, int i) {
                    if (place.reaches(key_of(l), c0 + i)) whole += r.weight(l);
                });
                whole = r.of_all(r.gather<1>(whole, 0, 0, 0), 0, 0);
            }
            // the first sum that is not below top_p * whole; at least the first token
            const u64 need = min(whole, max((u64)1, (u64)ceil(fmax((double)top_p, 0.0) * (double)whole)));
            // The bins' middles are off by exp(1 / 128) at most: the boundary is between the bins that reach 1 % less and 1 % more.
            // Their tokens are ranked by exact sums; where they are too many, those within 0.1 % and of the bins beside (errors of
            // many bins cancel).  What is then not among them (or too many again) is settled step by step.
            int b = min(r.bin_reaching<false>(need, before, [&](int k) { return r.bin_weight(k); }, max((u64)1, need - need / 100),
                                       need + need / 64 + 1, max((u64)1, need - need / 1024), need + need / 1024 + 1),
                        kBins - 1);
            int b0 = min(s.around[0], b), b1 = min(max(s.around[1], b), kBins - 1);
            const int c0_near = min(s.around[2], max(b - 1, 0)), c1_near = min(max(s.around[3], b + 1), kBins - 1);
            auto tokens_between = [&](int from, int to) {
                u64 n = 0;
                for (int k = from + tid; k <= to; k += kThreads) n += s.all_bins[k];
                n = __reduce_add_sync(0xffffffffu, (uint32_t)n);
                __syncthreads();
                if (lane == 0) s.warp_val[1][warp] = n;
                __syncthreads();
                n = 0;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) n += s.warp_val[1][w];
                __syncthreads();            // (the next gather writes them)
                return n;
            };
            u64 near = tokens_between(b0, b1);
            if (near > kCandidates || near > (u64)(kRankAlone / 4 * r.n_cta + kRankAlone)) {
                b0 = c0_near;
                b1 = c1_near;
                near = tokens_between(b0, b1);
            }
            if (!filtered) {
                b_listed = b1;
                r.make_list(r.least_of(b1));
            }
            Place q = place;
            bool found = false;
            if (near <= kCandidates && b1 <= b_listed) {
                u64 above = 0;
                r.for_each([&](float l, int i) {
                    const int bb = r.bin_of(l);
                    if (bb > b1 || !(l > -INFINITY)) return;
                    const u64 w = r.weight(l);
                    if (bb < b0) above += w;
                    else r.put_candidate(l, i, w);
                });
                above = r.of_all(r.gather<1>(above, 0, 0, 0), 0, 0);
                found = r.rank_candidates((int)near, need > above ? need - above : 0, q);        // (0: none does)
            }
            if (!found) {
                u64 total = 0;
                b = r.settle(b, b_listed, need, before, total, [&](float l) { return r.bin_of(l); });
                q = r.resolve(b, true, need - before, total);
            }
            if (!filtered || q.key > place.key || (q.key == place.key && q.index < place.index)) place = q;
            filtered = true;
        }
    }
    uint32_t least_key = 0;
    if (min_p > 0.f) {
        const double down = min_p < 1.f ? (double)T * log((double)min_p) : 0.0;         // (not an infinite T times the logarithm of 1)
        least_key = key_of(__double2float_ru((double)r.weight.top + down) + 0.f);
        if (!filtered) r.make_list(logit_of(least_key));
        filtered = true;
    }

    // ---- running sums in index order: of the CTAs, of the warps, and within the warp that has the token
    auto kept_weight = [&](float l, int i) -> u64 {
        if (!filtered) return r.weight(l);
        const uint32_t k = key_of(l);
        return l > -INFINITY && k >= least_key && place.reaches(k, c0 + i) ? r.weight(l) : 0;
    };
    u64 mine = 0;
    if (filtered) r.for_each([&](float l, int i) { mine += kept_weight(l, i); });
    else r.for_each([&](float l, int) { mine += r.weight(l); });
    const int slot = r.gather<1>(mine, 0, 0, 0);
    const u64 total = r.of_all(slot, 0, 0);
    u64 at = 0;
    for (int k = 0; k < r.rank; ++k) at += s.box[slot][k][0];
    // the token's running sum is the first above u * total
    const u64 goal = (u64)((double)u * (double)total);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) at += w < warp ? s.warp_val[0][w] : 0;
    if (goal < at || goal >= at + s.warp_val[0][warp]) return;
    const int step = r.listed >= 0 ? 32 : 128;
    for (int e = r.listed >= 0 ? 0 : r.g0 * 4; e < (r.listed >= 0 ? r.listed : r.g1 * 4); e += step) {
        // a lane's tokens: one of the list, or four neighbours
        int i = -pad;
        u64 w[4] = {0, 0, 0, 0};
        if (r.listed >= 0) {
            if (e + lane < r.listed) {
                i = s.list[warp][e + lane];
                w[0] = kept_weight(r.v[i], i);
            }
        } else if (e + 4 * lane < r.g1 * 4) {
            i = e + 4 * lane - pad;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (r.v[i + k] > -INFINITY) w[k] = kept_weight(r.v[i + k], i + k);
        }
        const u64 own = (w[0] + w[1]) + (w[2] + w[3]);
        u64 in = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const u64 y = __shfl_up_sync(0xffffffffu, in, o);
            if (lane >= o) in += y;
        }
        u64 from_here = at + in - own;
        at += __shfl_sync(0xffffffffu, in, 31);
        if (goal >= at) continue;
        if (goal >= from_here && goal < from_here + own) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (goal >= from_here && goal < from_here + w[k]) {
                    p.tokens[row] = c0 + i + k;
                    if (p.probs) p.probs[row] = (float)((double)w[k] / (double)total);
                }
                from_here += w[k];
            }
        }
        return;
    }
}

}  // namespace

size_t sample_smem_bytes(int vocab, int cluster)
{
    const int per = ((vocab + cluster - 1) / cluster + 7) / 8 * 8;
    return ((sizeof(Shared) + 15) & ~size_t(15)) + ((size_t)per + 16) * sizeof(float);
}

// CTAs of a row.  Many rows: as few as hold it with two CTAs an SM (19 K logits each, 76 KB), up to eight: every exchange costs
// the same however little a CTA has.  While the rows leave room for more at once: up to one for each 4 K, and of a large vocabulary
// sixteen: 12 rows of 152064 with top-p 0.9 take 24 us instead of 30, 18 rows 38 instead of 32 (then most SMs have two CTAs).
int sample_cluster(int vocab, int rows, int n_sm)
{
    int c = 1;
    while (c < 8 && vocab > c * 19456) c *= 2;
    while (c < 8 && vocab > c * 4096 && rows * c <= n_sm) c *= 2;
    if ((c == 8 && vocab > 65536 && 2 * rows * kMaxCluster <= 3 * n_sm) || sample_smem_bytes(vocab, c) > 227 * 1024) c = kMaxCluster;
    return c;
}

cudaError_t launch_sample(const SampleParams &params, int rows, bool bf16, bool pdl, int n_sm, cudaStream_t stream, int *launches)
{
    SampleParams p = params;
    p.rows = rows;
    // (128 rows of 152064 with mixed filters: 121 us in their order, 93 us like this; all of one kind 4 % slower)
    p.by_cost = rows <= kThreads && rows * p.cluster > 2 * n_sm;
    const size_t smem = sample_smem_bytes(p.vocab, p.cluster);
    const auto kernel = bf16 ? sample_kernel<true> : sample_kernel<false>;
    cudaError_t e = allow_shared_memory(kernel);
    if (e != cudaSuccess) return e;
    if (p.cluster > 8 && (e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1)) != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(rows * p.cluster), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, kernel, p);
    ++*launches;
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace lvspec
