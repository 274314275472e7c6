// Sampling from logits by temperature, top-k, top-p and min-p, from one given uniform number per row.
//
// With M the row's largest logit and T the temperature, token i has weight w_i = exp((l_i - M) / T).  In the
// order of falling logits (equal ones by rising index) every filter keeps a prefix: top-k its first k, top-p the
// shortest prefix of those with at least the share p of their weight, min-p the logits at or above
// M + T ln(min_p).  Of what the shortest prefix keeps, taken in index order again, the token is the first whose
// running sum exceeds u times the whole.
//
// Weights are integers, 2^40 for the largest: (l_i - M) log2(e) / T with its rounding errors carried, 2^x of its fraction to 2^-22.  Sums
// of integers do not depend on their order, so a row gives the same token however it is cut up.
//
// A row is read once, by a cluster of up to eight CTAs that keep it in their shared memory (a vocabulary of 152 K is 76 KB
// each, two CTAs an SM) and pass sums on through distributed shared memory; it is bound by the latency of these
// exchanges (a barrier each) and by the passes over shared memory, not by HBM.  A boundary is
// found without sorting: a histogram over (M - l) in steps of T / 32, then the few hundred tokens of the bin that holds the
// boundary are ranked by comparing all with all; a bin with more tokens than fit there (equal or nearly equal logits) is cut
// into bins of the logits' bit patterns until it fits or holds a single value.  Top-p's bin is chosen by sums of weights
// rounded to 2^-13, which is all 32-bit shared-memory atomics carry, and put right by exact sums.
#include "lvspec_internal.h"
#include "sm100_ptx.cuh"

namespace lvspec {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 1024;
constexpr int kCandidates = 1024;       // tokens of a bin that are ranked directly
constexpr int kMaxCluster = 8;
constexpr int kCoarse = 13;             // bits of a weight in the histogram
typedef unsigned long long u64;

// ---- cluster -----------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
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

struct Weight {
    float top;              // the row's largest logit
    float per, per_rest;    // log2(e) / T in two parts
    __device__ __forceinline__ void set(float top_, float T)
    {
        top = top_;
        const double c = 1.4426950408889634 / (double)T;
        per = (float)c;
        per_rest = isinf(per) ? 0.f : (float)(c - (double)per);
    }
    // round(2^40 exp((l - top) / T)): the difference and its product with `per` carried with their rounding errors, 2^x of
    // the fraction good to 2^-22, its 24 bits shifted into place
    __device__ __forceinline__ u64 operator()(float l) const
    {
        if (l == top) return 1ull << 40;        // (both infinite too)
        const float d = l - top, z = d - l;
        const float d_rest = (l - (d - z)) + (-top - z);
        const float y = d * per;
        if (!(y > -42.f)) return 0;             // (also -inf, and a top that is infinite)
        const float n = rintf(y);
        const float f = (y - n) + (fmaf(d, per, -y) + fmaf(d, per_rest, d_rest * per));
        const uint32_t e = __float_as_uint(ptx::ex2(f));
        const int shift = (int)n + (int)(e >> 23) - 127 + 17;
        const u64 m = (e & 0x7FFFFFu) | 0x800000u;
        return shift >= 0 ? m << shift : (m + (1ull << (-shift - 1))) >> -shift;
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
    uint32_t count[kBins], mass[kBins];             // of this CTA's tokens
    uint32_t all_count[kBins], all_mass[kBins];     // of the whole row's
    u64 cand[kCandidates];              // key, index of a bin's tokens
    u64 cum[2];
    int bin, n_cand, answer;
    Place place;
};

struct Row {
    Shared &s;
    const float *v;                     // this CTA's logits, v[0 .. n)
    int n, first;                       // first: the index of v[0]
    int n_cta, rank, turn;
    Weight weight;
    float bins_per;                     // 32 / T

    __device__ __forceinline__ Row(Shared &s_) : s(s_), turn(0) {}

    // Sums (op 0), or largest values (op 1), of up to three numbers per thread over the row; every CTA's in box[slot].
    __device__ int gather(u64 a, u64 b, u64 c, int op)
    {
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
        u64 x[3] = {a, b, c};
#pragma unroll
        for (int k = 0; k < 3; ++k) {
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
            for (int k = 0; k < 3; ++k) {
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
        for (int r = 0; r < n_cta; ++r) {
            const u64 y = s.box[slot][r][k];
            t = op ? (y > t ? y : t) : t + y;
        }
        return t;
    }
    __device__ __forceinline__ int bin_of(float l) const
    {
        // (falls as l rises, whatever the rounding; infinities: bin 0 for the top, the last for -inf)
        const float t = (weight.top - l) * bins_per;
        return l == weight.top ? 0 : t < (float)(kBins - 1) ? (int)t : kBins - 1;
    }
    // Bins of the whole row from those of the CTAs: each CTA adds up its share and hands it to all.
    __device__ void share_bins()
    {
        cluster_sync();
        const int per = kBins / n_cta;
        for (int i = threadIdx.x; i < per / 2; i += kThreads) {
            const int bin = rank * per + 2 * i;
            u64 c = 0, m = 0;           // two 32-bit counters side by side: neither overflows
            for (int r = 0; r < n_cta; ++r) {
                c += ld_peer(peer_address(ptx::smem_u32(&s.count[bin]), r));
                m += ld_peer(peer_address(ptx::smem_u32(&s.mass[bin]), r));
            }
            for (int r = 0; r < n_cta; ++r) {
                st_peer(peer_address(ptx::smem_u32(&s.all_count[bin]), r), c);
                st_peer(peer_address(ptx::smem_u32(&s.all_mass[bin]), r), m);
            }
        }
        cluster_sync();
    }
    __device__ void clear_bins()
    {
        for (int i = threadIdx.x; i < kBins; i += kThreads) s.count[i] = s.mass[i] = 0;
        __syncthreads();
    }
    // First bin at which the running sum of `a` reaches `want` (the last one if none does); the sum before it.
    __device__ int bin_reaching(const uint32_t *a, u64 want, u64 &before)
    {
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
        constexpr int kEach = kBins / kThreads;
        u64 mine = 0;
#pragma unroll
        for (int k = 0; k < kEach; ++k) mine += a[tid * kEach + k];
        u64 in = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const u64 y = __shfl_up_sync(0xffffffffu, in, o);
            if (lane >= o) in += y;
        }
        if (lane == 31) s.warp_val[0][warp] = in;
        if (tid == 0) s.bin = kBins;
        __syncthreads();
        u64 at = in - mine;
        for (int w = 0; w < warp; ++w) at += s.warp_val[0][w];
        for (int k = 0; k < kEach; ++k) {
            const u64 next = at + a[tid * kEach + k];
            const bool last = tid * kEach + k == kBins - 1;
            if (at < want && (next >= want || last)) {
                s.bin = tid * kEach + k;
                s.cum[0] = at;
            }
            at = next;
        }
        __syncthreads();
        const int bin = s.bin;
        before = s.cum[0];
        __syncthreads();
        return bin;
    }

    // Puts a bin right by exact sums of the row's weights: the one in which the running sum over the bins reaches `need`.  `bin_at`
    // says which bin of 0..kBins - 1 a token is in (-1: none).  `before`: the sum of the bins before it.
    template <typename BinAt>
    __device__ int settle(int b, u64 need, u64 &before, BinAt bin_at)
    {
        if (b >= kBins) b = 0;
        int lo = 0, hi = kBins - 1;
        for (int turn_no = 0;; ++turn_no) {
            u64 above = 0, inside = 0, below = 0;
            for (int i = threadIdx.x; i < n; i += kThreads) {
                const int bb = bin_at(i);
                if (bb < 0) continue;
                const u64 w = weight(v[i]);
                if (bb < b) above += w;
                else if (bb == b) inside += w;
                else below += w;
            }
            const int slot = gather(above, inside, below, 0);
            const u64 a = of_all(slot, 0, 0), in = of_all(slot, 1, 0), rest = of_all(slot, 2, 0);
            before = a;
            if (a >= need && b > lo) hi = b - 1;
            else if (a + in < need && rest > 0 && b < hi) lo = b + 1;
            else return b;
            // (the bin chosen by coarse sums is off by one if at all; without such a choice the range is halved)
            b = turn_no < 2 ? (a >= need ? b - 1 : b + 1) : (lo + hi) / 2;
        }
    }

    // The last token of the prefix: of the tokens of bin `bin` of (M - l), the one at which the count (by_mass = false) or the sum of
    // weights reaches `need`, counted from the bin's first.
    __device__ Place resolve(int bin, bool by_mass, u64 need)
    {
        const int tid = threadIdx.x, lane = tid & 31;
        uint32_t lo = 0, hi = 0xFFFFFFFFu;              // keys of the bin
        for (;;) {
            // how many tokens, and between which keys
            u64 most = 0, least = 0, count = 0;
            for (int i = tid; i < n; i += kThreads) {
                const uint32_t k = key_of(v[i]);
                if (bin_of(v[i]) == bin && k >= lo && k <= hi) {
                    most = max((u64)k, most);
                    least = max((u64)(0xFFFFFFFFu - k), least);
                    ++count;
                }
            }
            int slot = gather(count, 0, 0, 0);
            const u64 total = of_all(slot, 0, 0);
            int before = 0;
            for (int r = 0; r < rank; ++r) before += (int)s.box[slot][r][0];
            if (total <= kCandidates) {
                // ---- rank them all
                if (tid == 0) s.n_cand = before;
                __syncthreads();
                for (int i = tid; i < n; i += kThreads) {
                    const uint32_t k = key_of(v[i]);
                    if (bin_of(v[i]) == bin && k >= lo && k <= hi) {
                        const int at = atomicAdd(&s.n_cand, 1);
                        for (int r = 0; r < n_cta; ++r)
                            st_peer(peer_address(ptx::smem_u32(&s.cand[at]), r), ((u64)k << 32) | (0xFFFFFFFFu - (uint32_t)(first + i)));
                    }
                }
                cluster_sync();
                // larger words come first; lanes side by side share a candidate's comparisons
                const int m = (int)total;
                int side = 1;
                while (side < 32 && side * 2 * m <= kThreads) side *= 2;
                for (int c0 = 0; c0 < m; c0 += kThreads / side) {
                    const int c = c0 + tid / side;
                    const u64 mine = c < m ? s.cand[c] : 0;
                    u64 sum = 0;
                    if (c < m)
                        for (int j = tid % side; j < m; j += side) {
                            const u64 other = s.cand[j];
                            if (other > mine) sum += by_mass ? weight(logit_of((uint32_t)(other >> 32))) : 1;
                        }
                    for (int o = side / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    if (c < m && tid % side == 0) {
                        const u64 own = by_mass ? weight(logit_of((uint32_t)(mine >> 32))) : 1;
                        if (sum < need && sum + own >= need) {
                            s.place.key = (uint32_t)(mine >> 32);
                            s.place.index = (int)(0xFFFFFFFFu - (uint32_t)mine);
                        }
                    }
                }
                __syncthreads();
                const Place p = s.place;
                __syncthreads();
                return p;
            }
            slot = gather(most, least, 0, 1);
            const uint32_t k_hi = (uint32_t)of_all(slot, 0, 1), k_lo = 0xFFFFFFFFu - (uint32_t)of_all(slot, 1, 1);
            if (k_hi == k_lo) {
                // ---- one value: the place among equals is a matter of index
                const u64 each = by_mass ? weight(logit_of(k_hi)) : 1;
                u64 nth = each ? (need + each - 1) / each : 1;              // counted from 1
                if (nth > total) nth = total;
                if (nth < 1) nth = 1;
                // (`before` equals sit in the CTAs before this one)
                const u64 here = count_sum(count);
                if (tid == 0) s.answer = -1;
                __syncthreads();
                if (nth > (u64)before && nth <= (u64)before + here && tid < 32) {
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
                slot = gather(tid == 0 ? (u64)(s.answer + 1) : 0, 0, 0, 1);
                Place p;
                p.key = k_hi;
                p.index = (int)of_all(slot, 0, 1) - 1;
                return p;
            }
            // ---- bins of the keys; exact counts, and for weights a round of exact sums
            int shift = 0;
            while (((k_hi - k_lo) >> shift) >= (uint32_t)kBins) ++shift;
            clear_bins();
            for (int i = tid; i < n; i += kThreads) {
                const uint32_t k = key_of(v[i]);
                if (bin_of(v[i]) == bin && k >= k_lo && k <= k_hi) {
                    const int b = (int)((k_hi - k) >> shift);
                    atomicAdd(&s.count[b], 1u);
                    if (by_mass) atomicAdd(&s.mass[b], (uint32_t)(weight(v[i]) >> (40 - kCoarse)));
                }
            }
            share_bins();
            u64 at = 0;
            int b = bin_reaching(by_mass ? s.all_mass : s.all_count, by_mass ? (need >> (40 - kCoarse)) + 1 : need, at);
            if (by_mass)
                b = settle(b, need, at, [&](int i) {
                    const uint32_t k = key_of(v[i]);
                    return bin_of(v[i]) == bin && k >= k_lo && k <= k_hi ? (int)((k_hi - k) >> shift) : -1;
                });
            need -= at;
            const uint32_t top_key = k_hi - ((uint32_t)b << shift);
            hi = top_key;
            lo = max(k_lo, top_key - min(top_key, (1u << shift) - 1u));
        }
    }
    // this CTA's sum of a number per thread
    __device__ u64 count_sum(u64 x)
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        if (lane == 0) s.warp_val[0][warp] = x;
        __syncthreads();
        u64 t = 0;
        for (int w = 0; w < kWarps; ++w) t += s.warp_val[0][w];
        __syncthreads();
        return t;
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
    const int row = blockIdx.x / p.cluster;

    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();
    const float T = p.temperature ? p.temperature[row] : 1.f;
    int top_k = p.top_k ? p.top_k[row] : 0;
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
    r.n = c1 - c0;
    r.first = c0;
    bool nan_seen = false;
    float best = -INFINITY;
    int best_i = 0x7fffffff;
    auto take = [&](float x, int i) {
        // NaN ranks as -inf; -0 and 0 are one value
        if (x != x) {
            nan_seen = true;
            x = -INFINITY;
        }
        x += 0.f;
        if (x > best || (x == best && i < best_i)) {
            best = x;
            best_i = i;
        }
        return x;
    };
    const int groups = (pad + r.n + kVec - 1) / kVec;
    for (int g = tid; g < groups; g += kThreads) {
        const int e = g * kVec - pad;                   // of the chunk
        float x[kVec];
        if (e >= 0 && e + kVec <= r.n) {
            const uint4 w = *reinterpret_cast<const uint4 *>(from + (long long)e * (long long)esz);
            const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int k = 0; k < kVec; ++k)
                x[k] = kBf16 ? __uint_as_float(k & 1 ? ww[k / 2] & 0xFFFF0000u : ww[k / 2] << 16) : __uint_as_float(ww[k % 4]);
        } else {
#pragma unroll
            for (int k = 0; k < kVec; ++k) {
                x[k] = -INFINITY;
                if (e + k >= 0 && e + k < r.n)
                    x[k] = kBf16 ? __uint_as_float((uint32_t) reinterpret_cast<const uint16_t *>(from)[e + k] << 16)
                                 : reinterpret_cast<const float *>(from)[e + k];
            }
        }
#pragma unroll
        for (int k = 0; k < kVec; ++k)
            if (e + k >= 0 && e + k < r.n) x[k] = take(x[k], c0 + e + k);
#pragma unroll
        for (int k = 0; k < kVec; k += 4)
            *reinterpret_cast<float4 *>(values + g * kVec + k) = make_float4(x[k], x[k + 1], x[k + 2], x[k + 3]);
    }
    if (nan_seen) atomicOr(p.status, LVSPEC_DEV_NAN_LOGIT);
    r.clear_bins();
    // largest logit, at its lowest index
    const u64 first_best = best_i == 0x7fffffff ? 0 : ((u64)key_of(best) << 32) | (0xFFFFFFFFu - (uint32_t)best_i);
    const u64 largest = r.of_all(r.gather(first_best, 0, 0, 1), 0, 1);
    const float top = logit_of((uint32_t)(largest >> 32));
    const int top_i = (int)(0xFFFFFFFFu - (uint32_t)largest);
    if (!(T > 0.f) || !(top > -INFINITY)) {
        // greedy; a row with nothing above -inf gives token 0
        if (r.rank == 0 && tid == 0) {
            p.tokens[row] = top > -INFINITY ? top_i : 0;
            if (p.probs) p.probs[row] = 1.f;
        }
        return;
    }
    r.weight.set(top, T);
    // (a top that is infinite has all other tokens in the last bin; a temperature that is, all in the first)
    r.bins_per = fminf(32.f / T, 3.0e38f);

    // ---- the shortest prefix that the filters keep
    Place place = {0u, 0x7fffffff};                     // everything
    const bool by_k = top_k > 0 && top_k < p.vocab, by_p = top_p < 1.f;
    if (by_k || by_p) {
        u64 all = 0;
        for (int i = tid; i < r.n; i += kThreads) {
            const int b = r.bin_of(r.v[i]);
            if (by_k) atomicAdd(&s.count[b], 1u);
            if (by_p) {
                const u64 w = r.weight(r.v[i]);
                all += w;
                const uint32_t m = (uint32_t)(w >> (40 - kCoarse));
                if (m) atomicAdd(&s.mass[b], m);
            }
        }
        r.share_bins();
        u64 before = 0;
        if (by_k) {
            const int b = r.bin_reaching(s.all_count, (u64)top_k, before);
            place = r.resolve(b, false, (u64)top_k - before);
        }
        if (by_p) {
            // what top-k leaves, of which top-p keeps a share
            u64 kept = all;
            if (by_k) {
                kept = 0;
                for (int i = tid; i < r.n; i += kThreads)
                    if (place.reaches(key_of(r.v[i]), c0 + i)) kept += r.weight(r.v[i]);
            }
            const u64 whole = r.of_all(r.gather(kept, 0, 0, 0), 0, 0);
            // the first sum that is not below p * whole; at least the first token
            const double share = fmax((double)top_p, 0.0) * (double)whole;
            u64 need = (u64)ceil(share);
            if (need < 1) need = 1;
            if (need > whole) need = whole;
            // (top-k's boundary has been resolved through the same arrays: the coarse sums are still the row's unless it was cut
            // into bins of keys, and any bin will do to begin with)
            int b = r.bin_reaching(s.all_mass, (need >> (40 - kCoarse)) + 1, before);
            b = r.settle(b, need, before, [&](int i) { return r.bin_of(r.v[i]); });
            const Place q = r.resolve(b, true, need - before);
            if (!by_k || q.key > place.key || (q.key == place.key && q.index < place.index)) place = q;
        }
    }
    uint32_t least_key = 0;
    if (min_p > 0.f) least_key = key_of(__double2float_ru((double)top + (double)T * log(fmin((double)min_p, 1.0))) + 0.f);

    // ---- running sums in index order: a lane's tokens are neighbours (an odd number of them: no two lanes on a bank)
    const int each = ((r.n + kThreads - 1) / kThreads) | 1;
    const int i0 = min(r.n, tid * each), i1 = min(r.n, i0 + each);
    auto kept = [&](int i) -> u64 {
        const uint32_t k = key_of(r.v[i]);
        return k >= least_key && place.reaches(k, c0 + i) ? r.weight(r.v[i]) : 0;
    };
    u64 mine = 0;
    for (int i = i0; i < i1; ++i) mine += kept(i);
    const int slot = r.gather(mine, 0, 0, 0);
    const u64 total = r.of_all(slot, 0, 0);
    u64 at = 0;
    for (int k = 0; k < r.rank; ++k) at += s.box[slot][k][0];
    // the token's running sum is the first above u * total
    const u64 goal = (u64)((double)u * (double)total);
    if (goal < at || goal >= at + s.box[slot][r.rank][0]) return;
    u64 in = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 y = __shfl_up_sync(0xffffffffu, in, o);
        if (lane >= o) in += y;
    }
    for (int w = 0; w < warp; ++w) at += s.warp_val[0][w];
    at += in - mine;
    if (goal >= at && goal < at + mine) {
        for (int i = i0; i < i1; ++i) {
            const u64 w = kept(i);
            if (goal < at + w) {
                p.tokens[row] = c0 + i;
                if (p.probs) p.probs[row] = (float)((double)w / (double)total);
                break;
            }
            at += w;
        }
    }
}

}  // namespace

size_t sample_smem_bytes(int vocab, int cluster)
{
    const int per = ((vocab + cluster - 1) / cluster + 7) / 8 * 8;
    return ((sizeof(Shared) + 15) & ~size_t(15)) + ((size_t)per + 16) * sizeof(float);
}

// CTAs of a row: enough that its logits fit and a CTA has some 20 K of them at most (two CTAs an SM then), one per 4 K.
int sample_cluster(int vocab)
{
    int c = 1;
    while (c < kMaxCluster && vocab > c * 4096) c *= 2;
    return c;
}

cudaError_t launch_sample(const SampleParams &p, int rows, bool bf16, bool pdl, cudaStream_t stream, int *launches)
{
    const size_t smem = sample_smem_bytes(p.vocab, p.cluster);
    const auto kernel = bf16 ? sample_kernel<true> : sample_kernel<false>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
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
