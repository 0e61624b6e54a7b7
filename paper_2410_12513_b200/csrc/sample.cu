// Next tokens of a batch with generation settings of its own for every request (the paper samples with temperature
// 0.8 and top-k 10, appendix "Training and Inference Setup"; requests of one batch need not agree on that).
//
// A row's candidates stand in descending order of their logits, equal ones by index.  Every filter keeps a prefix of
// that order, and so does a draw: the token is the first candidate whose cumulative weight exceeds u times the sum.
// All of them are the same question -- where does a running sum (of ones, or of weights) reach a target -- and it is
// answered without sorting the row:
//   1. One thread-block cluster per row; the row is read once and stays in the cluster's registers.
//   2. A histogram over 32 bins of (max - x) / T, half a unit wide: the sum reaches the target in one of them.
//   3. If that bin holds many elements, it is cut into 32 parts of its range of values (and again, and, among equal
//      values, of indices), each time keeping the part that holds the target.
//   4. What is left, at most kList elements, goes to every CTA's shared memory, is sorted there and summed up.
// A histogram is private to every LANE of every warp (a bin is 32 words, a lane owns one): a bank each, no atomics, so
// sums are the same in every run.  Weights are taken relative to that of the upper end X of their bin: exp((x - X) / T)
// with the difference exact, as integers in units of 2^-23, which keeps float32's 24 bits; the bins' own weights and
// all prefix sums are 64-bit floating point.
#include <cfloat>
#include <cooperative_groups.h>

#include "common.cuh"
#include "first.h"
#include "ops.h"

namespace first {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kRegs = 32;            // elements a thread holds; a CTA 16384, a cluster of eight 131072 (more are re-read from L2)
constexpr int kCluster = 8;
constexpr int kBins = 32;
constexpr int kLocal = 2048;         // elements of one bin that a CTA keeps in shared memory
constexpr int kSlot = 64;            // elements that a CTA may put into a list ...
constexpr int kList = kCluster * kSlot;  // ... which every CTA of the cluster sorts, one element a thread
constexpr int kSorted = 320;         // longer lists are narrowed further first: sorting takes time with the square of them
constexpr int kSlices = 8;           // lane-private histograms of a CTA, each shared by two warps
constexpr double kUnit = 1.0 / 8388608.0;  // 2^-23

// descending: the largest logit has the smallest key; -0 has been turned into +0
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x);
    return (b & 0x80000000u) ? b : ~(b | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? k : ~(k | 0x80000000u));
}
__device__ __forceinline__ float clean(float x) { return x != x ? -INFINITY : x + 0.f; }

struct Result {  // the last element of a kept prefix, and the prefix's weight
    float x;
    int i;
    double mass;
};

struct Smem {
    uint32_t hist[kSlices][kBins][32];
    float X[kBins][32];              // a bin's upper end, once per lane: the same offset as in a histogram
    uint2 loc[kLocal];               // the bin being searched: this CTA's elements, (value, index)
    unsigned long long list[2][kList];  // (turn by turn: a CTA may be at the next search while another still reads)
    unsigned long long tmp[kList];   // value key << 32 | index
    uint32_t cnt[2][kCluster];
    unsigned long long xch[2][kCluster][kBins];
    double W[kBins];                 // weight of a bin's upper end, per unit
    double scan[kWarps];
    Result res;
    uint32_t key[2][kCluster], key_w[kWarps];
    uint32_t nloc, lcnt;
    int hit;
    float thr;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void red_add(uint32_t a, uint32_t v) { asm volatile("red.shared.add.u32 [%0], %1;" ::"r"(a), "r"(v)); }

struct Row {  // what a thread needs to know about the row
    float m, inv_T2, inv_Tl2;  // maximum; 2 / T (bins of half a unit), log2(e) / T
    // 2^23 + bin, as the bits of a float (monotone in x, like every step of it)
    __device__ __forceinline__ uint32_t bin_bits(float x) const {
        return __float_as_uint(fminf((m - x) * inv_T2, (float)(kBins - 1)) + 8388608.f);
    }
    __device__ __forceinline__ int bin(float x) const { return (int)(bin_bits(x) & (kBins - 1)); }
    // 2^23 + weight of x in units of 2^-23 of that of its bin's upper end X, on top of the bits of 1.0 (x - X is exact but
    // where it does not matter; it is above 0 by a rounding at most)
    __device__ __forceinline__ uint32_t unit_bits(float x, float X) const {
        return __float_as_uint(ex2(fminf((x - X) * inv_Tl2, 0.f)) + 1.f);
    }
    __device__ __forceinline__ uint32_t units(float x, float X) const { return unit_bits(x, X) - 0x3f800000u; }
};

template <bool VEC>
struct Slice {  // this thread's elements of the row
    const float* row;  // the CTA's first element
    int base, n;       // its index in the row; elements of the CTA
    float x[kRegs];

    __device__ __forceinline__ int local(int j) const {
        return VEC ? (j >> 2) * (4 * kThreads) + 4 * (int)threadIdx.x + (j & 3) : j * kThreads + (int)threadIdx.x;
    }
    __device__ __forceinline__ void load() {
#pragma unroll
        for (int j = 0; j < kRegs; j += VEC ? 4 : 1) {
            const int i = local(j);
            if constexpr (VEC) {
                float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                if (i + 3 < n) v = __ldcs(reinterpret_cast<const float4*>(row + i));
                else {
                    if (i < n) v.x = row[i];
                    if (i + 1 < n) v.y = row[i + 1];
                    if (i + 2 < n) v.z = row[i + 2];
                }
                x[j] = v.x; x[j + 1] = v.y; x[j + 2] = v.z; x[j + 3] = v.w;
            } else {
                x[j] = i < n ? __ldcs(row + i) : -INFINITY;
            }
        }
#pragma unroll
        for (int j = 0; j < kRegs; ++j) x[j] = clean(x[j]);
    }
    // elements beyond the registers (rows of more than 131072): f(value, index in the row)
    template <typename F>
    __device__ __forceinline__ void rest(bool infinite, F f) const {
        for (int i = kRegs * kThreads + (int)threadIdx.x; i < n; i += kThreads) {
            float v = clean(row[i]);
            if (infinite) v = v == INFINITY ? 0.f : -INFINITY;
            f(v, base + i);
        }
    }
    // f(value, index in the row); values are clean, elements that do not exist are -inf
    template <typename F>
    __device__ __forceinline__ void each(bool infinite, F f) const {
#pragma unroll
        for (int j = 0; j < kRegs; ++j) f(x[j], base + local(j));
        rest(infinite, f);
    }
};

__device__ __forceinline__ double warp_scan(double run, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double v = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += v;
    }
    return run;
}
__device__ __forceinline__ uint32_t warp_scan(uint32_t run, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += v;
    }
    return run;
}

// grid B * C in clusters of C; one cluster per row.  Every decision is taken by every warp of every CTA from the same
// numbers, so the cluster stays together without anyone telling the others.
template <bool VEC>
__global__ void __launch_bounds__(kThreads, 2) sample_rows(const SampleArgs p) {
    const Stamp stamp_guard(p.stamp);
    extern __shared__ __align__(16) uint8_t smem_raw[];
    Smem& s = *reinterpret_cast<Smem*>(smem_raw);
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int b = blockIdx.x / C, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    {
        uint4* h = reinterpret_cast<uint4*>(s.hist);
        for (int i = tid; i < (int)(sizeof s.hist / 16); i += kThreads) h[i] = make_uint4(0, 0, 0, 0);
    }
    cluster.barrier_arrive();  // (waited for before the first access to another CTA's shared memory)
    pdl_trigger();
    pdl_wait();
    Slice<VEC> el;
    const int chunk = ((p.V + C - 1) / C + 3) / 4 * 4;
    el.base = rank * chunk;
    el.n = max(0, min(chunk, p.V - el.base));
    el.row = p.logits + (int64_t)b * p.ld + el.base;
    el.load();
    const float T0 = p.temperature ? p.temperature[b] : 1.f, mp0 = p.min_p ? p.min_p[b] : 0.f;
    const double T = fmax((double)T0, 1e-37), inv_T = 1.0 / T;
    // a weight is at least min_p when the logit is at most this far (negative) from the maximum
    double thr = -INFINITY;
    if (tid == 0 && mp0 > 0.f && T < 1e300) thr = T * log(fmin((double)mp0, 1.0));

    // the smallest of one 32-bit word per thread, over the cluster
    auto cluster_min = [&](uint32_t v, int slot) {
        v = __reduce_min_sync(0xffffffffu, v);
        if (lane == 0) s.key_w[warp] = v;
        __syncthreads();
        if (warp == 0) {
            v = __reduce_min_sync(0xffffffffu, lane < kWarps ? s.key_w[lane] : 0xffffffffu);
            if (lane < C) cluster.map_shared_rank(&s.key[slot][0], lane)[rank] = v;
        }
        cluster.sync();
        return __reduce_min_sync(0xffffffffu, lane < C ? s.key[slot][lane] : 0xffffffffu);
    };

    // ---- maximum
    float mx = -INFINITY;
    el.each(false, [&](float x, int) { mx = fmaxf(mx, x); });
    cluster.barrier_wait();
    mx = value_of(cluster_min(key_of(mx), 0));
    if (rank == 0 && tid == 0 && p.pos) p.pos[b] += 1;
    if (mx == -INFINITY || !(T0 > 0.f)) {  // nothing to choose from, or greedy: the first of the largest
        int at = 0x7fffffff;
        if (mx > -INFINITY) {
            el.each(false, [&](float x, int i) { at = x == mx ? min(at, i) : at; });
            at = (int)cluster_min((uint32_t)at, 1);
        } else {
            at = -1;
        }
        if (rank == 0 && tid == 0) p.tokens[b] = at;
        return;  // (nothing of another CTA's shared memory is touched after a sync)
    }
    const bool infinite = mx == INFINITY;
    if (infinite) {  // infinities share all the weight: they become the only candidates
#pragma unroll
        for (int j = 0; j < kRegs; ++j) el.x[j] = el.x[j] == INFINITY ? 0.f : -INFINITY;
        mx = 0.f;
    }
    const double m = (double)mx;
    Row r;
    r.m = mx;
    r.inv_T2 = (float)(2.0 * inv_T);
    r.inv_Tl2 = (float)(1.4426950408889634 * inv_T);
    {
        // two lanes' columns of a bin's upper end per thread; its weight once
        const int bin = tid >> 4;
        const float X = T > 1e300 ? mx : (float)fmin(fmax(m - 0.5 * (bin - 0.5) * T, -(double)FLT_MAX), (double)FLT_MAX);
        s.X[bin][2 * (tid & 15)] = X;
        s.X[bin][2 * (tid & 15) + 1] = X;
        if ((tid & 15) == 0) s.W[bin] = kUnit * exp(((double)X - m) * inv_T);
        if (tid == 0) s.thr = fmaxf(__double2float_ru(m + thr), -FLT_MAX) + 0.f;
    }
    __syncthreads();
    // the kept prefix: elements above lim_x, and those equal to it with an index up to lim_i
    constexpr int kAll = 0x7fffffff;
    float lim_x = s.thr;
    int lim_i = kAll;
    int par = 0, turn = 0;

    // Adds one lane-private histogram up over the cluster: every warp of every CTA gets the total of bin `lane`; the CTAs' parts
    // stay in s.xch[par ^ 1] until the next but one.
    auto totals = [&]() {
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kBins / kWarps; ++q) {
            const int bin = warp * (kBins / kWarps) + q;
            uint32_t lo = 0, hi = 0;  // (two warps' sums of a lane have 31 bits at most)
#pragma unroll
            for (int w = 0; w < kSlices; ++w) {
                const uint32_t v = s.hist[w][bin][lane];
                s.hist[w][bin][lane] = 0;
                lo += v & 0xffffu;
                hi += v >> 16;
            }
            lo = __reduce_add_sync(0xffffffffu, lo);
            hi = __reduce_add_sync(0xffffffffu, hi);
            if (lane < C)
                cluster.map_shared_rank(&s.xch[par][0][0], lane)[rank * kBins + bin] = ((unsigned long long)hi << 16) + lo;
        }
        cluster.sync();
        unsigned long long t = 0;
        for (int c = 0; c < C; ++c) t += s.xch[par][c][lane];
        par ^= 1;
        return t;
    };
    auto largest_part = [&](int bin) {  // of the totals just taken, the largest CTA's share of a bin
        unsigned long long v = 0;
        for (int c = 0; c < C; ++c) v = max(v, s.xch[par ^ 1][c][bin]);
        return (double)v;
    };
    const uint32_t my_hist = (uint32_t)__cvta_generic_to_shared(&s.hist[warp % kSlices][0][lane]);  // + bin * 128
    const uint32_t hist_a = my_hist - 0x4b000000u * 128u;                                              // + bin_bits * 128
    const char* const X_a = reinterpret_cast<const char*>(&s.X[0][lane]);

    // The bins of the whole row up to the limit.  Elements beyond it add nothing: no branches.
    auto level0 = [&](bool mass) {
        if (mass)
            el.each(infinite, [&](float x, int i) {
                const uint32_t o = r.bin_bits(x) * 128u;
                uint32_t u = r.units(x, *reinterpret_cast<const float*>(X_a + (o & (kBins * 128u - 1u))));
                if (!(x >= lim_x)) u = 0;
                if (lim_i != kAll && x == lim_x && i > lim_i) u = 0;
                red_add(hist_a + o, u);
            });
        else
            el.each(infinite, [&](float x, int) {  // (top-k comes first: no limit by index yet)
                red_add(hist_a + r.bin_bits(x) * 128u, x >= lim_x ? 1u : 0u);
            });
        return totals();
    };

    // A range of elements: values ka..kb (as keys, so descending), indices ia..ib once ka = kb.
    struct Range { uint32_t ka, kb; int ia, ib; };
    auto inside = [&](float x, int i, const Range& g) {  // (of an element whose value is in the range)
        return (x != lim_x || i <= lim_i) && i >= g.ia && i <= g.ib;
    };
    // The smallest key whose bin is at least j.  It lies next to that of the bin's upper end: 32 probes around it nearly
    // always hold it; if not (values near zero have finer keys), the whole range is searched, 32 probes a round.
    auto first_key = [&](int j) -> uint32_t {
        const uint32_t k0 = key_of(r.m), k1 = key_of(-FLT_MAX) + 1;  // the answer is in k0..k1
        if (j <= 0) return k0;
        if (j >= kBins) return k1;
        {
            const uint32_t mid = key_of(s.X[j][0] + 0.f), a = mid > k0 + 16 ? mid - 16 : k0, at = a + lane;
            const unsigned ok = __ballot_sync(0xffffffffu, at >= k1 || r.bin(value_of(at)) >= j);
            if (ok && (!(ok & 1u) || a == k0)) return a + __ffs(ok) - 1;
        }
        uint32_t a = k0, e = k1;
        while (a < e) {
            const uint32_t step = (e - a + 31) / 32;
            const unsigned long long at = (unsigned long long)a + (unsigned long long)lane * step;
            const unsigned ok = __ballot_sync(0xffffffffu, at >= e || r.bin(value_of((uint32_t)at)) >= j);
            const int f = __ffs(ok) - 1;  // (-1: none)
            if (f < 0) { a += 31 * step + 1; continue; }
            if (f == 0) { e = a; break; }
            e = (uint32_t)min((unsigned long long)e, (unsigned long long)a + (unsigned long long)f * step);
            a += (f - 1) * step + 1;
        }
        return a;
    };
    auto range_of_bin = [&](int j) {
        const uint32_t a = first_key(j), e = first_key(j + 1);
        return Range{a, max(a, min(e - 1, key_of(lim_x))), 0, kAll};
    };

    // Copies this CTA's elements of a range to s.loc (the caller knows that they fit).
    auto compact = [&](const Range& g) {
        const float xa = value_of(g.ka), xb = value_of(g.kb);
        if (tid == 0) s.nloc = 0;
        __syncthreads();
        uint32_t mask = 0;
#pragma unroll
        for (int j = 0; j < kRegs; ++j) mask |= (el.x[j] <= xa && el.x[j] >= xb) ? 1u << j : 0u;
        if (lim_i != kAll || g.ia > 0 || g.ib != kAll) {
#pragma unroll
            for (int j = 0; j < kRegs; ++j)
                if (!inside(el.x[j], el.base + el.local(j), g)) mask &= ~(1u << j);
        }
        const uint32_t cnt = __popc(mask), upto = warp_scan(cnt, lane);
        uint32_t at = 0;
        if (lane == 31 && upto) at = atomicAdd(&s.nloc, upto);
        at = __shfl_sync(0xffffffffu, at, 31) + upto - cnt;
        if (__any_sync(0xffffffffu, mask != 0)) {
#pragma unroll
            for (int j = 0; j < kRegs; ++j)
                if (mask & (1u << j)) {
                    if (at < kLocal) s.loc[at] = make_uint2(__float_as_uint(el.x[j]), (uint32_t)(el.base + el.local(j)));
                    ++at;
                }
        }
        el.rest(infinite, [&](float x, int i) {
            if (x <= xa && x >= xb && inside(x, i, g)) {
                const uint32_t q = atomicAdd(&s.nloc, 1u);
                if (q < kLocal) s.loc[q] = make_uint2(__float_as_uint(x), (uint32_t)i);
            }
        });
        __syncthreads();
    };
    auto local_inside = [&](const uint2& v, const Range& g, uint32_t& k, int& i) {
        k = key_of(__uint_as_float(v.x));
        i = (int)v.y;
        return k >= g.ka && k <= g.kb && i >= g.ia && i <= g.ib;
    };
    // Counts the elements of a range (the weights of the open last bin say nothing about that).
    auto tally = [&](const Range& g, bool local, double& tot, double& part) {
        uint32_t n = 0, k;
        int i;
        if (local) {
            for (uint32_t e = tid; e < min(s.nloc, (uint32_t)kLocal); e += kThreads) n += local_inside(s.loc[e], g, k, i);
        } else {
            const float xa = value_of(g.ka), xb = value_of(g.kb);
            el.each(infinite, [&](float x, int i) { n += x <= xa && x >= xb && inside(x, i, g); });
        }
        red_add(my_hist, n);
        const unsigned long long t = totals();
        tot = (double)__shfl_sync(0xffffffffu, t, 0);
        part = largest_part(0);
    };
    // Brings the local elements of a range together in every CTA: CTA c's go to slots 64 c .. (the caller knows that no
    // CTA has more).
    auto gather = [&](const Range& g) {
        if (tid == 0) s.lcnt = 0;
        __syncthreads();
        const uint32_t nloc = min(s.nloc, (uint32_t)kLocal);
        for (uint32_t e0 = warp * 32; e0 < nloc; e0 += kThreads) {
            const uint32_t e = e0 + lane;
            uint32_t k = 0;
            int i = 0;
            const bool in = e < nloc && local_inside(s.loc[e], g, k, i);
            const unsigned who = __ballot_sync(0xffffffffu, in);
            if (!who) continue;
            uint32_t at = 0;
            if (lane == 0) at = atomicAdd(&s.lcnt, (uint32_t)__popc(who));
            at = __shfl_sync(0xffffffffu, at, 0) + __popc(who & ((1u << lane) - 1u));
            if (in && at < kSlot) s.tmp[at] = ((unsigned long long)k << 32) | (uint32_t)i;
        }
        __syncthreads();
        const uint32_t n = min(s.lcnt, (uint32_t)kSlot), c = tid / kSlot, e = tid % kSlot;
        if (c < C) {
            if (e < n) cluster.map_shared_rank(&s.list[turn][0], c)[rank * kSlot + e] = s.tmp[e];
            if (e == 0) cluster.map_shared_rank(&s.cnt[turn][0], c)[rank] = n;
        }
        cluster.sync();
        turn ^= 1;
        int all = 0;
        for (int q = 0; q < C; ++q) all += (int)s.cnt[turn ^ 1][q];
        return all;
    };
    // The collected elements in order, element e in thread e: each counts those before it.
    auto sorted = [&](int n) {
        const unsigned long long* list = s.list[turn ^ 1];
        const uint32_t* cnt = s.cnt[turn ^ 1];
        const int c0 = tid / kSlot;
        const bool mine = c0 < C && (uint32_t)(tid % kSlot) < cnt[c0];
        if (__any_sync(0xffffffffu, mine)) {
            const unsigned long long k = mine ? list[tid] : ~0ull;
            int before = 0;
            for (int c = 0; c < C; ++c) {
                const int m = (int)cnt[c];
                const unsigned long long* l = list + c * kSlot;
#pragma unroll 8
                for (int e = 0; e < m; ++e) before += l[e] < k;
            }
            if (mine) s.tmp[before] = k;
        }
        __syncthreads();
        return tid < n ? s.tmp[tid] : ~0ull;
    };
    // Running sum of the elements' weights, on top of `before`.
    auto summed = [&](int n, unsigned long long k, double before, double& w) {
        w = 0.0;
        if (tid < n) {
            const float x = value_of((uint32_t)(k >> 32));
            const int bin = r.bin(x);
            w = s.W[bin] * (double)r.units(x, s.X[bin][0]);
        }
        const double run = warp_scan(w, lane);
        if (lane == 31) s.scan[warp] = run;
        __syncthreads();
        const int nw = min(warp, (n + 31) / 32);
        for (int v = 0; v < nw; ++v) before += s.scan[v];
        return before + run;
    };
    // The first of the elements 0..n-1 whose running sum is above (strict) or at least t; the last one if none is.
    auto first_at = [&](int n, unsigned long long k, double run, double t, bool strict) {
        if (tid == 0) s.hit = max(n - 1, 0);
        __syncthreads();
        const unsigned ok = __ballot_sync(0xffffffffu, tid < n && (strict ? run > t : run >= t));
        if (ok && lane == 0) atomicMin(&s.hit, warp * 32 + __ffs(ok) - 1);
        __syncthreads();
        const int h = s.hit;
        if (tid == h) s.res = Result{value_of((uint32_t)(k >> 32)), (int)(uint32_t)k, run};
        __syncthreads();
        return h;
    };
    const float u0 = p.u[b], one = 0.99999994f;
    const double u = u0 >= 0.f ? (double)fminf(u0, one) : (u0 < 0.f ? 0.0 : (double)one);
    const float tp0 = p.top_p ? p.top_p[b] : 1.f;
    const bool nucleus = tp0 < 1.f;
    const double tp = (double)fmaxf(tp0, 0.f);

    // Narrows a range of bin j around the target until its elements can be collected; `before` is the running sum in front of
    // it, tot and part about how many elements the cluster and the fullest CTA have in it.  Returns the number collected.
    auto narrow = [&](Range g, int j, bool by_rank, double target, bool strict, double& before, double tot, double part) {
        bool local = false;
        const bool open = !by_rank && j == kBins - 1;  // (weights there may be anything down to 0)
        for (int level = 0; level < 16; ++level) {
            if (open) tally(g, local, tot, part);
            if (!local && part <= kLocal) {
                compact(g);
                local = true;
            }
            if (local && part <= kSlot && tot <= kSorted) return gather(g);
            // 32 parts of its values, or of its indices where there is only one value
            const bool by_value = g.ka != g.kb;
            if (!by_value && g.ib == kAll) g.ib = p.V - 1;
            const uint32_t lo = by_value ? g.ka : (uint32_t)g.ia, span = by_value ? g.kb - g.ka : (uint32_t)(g.ib - g.ia);
            const int sh = max(0, 32 - __clz(span) - 5);
            const float X = s.X[j][0];
            if (local) {
                for (uint32_t e = tid; e < min(s.nloc, (uint32_t)kLocal); e += kThreads) {
                    uint32_t k;
                    int i;
                    if (local_inside(s.loc[e], g, k, i))
                        red_add(my_hist + (((by_value ? k : (uint32_t)i) - lo) >> sh) * 128u, by_rank ? 1u : r.units(value_of(k), X));
                }
            } else {
                const float xa = value_of(g.ka), xb = value_of(g.kb);
                el.each(infinite, [&](float x, int i) {
                    if (x <= xa && x >= xb)
                        if (inside(x, i, g))
                            red_add(my_hist + (((by_value ? key_of(x) : (uint32_t)i) - lo) >> sh) * 128u, by_rank ? 1u : r.units(x, X));
                });
            }
            const unsigned long long t = totals();
            const double w = by_rank ? (double)t : s.W[j] * (double)t, run = warp_scan(w, lane);
            const unsigned ok = __ballot_sync(0xffffffffu, t > 0 && (strict ? before + run > target : before + run >= target));
            const unsigned any = __ballot_sync(0xffffffffu, t > 0);
            const int cut = ok ? __ffs(ok) - 1 : 31 - __clz(any | 1u);
            before += __shfl_sync(0xffffffffu, run - w, cut);
            const double per = by_rank ? 1.0 : 1.7 * kUnit;  // elements per unit: a weight inside a bin is at least exp(-1/2)
            tot = per * __shfl_sync(0xffffffffu, (double)t, cut);
            part = per * largest_part(cut);
            const uint32_t a = lo + ((uint32_t)cut << sh), last = (uint32_t)min((unsigned long long)a + (1u << sh) - 1, (unsigned long long)lo + span);
            if (by_value) { g.ka = a; g.kb = last; }
            else { g.ia = (int)a; g.ib = (int)last; }
        }
        return 0;  // (not reached: 52 bits of value and index, five a level)
    };

    // ---- top-k: the value and index of the last candidate it keeps
    const int k = p.top_k ? p.top_k[b] : 0;
    if (k > 0 && k < p.V) {
        const unsigned long long t = level0(false);
        const uint32_t run = warp_scan((uint32_t)t, lane);
        const unsigned ok = __ballot_sync(0xffffffffu, run >= (uint32_t)k);
        if (ok) {  // (else there are no more than k candidates)
            const int j = __ffs(ok) - 1;
            const uint32_t upto = __shfl_sync(0xffffffffu, run, j), in = __shfl_sync(0xffffffffu, (uint32_t)t, j);
            Range g = range_of_bin(j);
            uint32_t most = 0;  // elements of the fullest CTA up to this bin
            for (int c = 0; c < C; ++c)
                most = max(most, __reduce_add_sync(0xffffffffu, lane <= j ? (uint32_t)s.xch[par ^ 1][c][lane] : 0u));
            if (upto <= kSorted && most <= kSlot) {  // few enough from the top down: the rest happens in the list
                g.ka = key_of(r.m);
                compact(g);
                const int n = gather(g);
                const unsigned long long e = sorted(n);
                double w;
                const double cum = summed(n, e, 0.0, w);
                int kept = min(k, n);
                if (tid == kept - 1) s.res.mass = cum;
                __syncthreads();
                double Z = s.res.mass;
                if (nucleus) {
                    kept = 1 + first_at(kept, e, cum, tp * Z, false);
                    Z = s.res.mass;
                }
                first_at(kept, e, cum, u * Z, true);
                if (rank == 0 && tid == 0) p.tokens[b] = s.res.i;
                return;
            }
            double before = (double)(upto - in);
            const double part = largest_part(j);
            const int n = narrow(g, j, true, (double)k, false, before, (double)in, part);
            const unsigned long long e = sorted(n);
            if (tid == max(0, min(n, k - (int)before) - 1)) s.res = Result{value_of((uint32_t)(e >> 32)), (int)(uint32_t)e, 0.0};
            __syncthreads();
            lim_x = s.res.x;
            lim_i = s.res.i;
        }
    }

    // ---- weights of the bins; lane j: bin j
    const unsigned long long t = level0(true);
    const double w0 = s.W[lane] * (double)t, run0 = warp_scan(w0, lane);
    const unsigned any0 = __ballot_sync(0xffffffffu, t > 0);
    const int par0 = par ^ 1;
    unsigned long long most = 0;  // the fullest CTA's share of bin `lane`
    for (int c = 0; c < C; ++c) most = max(most, s.xch[par0][c][lane]);
    double Z = __shfl_sync(0xffffffffu, run0, 31);
    // Element at which the running sum reaches a target: its place and the sum go to s.res.
    auto search = [&](double target, bool strict) {
        const unsigned ok = __ballot_sync(0xffffffffu, t > 0 && (strict ? run0 > target : run0 >= target));
        const int j = ok ? __ffs(ok) - 1 : 31 - __clz(any0 | 1u);
        double before = __shfl_sync(0xffffffffu, run0 - w0, j);
        const double tot = 1.7 * kUnit * (double)__shfl_sync(0xffffffffu, t, j), part = 1.7 * kUnit * (double)__shfl_sync(0xffffffffu, most, j);
        const int n = narrow(range_of_bin(j), j, false, target, strict, before, tot, part);
        const unsigned long long e = sorted(n);
        double w;
        const double cum = summed(n, e, before, w);
        first_at(n, e, cum, target, strict);
    };
    if (nucleus) {
        search(tp * Z, false);
        lim_x = s.res.x;
        lim_i = s.res.i;
        Z = s.res.mass;
    }
    search(u * Z, true);
    if (rank == 0 && tid == 0) p.tokens[b] = s.res.i;
}

}  // namespace

cudaError_t sample_launch(const SampleArgs& a, cudaStream_t st, bool pdl) {
    // as many CTAs as hold the row in registers (a power of two, eight at most)
    int C = 1;
    while (C < kCluster && (int64_t)C * kThreads * kRegs < a.V) C *= 2;
    const bool vec = reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 && (a.B == 1 || a.ld % 4 == 0);
    auto kern = vec ? sample_rows<true> : sample_rows<false>;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem));
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(a.B * C);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(Smem);
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = C;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, a);
}

}  // namespace first

using namespace first;

extern "C" int first_sample(const float* logits, int64_t row_stride, int32_t B, int32_t vocab, const float* temperature,
                            const int32_t* top_k, const float* top_p, const float* min_p, const float* uniforms,
                            int32_t* tokens, void* stream) {
    if (B < 0 || vocab <= 0) return FIRST_E_ARG;
    if (B == 0) return FIRST_OK;
    if (!logits || !uniforms || !tokens) return FIRST_E_ARG;
    if (vocab > FIRST_SAMPLE_MAX_VOCAB) return FIRST_E_UNSUPPORTED;
    if (B > 1 && row_stride < vocab) return FIRST_E_SHAPE;
    SampleArgs a;
    a.logits = logits; a.ld = row_stride; a.B = B; a.V = vocab;
    a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p; a.u = uniforms;
    a.tokens = tokens;
    return sample_launch(a, static_cast<cudaStream_t>(stream), false) == cudaSuccess ? FIRST_OK : FIRST_E_CUDA;
}
