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
//   4. What is left, at most kList elements, goes to the first CTA's shared memory, is sorted there and summed up.
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
constexpr int kList = 1024;          // elements that are sorted in shared memory (two a thread)
constexpr int kGathers = 64;         // attempts to collect a list, at most: 3 searches of up to 12 levels each
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

struct Best { float x; int i; };

struct Result {  // of a search: where the kept prefix ends, and its weight
    float x;     // the last kept element's value ...
    int i;       // ... and index: elements of that value with a larger one are not kept
    double mass;
};

struct Smem {
    uint32_t hist[kWarps][kBins][32];
    unsigned long long list[kList], sorted[kList];
    double cum[kList];
    unsigned long long xch[2][kCluster][kBins];
    double W[kBins];                 // weight of a bin's upper end, per unit
    float X[kBins];                  // a bin's upper end
    Best best[kCluster], best_w[kWarps];
    double scan[kWarps];
    Result res;
    unsigned int gcnt[kGathers];     // (first CTA) elements collected by each attempt
    unsigned int lcnt, loff;
    int hit;
    float thr;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

struct Row {  // what a thread needs to know about the row
    float m, inv_T2, inv_Tl2;  // maximum; 2 / T (bins of half a unit), log2(e) / T
};

__device__ __forceinline__ int bin_of(float x, const Row& r) {  // (monotone in x, like every step of it)
    return (int)(__float_as_uint(fminf((r.m - x) * r.inv_T2, (float)(kBins - 1)) + 8388608.f) & (kBins - 1));
}
// weight of x in units of 2^-23 of its bin's weight
__device__ __forceinline__ uint32_t units_of(float x, float X, const Row& r) {
    const float d = fmaxf(fminf(X - x, FLT_MAX) * r.inv_Tl2, -1.f);  // (X - x is exact but where it does not matter)
    return __float_as_uint(ex2(-d) + 1.f) - 0x3f800000u;
}

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
    // f(value, index in the row); values are clean, elements that do not exist are -inf
    template <typename F>
    __device__ __forceinline__ void each(bool infinite, F f) const {
#pragma unroll
        for (int j = 0; j < kRegs; ++j) f(x[j], base + local(j));
        for (int i = kRegs * kThreads + (int)threadIdx.x; i < n; i += kThreads) {
            float v = clean(row[i]);
            if (infinite) v = v == INFINITY ? 0.f : -INFINITY;
            f(v, base + i);
        }
    }
};

__device__ __forceinline__ unsigned long long warp_sum_u64(unsigned long long v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// grid B * C in clusters of C; one cluster per row.
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
        if (tid < kGathers) s.gcnt[tid] = 0;
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
    const float T0 = p.temperature ? p.temperature[b] : 1.f;

    // ---- maximum, and its first index
    Best me{-INFINITY, 0x7fffffff};
    el.each(false, [&](float x, int i) {
        if (x > me.x) { me.x = x; me.i = i; }  // (a thread's indices ascend)
    });
    auto better = [](const Best& a, const Best& c) { return a.x > c.x || (a.x == c.x && a.i < c.i); };
    auto warp_best = [&](Best v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const Best w{__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.i, o)};
            if (better(w, v)) v = w;
        }
        return v;
    };
    me = warp_best(me);
    if (lane == 0) s.best_w[warp] = me;
    __syncthreads();
    cluster.barrier_wait();
    if (warp == 0) {
        me = warp_best(lane < kWarps ? s.best_w[lane] : Best{-INFINITY, 0x7fffffff});
        if (lane < C) cluster.map_shared_rank(s.best, lane)[rank] = me;
    }
    cluster.sync();
    me = warp_best(lane < C ? s.best[lane] : Best{-INFINITY, 0x7fffffff});
    if (rank == 0 && tid == 0 && p.pos) p.pos[b] += 1;
    if (me.x == -INFINITY || !(T0 > 0.f)) {  // nothing to choose from, or greedy
        if (rank == 0 && tid == 0) p.tokens[b] = me.x == -INFINITY ? -1 : me.i;
        return;  // (nothing of another CTA's shared memory is touched after the sync)
    }
    const bool infinite = me.x == INFINITY;
    if (infinite) {  // infinities share all the weight: they become the only candidates
#pragma unroll
        for (int j = 0; j < kRegs; ++j) el.x[j] = el.x[j] == INFINITY ? 0.f : -INFINITY;
        me.x = 0.f;
    }
    const double T = fmax((double)T0, 1e-37), m = (double)me.x, inv_T = 1.0 / T;
    Row r;
    r.m = me.x;
    r.inv_T2 = (float)(2.0 * inv_T);
    r.inv_Tl2 = (float)(1.4426950408889634 * inv_T);
    if (tid < kBins) {
        const float X = T > 1e300 ? me.x : (float)fmin(fmax(m - 0.5 * (tid - 0.5) * T, -(double)FLT_MAX), (double)FLT_MAX);
        s.X[tid] = X;
        s.W[tid] = kUnit * exp(((double)X - m) * inv_T);
    }
    // the smallest value that min_p keeps
    const float mp0 = p.min_p ? p.min_p[b] : 0.f;
    if (tid == 32) {
        float x = -FLT_MAX;
        if (mp0 > 0.f && T < 1e300) {
            const double mp = fmin((double)mp0, 1.0);
            auto kept = [&](float v) { return exp(((double)v - m) / T) >= mp; };
            x = (float)fmax(m + T * log(mp), -(double)FLT_MAX);
            for (int i = 0; i < 4 && x > -FLT_MAX && kept(nextafterf(x, -INFINITY)); ++i) x = nextafterf(x, -INFINITY);
            for (int i = 0; i < 4 && x < me.x && !kept(x); ++i) x = nextafterf(x, INFINITY);
            x = fminf(x, me.x);
        }
        s.thr = x + 0.f;
    }
    __syncthreads();
    // the kept prefix: elements above lim_x, and those equal to it with an index up to lim_i
    float lim_x = s.thr;
    int lim_i = 0x7fffffff;
    int par = 0, gathers = 0;

    // Adds one lane-private histogram up over the cluster: every warp of every CTA gets the total of bin `lane`.
    auto totals = [&]() {
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kBins / kWarps; ++q) {
            const int bin = warp * (kBins / kWarps) + q;
            unsigned long long v = 0;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                v += s.hist[w][bin][lane];
                s.hist[w][bin][lane] = 0;
            }
            v = warp_sum_u64(v);
            if (lane < C) cluster.map_shared_rank(&s.xch[par][0][0], lane)[rank * kBins + bin] = v;
        }
        cluster.sync();
        unsigned long long t = 0;
        for (int c = 0; c < C; ++c) t += s.xch[par][c][lane];
        par ^= 1;
        return t;
    };
    uint32_t* const my_hist = &s.hist[warp][0][lane];

    // A range of elements: values ka..kb (as keys, so descending), indices ia..ib once ka = kb.
    struct Range { uint32_t ka, kb; int ia, ib; };
    auto inside = [&](float x, int i, float xa, float xb, const Range& g) {
        return x <= xa && x >= xb && (x != lim_x || i <= lim_i) && i >= g.ia && i <= g.ib;
    };

    // The bins of the whole row up to the limit.
    auto level0 = [&](bool mass) {
        el.each(infinite, [&](float x, int i) {
            if (x >= lim_x && (x != lim_x || i <= lim_i)) {
                const int bin = bin_of(x, r);
                my_hist[bin * 32] += mass ? units_of(x, s.X[bin], r) : 1u;
            }
        });
        return totals();
    };
    // The values of bin j: the first and the last key with bin_of = j, searched by a whole warp (32 probes a round).
    auto first_key = [&](int j) {  // smallest key whose bin is at least j
        unsigned long long a = key_of(r.m), e = (unsigned long long)key_of(-FLT_MAX) + 1;  // the answer is in [a, e]
        while (a < e) {
            const unsigned long long step = (e - a + 31) / 32, at = a + lane * step;
            const unsigned ok = __ballot_sync(0xffffffffu, at >= e || bin_of(value_of((uint32_t)at), r) >= j);
            const int f = __ffs(ok) - 1;  // (0: none true)
            if (f < 0) { a = a + 31 * step + 1; continue; }
            e = a + f * step < e ? a + f * step : e;
            if (f > 0) a = a + (unsigned long long)(f - 1) * step + 1;
            else e = a;
        }
        return a;
    };
    auto range_of_bin = [&](int j) {
        const unsigned long long a = first_key(j), e = first_key(j + 1);
        return Range{(uint32_t)a, (uint32_t)(e > a ? e - 1 : a), 0, 0x7fffffff};
    };

    // Collects the elements of a range in the first CTA; returns how many there are (more than kList: not collected).
    auto gather = [&](const Range& g) {
        const float xa = value_of(g.ka), xb = value_of(g.kb);
        if (tid == 0) s.lcnt = 0;
        __syncthreads();
        el.each(infinite, [&](float x, int i) {
            if (inside(x, i, xa, xb, g)) {
                const unsigned at = atomicAdd(&s.lcnt, 1u);
                if (at < kList) s.sorted[at] = ((unsigned long long)key_of(x) << 32) | (unsigned)i;
            }
        });
        __syncthreads();
        const unsigned n = s.lcnt;
        unsigned* cnt = cluster.map_shared_rank(s.gcnt, 0) + gathers;
        if (tid == 0 && n) s.loff = atomicAdd(cnt, n);
        __syncthreads();
        if (n) {
            unsigned long long* dst = cluster.map_shared_rank(s.list, 0);
            for (unsigned e = tid; e < n && e < kList; e += kThreads)
                if (s.loff + e < kList) dst[s.loff + e] = s.sorted[e];
        }
        cluster.sync();
        ++gathers;
        return *static_cast<volatile unsigned*>(cnt);
    };
    // (first CTA) Sorts the n collected elements by (value, index): every element counts those before it.
    auto sort_list = [&](int n) {
        __syncthreads();
        unsigned long long k0 = tid < n ? s.list[tid] : ~0ull, k1 = tid + kThreads < n ? s.list[tid + kThreads] : ~0ull;
        int r0 = 0, r1 = 0;
        if (n > kThreads) {
            for (int e = 0; e < n; ++e) {
                const unsigned long long k = s.list[e];
                r0 += k < k0;
                r1 += k < k1;
            }
        } else if (tid < (n + 31) / 32 * 32) {
#pragma unroll 4
            for (int e = 0; e < n; ++e) r0 += s.list[e] < k0;
        }
        if (tid < n) s.sorted[r0] = k0;
        if (tid + kThreads < n) s.sorted[r1] = k1;
        __syncthreads();
    };
    // (first CTA) Running sums of the sorted elements' weights, on top of `before`.
    auto sum_list = [&](int n, double before) {
        double w[2], mine = 0.0;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int e = 2 * tid + q;
            w[q] = 0.0;
            if (e < n) {
                const float x = value_of((uint32_t)(s.sorted[e] >> 32));
                const int bin = bin_of(x, r);
                w[q] = s.W[bin] * (double)units_of(x, s.X[bin], r);
            }
            mine += w[q];
        }
        double run = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double v = __shfl_up_sync(0xffffffffu, run, o);
            if (lane >= o) run += v;
        }
        if (lane == 31) s.scan[warp] = run;
        __syncthreads();
        double off = before;
        for (int w2 = 0; w2 < warp; ++w2) off += s.scan[w2];
        run = off + run - mine;
        if (2 * tid < n) s.cum[2 * tid] = run + w[0];
        if (2 * tid + 1 < n) s.cum[2 * tid + 1] = run + w[0] + w[1];
        __syncthreads();
    };
    // (first CTA) The first of the elements 0..n-1 whose running sum is above (strict) or at least t; the last one if none is.
    auto first_at = [&](int n, double t, bool strict) {
        if (tid == 0) s.hit = n - 1;
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int e = 2 * tid + q;
            if (e < n && (strict ? s.cum[e] > t : s.cum[e] >= t)) { atomicMin(&s.hit, e); break; }
        }
        __syncthreads();
        const int h = s.hit;
        __syncthreads();
        return h;
    };
    const float u0 = p.u[b], one = 0.99999994f;
    const double u = u0 >= 0.f ? (double)fminf(u0, one) : (u0 < 0.f ? 0.0 : (double)one);
    const float tp0 = p.top_p ? p.top_p[b] : 1.f;
    const bool nucleus = tp0 < 1.f;
    const double tp = (double)fmaxf(tp0, 0.f);
    auto finish = [&](int e) {
        if (tid == 0) p.tokens[b] = (int)(uint32_t)s.sorted[max(e, 0)];
    };
    // The other CTAs may leave once they have read what the first one holds; the first one leaves after them.
    auto leave = [&]() {
        cluster.barrier_arrive();
        if (rank == 0) cluster.barrier_wait();
    };

    // Narrows a range of bin j (its elements' running sum starts at `before`) around the target until it can be
    // collected; the first CTA then holds it sorted, with running sums.  Returns the number of elements.
    auto narrow = [&](Range g, int j, bool by_rank, double target, bool strict, double& before, double expect) {
        for (int level = 0; level < 16; ++level) {
            if (expect <= kList) {
                const int n = (int)gather(g);
                if (n <= kList) return n;
            }
            // 32 parts of its values, or of its indices where there is only one value
            const bool by_value = g.ka != g.kb;
            if (!by_value && g.ib == 0x7fffffff) g.ib = p.V - 1;
            const uint32_t lo = by_value ? g.ka : (uint32_t)g.ia, span = by_value ? g.kb - g.ka : (uint32_t)(g.ib - g.ia);
            const int sh = max(0, 32 - __clz(span) - 5);
            const float xa = value_of(g.ka), xb = value_of(g.kb), X = s.X[j];
            el.each(infinite, [&](float x, int i) {
                if (inside(x, i, xa, xb, g)) {
                    const uint32_t part = ((by_value ? key_of(x) : (uint32_t)i) - lo) >> sh;
                    my_hist[part * 32] += by_rank ? 1u : units_of(x, X, r);
                }
            });
            const unsigned long long t = totals();
            const double w = by_rank ? (double)t : s.W[j] * (double)t;
            double run = w;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double v = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += v;
            }
            const unsigned ok = __ballot_sync(0xffffffffu, t > 0 && (strict ? before + run > target : before + run >= target));
            const unsigned any = __ballot_sync(0xffffffffu, t > 0);
            const int part = ok ? __ffs(ok) - 1 : 31 - __clz(any | 1u);
            before += __shfl_sync(0xffffffffu, run - w, part);
            const double tt = __shfl_sync(0xffffffffu, (double)t, part);
            expect = by_rank ? tt : (j < kBins - 1 ? 1.7 * tt * kUnit : 0.0);  // (a weight inside a bin is at least exp(-1/2))
            const uint32_t a = lo + ((uint32_t)part << sh), last = (uint32_t)min((unsigned long long)a + (1u << sh) - 1, (unsigned long long)lo + span);
            if (by_value) { g.ka = a; g.kb = last; }
            else { g.ia = (int)a; g.ib = (int)last; }
        }
        return 0;  // (not reached: 52 bits of value and index, five a level)
    };

    // ---- top-k: the value and index of the last candidate it keeps
    const int k = p.top_k ? p.top_k[b] : 0;
    if (k > 0 && k < p.V) {
        const unsigned long long t = level0(false);
        uint32_t run = (uint32_t)t;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, run, o);
            if (lane >= o) run += v;
        }
        const unsigned ok = __ballot_sync(0xffffffffu, run >= (uint32_t)k);
        if (ok) {  // (else there are no more than k candidates)
            const int j = __ffs(ok) - 1;
            const uint32_t upto = __shfl_sync(0xffffffffu, run, j), in = __shfl_sync(0xffffffffu, (uint32_t)t, j);
            Range g = range_of_bin(j);
            if (upto <= kList) {  // few enough from the top down: the rest happens in the list
                g.ka = key_of(r.m);
                const int n = (int)gather(g);
                if (rank == 0) {
                    sort_list(n);
                    sum_list(n, 0.0);
                    int kept = min(k, n);
                    if (nucleus) kept = 1 + first_at(kept, tp * s.cum[kept - 1], false);
                    finish(first_at(kept, u * s.cum[kept - 1], true));
                }
                leave();
                return;
            }
            double before = (double)(upto - in);
            const int n = narrow(g, j, true, (double)k, false, before, (double)in);
            if (rank == 0) {
                sort_list(n);
                if (tid < C) {
                    const unsigned long long e = s.sorted[max(0, min(n, k - (int)before) - 1)];
                    Result* to = cluster.map_shared_rank(&s.res, tid);
                    to->x = value_of((uint32_t)(e >> 32));
                    to->i = (int)(uint32_t)e;
                }
            }
            cluster.sync();
            lim_x = s.res.x;
            lim_i = s.res.i;
        }
    }

    // ---- weights of the bins; lane j: bin j
    const unsigned long long t = level0(true);
    const double w = s.W[lane] * (double)t;
    double run = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double v = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += v;
    }
    const unsigned any = __ballot_sync(0xffffffffu, t > 0);
    double Z = __shfl_sync(0xffffffffu, run, 31);
    // bin of the first sum that reaches a target, the sum before it, and about how many elements it has
    auto find = [&](double target, bool strict, double& before, double& expect) {
        const unsigned ok = __ballot_sync(0xffffffffu, t > 0 && (strict ? run > target : run >= target));
        const int j = ok ? __ffs(ok) - 1 : 31 - __clz(any | 1u);
        before = __shfl_sync(0xffffffffu, run - w, j);
        expect = j < kBins - 1 ? 1.7 * kUnit * __shfl_sync(0xffffffffu, (double)t, j) : 0.0;
        return j;
    };
    double before, expect;
    if (nucleus) {
        const int j = find(tp * Z, false, before, expect);
        const int n = narrow(range_of_bin(j), j, false, tp * Z, false, before, expect);
        if (rank == 0) {
            sort_list(n);
            sum_list(n, before);
            const int e = max(first_at(n, tp * Z, false), 0);
            if (tid < C) {
                Result* to = cluster.map_shared_rank(&s.res, tid);
                to->x = value_of((uint32_t)(s.sorted[e] >> 32));
                to->i = (int)(uint32_t)s.sorted[e];
                to->mass = s.cum[e];
            }
        }
        cluster.sync();
        lim_x = s.res.x;
        lim_i = s.res.i;
        Z = s.res.mass;
    }
    const int j = find(u * Z, true, before, expect);
    const int n = narrow(range_of_bin(j), j, false, u * Z, true, before, expect);
    if (rank == 0) {
        sort_list(n);
        sum_list(n, before);
        finish(first_at(n, u * Z, true));
    }
    leave();
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
