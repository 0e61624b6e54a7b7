// Next tokens of a batch with generation settings of its own for every request (the paper samples with temperature
// 0.8 and top-k 10, appendix "Training and Inference Setup"; requests of one batch need not agree on that).
//
// A row's candidates stand in descending order of their logits, equal ones by index.  Every filter keeps a prefix of
// that order, and so does a draw: the token is the first candidate whose cumulative weight exceeds u times the sum.
// All of them are the same question -- where does a running sum (of ones, or of weights) reach a target -- and it is
// answered without sorting the row:
//   1. One thread-block cluster per row; the row is read once and stays in the cluster's shared memory.
//   2. A histogram over 32 bins of (max - x) / T, half a unit wide: the sum reaches the target in one of them.
//   3. That bin's elements are copied out, with all above them if there is room: the searches after this one then look
//      there only, and if they are few thousand the first CTA takes them all and the others leave.
//   4. If there are many, their range of values is cut into 32 parts (and again, and, among equal values, that of their
//      indices), each time keeping the part that holds the target.
//   5. What is left, at most kSorted elements, is sorted in shared memory and summed up.
// A histogram is private to every lane (a bin is 32 words, a lane owns one): a bank each, and integer sums, which are the
// same in every run.  Weights are taken relative to that of the upper end X of their bin: exp((x - X) / T) with the
// difference exact, as integers in units of 2^-23, which keeps float32's 24 bits; the bins' own weights and all prefix
// sums are 64-bit floating point.
// Bound by the latency of these phases, one after the other with an exchange between the CTAs each: 10.6 us for one row of
// 128256 at top-k 10, 32 us for 32 rows with settings of their own, 161 us for 256 (0.82 TB/s: two rows' CTAs share a
// multiprocessor, the launch is seven waves of rows).
#include <cfloat>
#include <cooperative_groups.h>

#include "common.cuh"
#include "first.h"
#include "ops.h"

namespace first {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBlock = 16;           // elements a thread looks at at a time
constexpr int kHeld = 2 * kBlock * kThreads;  // elements that a CTA can hold in shared memory
constexpr int kCluster = 8;
constexpr int kBins = 32;
constexpr int kResident = 2 * kSMs;  // CTAs on the GPU at a time
constexpr int kLocal = 2560;         // elements that a CTA can copy to shared memory for a search
constexpr int kMoved = kHeld / 2;    // the same in the place of a row, once the row itself is not needed any more
constexpr int kList = 256;           // elements that are sorted in every CTA of a cluster; of each CTA an equal share
constexpr int kSorted = 224;         // longer lists are narrowed further first: sorting takes time with the square of them
constexpr int kSlices = 4;           // lane-private histograms of a CTA, each shared by four warps
constexpr double kUnit = 1.0 / 8388608.0;  // 2^-23

// descending: the largest logit has the smallest key; -0 equals +0
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return (b & 0x80000000u) ? b : ~(b | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? k : ~(k | 0x80000000u));
}

struct Result {  // the last element of a kept prefix, and the prefix's weight
    float x;
    int i;
    double mass;
};

// A range of elements: values ka..kb (as keys, so descending), indices ia..ib once ka = kb.
struct Range { uint32_t ka, kb; int ia, ib; };
struct Search {  // what the first warp has found out, for all
    double target, before;  // the sum that is looked for; the sum in front of the range
    float tot, part;        // about how many elements (not more) the range has in the cluster and in its fullest CTA
    float all, upto;        // the same of the range and all before it
    Range g;
    int j;                  // the range's bin, -1: nothing to search for
};

struct Smem {
    uint32_t hist[kSlices][kBins][32];
    uint2 loc[kLocal];               // this CTA's elements of the range that was copied last, (value key, index)
    unsigned long long list[2][kList];  // value key << 32 | index; turn by turn: a CTA may be at the next search while another still reads
    unsigned long long tmp[kList];
    uint32_t cnt[2][kCluster];
    unsigned long long xch[2][kCluster][kBins];
    double W[kBins];                 // weight of a bin's upper end, per unit
    double scan[kWarps];
    Result res;
    Search at;
    uint32_t key[2][kCluster * kWarps];
    unsigned long long bar[2];       // mbarriers of the exchanges, by turns
    uint32_t moved[kCluster];
    uint32_t nloc, lcnt;
    int hit, late;
    float thr;
    alignas(16) float row[4];        // (HELD) the CTA's elements, as many as there are; -inf up to a multiple of a block; later kMoved of the cluster's
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void red_add(uint32_t a, uint32_t v) { asm volatile("red.shared.add.u32 [%0], %1;" ::"r"(a), "r"(v)); }

// Exchanges between the CTAs of a cluster: words are written to another CTA's shared memory with their bytes counted on its
// mbarrier, so that one trip does it where a store and a cluster barrier take several (256 rows: 168 us with barriers, 162
// so).  Exchange n uses mbarrier and buffers n & 1: a CTA that sends exchange n + 2 has had
// everybody's n + 1, sent after they had read n.
constexpr uint32_t kPolls = 1u << 20;  // a wait gives up after so many polls
__device__ __forceinline__ uint32_t shared_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t in_cta(uint32_t a, int cta) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(cta));
    return r;
}
__device__ __forceinline__ void send(uint32_t to, uint32_t bar, uint32_t v) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.u32 [%0], %1, [%2];" ::"r"(to), "r"(v), "r"(bar) : "memory");
}
__device__ __forceinline__ void send(uint32_t to, uint32_t bar, unsigned long long v) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.u64 [%0], %1, [%2];" ::"r"(to), "l"(v), "r"(bar) : "memory");
}
__device__ __forceinline__ void expect_bytes(uint32_t bar, uint32_t n) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(n) : "memory");
}
__device__ __forceinline__ bool arrived(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}

struct Row {  // what a thread needs to know about the row
    float m, inv_T2, inv_Tl2;  // maximum; 2 / T (bins of half a unit), log2(e) / T
    float half_T, top;         // T / 2; upper end of the first bin, m + T / 4 - shift
    float shift;               // what a weight's argument is measured from: 0, or m where T is a few steps of m
    // 2^23 + bin, as a float (monotone in x, like every step of it; NaN lands in the last bin)
    __device__ __forceinline__ float bin_number(float x) const { return fminf((m - x) * inv_T2, (float)(kBins - 1)) + 8388608.f; }
    __device__ __forceinline__ int bin(float x) const { return (int)(__float_as_uint(bin_number(x)) & (kBins - 1)); }
    // a bin's upper end, above shift; rounded up, so that no element of the bin is above it
    __device__ __forceinline__ float end_of(float bin) const { return __fmaf_ru(-bin, half_T, top); }
    // Weight of x in units of 2^-23 of that of its bin's upper end X (x - shift - X is exact but where it does not matter; it
    // is above 0 by a rounding at most): at most 2^23 - 1, so that 512 of them have 32 bits.  That keeps a float32 weight's 24 bits,
    // and each is right to 2^-21 of itself, the hardware's exponential included; the errors of many weights cancel for the most
    // part.  Draws placed next to tokens' borders (50257 to 262144 tokens, spreads of 0 to 4 T) came out with another token
    // only when within 2^-26 of the sum, where a float32 draw itself has steps of 2^-24.  More bits (64-bit weights to 2^-31)
    // would take about twice the instructions of a pass over the row.
    __device__ __forceinline__ uint32_t units(float x, float X) const {
        return __float_as_uint(ex2(fminf((x - shift - X) * inv_Tl2, -2.5e-7f)) + 1.f) - 0x3f800000u;
    }
};
// Elements per unit of weight inside a bin (not the last), at most.  A bin is half a T wide and X lies at most two steps of
// the row's values above it, which are T / 128 each at the most (see shift): weights are at least exp(-0.516) = 1 / 1.675.
constexpr float kPerUnit = (float)(1.7 * kUnit);

// This thread's elements of the row.  HELD: the CTA keeps them in shared memory; otherwise every pass reads them again
// (from L2).  VEC: 16-byte loads.  Elements that do not exist are -inf.
template <bool HELD, bool VEC>
struct Slice {
    const float* row;  // the CTA's first element
    float* held;       // their copy
    int base, n;       // its index in the row; elements of the CTA

    static __device__ __forceinline__ int place(int e) {  // of a block's element, after the block's first one of thread 0
        return (e >> 2) * (4 * kThreads) + 4 * (int)threadIdx.x + (e & 3);
    }
    __device__ __forceinline__ void load(float (&v)[kBlock], int i0) const {
#pragma unroll
        for (int e = 0; e < kBlock; e += 4) {
            const int i = i0 + place(e);
            float4 w = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            if (VEC && i + 3 < n) w = *reinterpret_cast<const float4*>(row + i);
            else if (i < n) {
                w.x = row[i];
                if (i + 1 < n) w.y = row[i + 1];
                if (i + 2 < n) w.z = row[i + 2];
                if (i + 3 < n) w.w = row[i + 3];
            }
            v[e] = w.x; v[e + 1] = w.y; v[e + 2] = w.z; v[e + 3] = w.w;
        }
    }
    // The first pass: f(block) of every block, which are kept (HELD).
    template <typename F>
    __device__ __forceinline__ void first(F f) const {
        for (int i0 = 0; i0 < n; i0 += 2 * kBlock * kThreads) {
            float v[2][kBlock];
            load(v[0], i0);
            load(v[1], i0 + kBlock * kThreads);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                f(v[q]);
                if (HELD && i0 + q * kBlock * kThreads < n)
#pragma unroll
                    for (int e = 0; e < kBlock; e += 4)
                        *reinterpret_cast<float4*>(held + i0 + q * kBlock * kThreads + place(e)) = make_float4(v[q][e], v[q][e + 1], v[q][e + 2], v[q][e + 3]);
            }
        }
    }
    // f(block, index in the row of its place 0), for every block of the CTA
    template <typename F>
    __device__ __forceinline__ void blocks(F f) const {
        for (int i0 = 0; i0 < n; i0 += kBlock * kThreads) {
            float v[kBlock];
            if constexpr (HELD) {
#pragma unroll
                for (int e = 0; e < kBlock; e += 4) {
                    const float4 w = *reinterpret_cast<const float4*>(held + i0 + place(e));
                    v[e] = w.x; v[e + 1] = w.y; v[e + 2] = w.z; v[e + 3] = w.w;
                }
            } else {
                load(v, i0);
            }
            f(v, base + i0);
        }
    }
    // f(value, index in the row) of every element, one by one: for what is done seldom
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll 4
        for (int i = (int)threadIdx.x; i < n; i += kThreads) f(HELD ? held[i] : row[i], base + i);
    }
};

template <typename T>
__device__ __forceinline__ T warp_scan(T run, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T v = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += v;
    }
    return run;
}

// grid B * C in clusters of C; one cluster per row.  Every decision is taken by the first warp of every CTA from the same
// numbers, so the cluster stays together without anyone telling the others.
template <bool HELD, bool VEC>
__global__ void __launch_bounds__(kThreads, 2) sample_rows(const SampleArgs p) {
    const Stamp stamp_guard(p.stamp);
    extern __shared__ __align__(16) uint8_t smem_raw[];
    Smem& s = *reinterpret_cast<Smem*>(smem_raw);
    cg::cluster_group cluster = cg::this_cluster();
    int C = (int)cluster.num_blocks();  // (CTAs that take part: 1 once the first goes on alone)
    const int rank = (int)cluster.block_rank(), b = blockIdx.x / C, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    {
        uint4* h = reinterpret_cast<uint4*>(s.hist);
        for (int i = tid; i < (int)(sizeof s.hist / 16); i += kThreads) h[i] = make_uint4(0, 0, 0, 0);
    }
    const uint32_t bars = shared_addr(&s.bar[0]);
    if (tid == 0) {
        for (int q = 0; q < 2; ++q) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bars + 8 * q) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        s.late = 0;
    }
    cluster.barrier_arrive();  // (waited for before the first access to another CTA's shared memory)
    pdl_trigger();
    pdl_wait();
    Slice<HELD, VEC> el;
    const int chunk = ((p.V + C - 1) / C + 3) / 4 * 4;
    el.base = rank * chunk;
    el.n = max(0, min(chunk, p.V - el.base));
    el.row = p.logits + (int64_t)b * p.ld + el.base;
    el.held = s.row;
    const float T0 = p.temperature ? p.temperature[b] : 1.f, mp0 = p.min_p ? p.min_p[b] : 0.f;
    // (from 1e30 on a temperature makes all weights equal, as far as logits go)
    const bool flat = T0 >= 1e30f;
    const double T = fmax((double)T0, 1e-37), inv_T = flat ? 0.0 : 1.0 / T;

    bool solo = C == 1;
    uint32_t turn = 0;  // exchanges so far
    auto expect = [&](uint32_t bytes) {  // what the next exchange brings this CTA
        if (tid == 0) expect_bytes(bars + 8 * (turn & 1), bytes);
    };
    auto wait_for = [&](uint32_t n) {
        const uint32_t bar = bars + 8 * (n & 1), parity = n >> 1 & 1;
        for (uint32_t q = 0; q < kPolls; ++q)
            if (arrived(bar, parity)) return;
        s.late = 1;  // (cannot be; the row is given up at the end, with every CTA still there)
    };
    // the smallest of one 32-bit word per thread, over the cluster
    auto cluster_min = [&](uint32_t v) {
        v = __reduce_min_sync(0xffffffffu, v);
        uint32_t* const at = s.key[turn & 1];
        if (solo) {
            if (lane == 0) at[warp] = v;
            __syncthreads();
        } else {
            expect(C * kWarps * 4);
            if (lane < C) send(in_cta(shared_addr(at + rank * kWarps + warp), lane), in_cta(bars + 8 * (turn & 1), lane), v);
            wait_for(turn);
        }
        ++turn;
        v = 0xffffffffu;
        for (int i = lane; i < C * kWarps; i += 32) v = min(v, at[i]);
        return __reduce_min_sync(0xffffffffu, v);
    };

    // ---- maximum (fmaxf passes NaN over)
    float mx = -INFINITY;
    el.first([&](const float (&v)[kBlock]) {
#pragma unroll
        for (int e = 0; e < kBlock; ++e) mx = fmaxf(mx, v[e]);
    });
    cluster.barrier_wait();
    mx = value_of(cluster_min(key_of(mx)));
    if (rank == 0 && tid == 0 && p.pos) p.pos[b] += 1;
    if (mx == -INFINITY || !(T0 > 0.f) || mp0 > 1.f) {  // nothing to choose from, or greedy (no weight is above 1): the first of the largest
        int at = -1;
        if (mx > -INFINITY) {
            at = 0x7fffffff;
            __syncthreads();  // (the row's copy was written by other threads than those that read it now)
            el.each([&](float x, int i) { at = x == mx ? min(at, i) : at; });
            at = (int)cluster_min((uint32_t)at);
        }
        __syncthreads();
        if (s.late) cluster.sync();
        if (rank == 0 && tid == 0) p.tokens[b] = s.late ? -1 : at;
        return;  // (nothing is sent after an exchange that all have had)
    }
    // (infinities share all the weight and are the only candidates: all in the last bin, units() is 1 there)
    const bool infinite = mx == INFINITY;
    const double m = (double)mx;
    Row r;
    r.m = mx;
    r.inv_T2 = (float)(2.0 * inv_T);
    r.inv_Tl2 = (float)(1.4426950408889634 * inv_T);
    r.half_T = flat ? 0.f : (float)(0.5 * T);
    // Where T is less than 2^-16 of the maximum, sums of both lose T's own bits: there everything is measured from the maximum,
    // which x - m is exact for (16 T is 2^-12 of m at most; what is farther away has no weight).
    r.shift = !flat && !infinite && T < 0x1p-16 * fabs(m) ? mx : 0.f;
    r.top = flat ? mx : __double2float_ru(r.shift != 0.f ? 0.25 * T : m + 0.25 * T);
    if (tid < kBins) s.W[tid] = infinite ? kUnit : kUnit * exp((r.shift != 0.f ? (double)r.end_of((float)tid) : (double)r.end_of((float)tid) - m) * inv_T);
    if (tid == 32) {  // a weight is at least min_p when the logit is at most this far (negative) from the maximum
        const double thr = mp0 > 0.f && !flat ? T * log((double)mp0) : -INFINITY;
        s.thr = infinite ? mx : fmaxf(__double2float_ru(m + thr), -FLT_MAX);
    }
    __syncthreads();
    // the kept prefix: elements above lim_x, and those equal to it with an index up to lim_i
    constexpr int kAll = 0x7fffffff;
    float lim_x = s.thr;
    int lim_i = kAll;
    // Adds the lane-private histograms up over the cluster: the CTAs' totals of bin `lane` are in s.xch[(turn - 1) & 1][CTA][lane]
    // once have_totals() is through.
    auto totals = [&]() {
        __syncthreads();
        if (!solo) expect(C * kBins * 8);
#pragma unroll
        for (int q = 0; q < kBins / kWarps; ++q) {
            const int bin = warp * (kBins / kWarps) + q;
            uint32_t lo = 0, hi = 0;  // (a lane's sum has 32 bits)
#pragma unroll
            for (int w = 0; w < kSlices; ++w) {
                const uint32_t v = s.hist[w][bin][lane];
                s.hist[w][bin][lane] = 0;
                lo += v & 0xffffu;
                hi += v >> 16;
            }
            lo = __reduce_add_sync(0xffffffffu, lo);
            hi = __reduce_add_sync(0xffffffffu, hi);
            unsigned long long* const to = &s.xch[turn & 1][solo ? 0 : rank][bin];
            const unsigned long long sum = ((unsigned long long)hi << 16) + lo;
            if (!solo && lane < C) send(in_cta(shared_addr(to), lane), in_cta(bars + 8 * (turn & 1), lane), sum);
            if (solo && lane == 0) *to = sum;
        }
        if (solo) __syncthreads();
        ++turn;
    };
    auto have_totals = [&]() { if (!solo) wait_for(turn - 1); };
    auto total = [&](float& most) {  // (first warp) of bin `lane`: the total, and the largest CTA's share
        have_totals();
        unsigned long long v[kCluster], t = 0, m = 0;
#pragma unroll
        for (int c = 0; c < kCluster; ++c) v[c] = c < C ? s.xch[(turn - 1) & 1][c][lane] : 0;
#pragma unroll
        for (int c = 0; c < kCluster; ++c) {
            t += v[c];
            m = max(m, v[c]);
        }
        most = (float)m;
        return t;
    };
    const uint32_t my_hist = (uint32_t)__cvta_generic_to_shared(&s.hist[warp % kSlices][0][lane]);  // + bin * 128
    const uint32_t hist_a = my_hist - 0x4b000000u * 128u;                                           // + the bits of bin_number * 128

    Range have{1, 0, 0, -1};  // what loc holds (nothing)
    bool have_all = false;    // (all that can still be asked for)
    uint2* loc = s.loc;

    // The bins of the whole row up to the limit.  Elements beyond it add nothing: no branches.
    auto level0 = [&](bool mass) {
        if (have_all) {
            const uint32_t lk = key_of(lim_x);
            const uint32_t nloc = s.nloc;
#pragma unroll 4
            for (uint32_t e = tid; e < nloc; e += kThreads) {
                const uint2 v = loc[e];
                const float x = value_of(v.x);
                if (v.x < lk || (v.x == lk && (int)v.y <= lim_i)) red_add(my_hist + r.bin(x) * 128u, r.units(x, r.end_of((float)r.bin(x))));
            }
        } else if (!mass) {
            el.blocks([&](const float (&v)[kBlock], int) __attribute__((always_inline)) {  // (top-k comes first: no limit by index yet)
#pragma unroll
                for (int e = 0; e < kBlock; ++e) red_add(hist_a + __float_as_uint(r.bin_number(v[e])) * 128u, v[e] >= lim_x ? 1u : 0u);
            });
        } else {
            el.blocks([&](const float (&v)[kBlock], int) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < kBlock; ++e) {
                    const float n = r.bin_number(v[e]);
                    const uint32_t u = r.units(v[e], r.end_of(n - 8388608.f));
                    red_add(hist_a + __float_as_uint(n) * 128u, v[e] >= lim_x ? u : 0u);
                }
            });
            if (lim_i != kAll) {  // equal to the limit, but behind it: their weight is taken back where it was put
                const uint32_t at_lim = my_hist + r.bin(lim_x) * 128u, back = 0u - r.units(lim_x, r.end_of((float)r.bin(lim_x)));
                el.blocks([&](const float (&v)[kBlock], int at) {
                    for (int e = 0; e < kBlock; ++e)
                        if (v[e] == lim_x && at + el.place(e) > lim_i) red_add(at_lim, back);
                });
            }
        }
        totals();
    };

    // The smallest key whose bin is at least j.  It lies next to that of the bin's upper end: 32 probes around it nearly
    // always hold it; if not (values near zero have finer keys), the whole range is searched, 32 probes a round.
    const uint32_t k0 = key_of(r.m), k1 = key_of(-FLT_MAX) + 1;  // the answer is in k0..k1
    auto probe = [&](int j, uint32_t& a) {
        const uint32_t mid = key_of(fmaxf(r.end_of((float)j) + r.shift, -FLT_MAX));
        a = mid > k0 + 16 ? mid - 16 : k0;
        const uint32_t at = a + lane;
        return __ballot_sync(0xffffffffu, at >= k1 || r.bin(value_of(at)) >= j);
    };
    auto first_key = [&](int j, unsigned near, uint32_t a) -> uint32_t {  // (near, a: the probes)
        if (j <= 0) return k0;
        if (j >= kBins) return k1;
        if (near && (!(near & 1u) || a == k0)) return a + __ffs(near) - 1;
        uint32_t e = k1;
        a = k0;
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
        if (infinite) return Range{key_of(mx), key_of(mx), 0, kAll};
        uint32_t pa, pe;
        const unsigned near_a = probe(j, pa), near_e = probe(j + 1, pe);
        const uint32_t a = first_key(j, near_a, pa), e = first_key(j + 1, near_e, pe);
        return Range{a, max(a, min(e - 1, key_of(lim_x))), 0, kAll};
    };

    // Copies this CTA's elements of a range to s.loc (the caller knows that they fit).
    auto compact = [&](const Range& g) {
        const float xa = value_of(g.ka), xb = value_of(g.kb);
        if (tid == 0) s.nloc = 0;
        __syncthreads();
        auto inside = [&](float x, int i) { return (x != lim_x || i <= lim_i) && i >= g.ia && i <= g.ib; };
        const bool by_index = lim_i != kAll || g.ia > 0 || g.ib != kAll;
        el.blocks([&](const float (&v)[kBlock], int first) __attribute__((always_inline)) {
            uint32_t mask = 0;
#pragma unroll
            for (int e = 0; e < kBlock; ++e) mask |= (v[e] <= xa && v[e] >= xb) ? 1u << e : 0u;
            if (by_index) {
#pragma unroll
                for (int e = 0; e < kBlock; ++e)
                    if (!inside(v[e], first + el.place(e))) mask &= ~(1u << e);
            }
            if (!__any_sync(0xffffffffu, mask != 0)) return;
            const uint32_t cnt = __popc(mask), upto = warp_scan(cnt, lane);
            uint32_t at = 0;
            if (lane == 31) at = atomicAdd(&s.nloc, upto);
            at = __shfl_sync(0xffffffffu, at, 31) + upto - cnt;
            for (; mask; mask &= mask - 1, ++at) {  // (few: read them once more instead of asking for each of the block)
                const int i = first + el.place(__ffs(mask) - 1);
                if (at < kLocal) s.loc[at] = make_uint2(key_of(HELD ? el.held[i - el.base] : el.row[i - el.base]), (uint32_t)i);
            }
        });
        __syncthreads();
        if (tid == 0) s.nloc = min(s.nloc, (uint32_t)kLocal);
        __syncthreads();
        have = g;
    };
    // f(key, index) of this CTA's elements of a range, from loc or from the row.  (loc may have been filled before a top-k cut
    // among equal logits: those behind the cut are passed over.)
    auto visit = [&](const Range& g, bool local, auto f) {
        if (local) {
            const uint32_t nloc = s.nloc, lk = key_of(lim_x);
#pragma unroll 4
            for (uint32_t e = tid; e < nloc; e += kThreads) {
                const uint2 v = loc[e];
                if (v.x >= g.ka && v.x <= g.kb && (int)v.y >= g.ia && (int)v.y <= g.ib && (v.x != lk || (int)v.y <= lim_i)) f(v.x, (int)v.y);
            }
        } else {
            el.each([&](float x, int i) {
                const uint32_t k = key_of(x);
                if (x == x && k >= g.ka && k <= g.kb && (x != lim_x || i <= lim_i) && i >= g.ia && i <= g.ib) f(k, i);
            });
        }
    };
    // Brings the local elements of a range together in every CTA: CTA c's go to slots c * kList / C .. (the caller knows
    // that no CTA has more).
    int slot_bits = __ffs(kList / C) - 1, slot = 1 << slot_bits;
    auto gather = [&](const Range& g) {
        if (tid == 0) s.lcnt = 0;
        __syncthreads();
        const uint32_t nloc = s.nloc, lk = key_of(lim_x);
        for (uint32_t e0 = 0; e0 < nloc; e0 += 4 * kThreads) {
            uint2 v[4];
            unsigned who[4], any = 0, cnt = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = loc[min(e0 + q * kThreads + tid, nloc - 1)];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const bool in = e0 + q * kThreads + tid < nloc && v[q].x >= g.ka && v[q].x <= g.kb && (int)v[q].y >= g.ia && (int)v[q].y <= g.ib &&
                                (v[q].x != lk || (int)v[q].y <= lim_i);
                who[q] = __ballot_sync(0xffffffffu, in);
                any |= who[q];
                cnt += __popc(who[q]);
            }
            if (!any) continue;
            uint32_t at = 0;
            if (lane == 0) at = atomicAdd(&s.lcnt, cnt);
            at = __shfl_sync(0xffffffffu, at, 0);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t to = at + __popc(who[q] & ((1u << lane) - 1u));
                if ((who[q] >> lane & 1u) && to < slot) s.tmp[to] = ((unsigned long long)v[q].x << 32) | v[q].y;
                at += __popc(who[q]);
            }
        }
        __syncthreads();
        if (tid < kList) {
            const uint32_t n = min(s.lcnt, (uint32_t)slot), c = tid >> slot_bits, e = tid & (slot - 1);
            unsigned long long* const to = &s.list[turn & 1][solo ? e : rank * slot + e];
            uint32_t* const to_n = &s.cnt[turn & 1][solo ? 0 : rank];
            if (!solo) {  // (all slots: the other side counts bytes)
                const uint32_t bar = in_cta(bars + 8 * (turn & 1), c);
                send(in_cta(shared_addr(to), c), bar, e < n ? s.tmp[e] : ~0ull);
                if (e == 0) send(in_cta(shared_addr(to_n), c), bar, n);
            } else {
                if (e < n) *to = s.tmp[e];
                if (e == 0) *to_n = n;
            }
        }
        if (!solo) expect(kList * 8 + C * 4);
        __syncthreads();  // (tmp is written again once the lists are there: by then every warp has sent its part of it)
        if (!solo) wait_for(turn);
        ++turn;
        int all = 0;
        for (int q = 0; q < C; ++q) all += (int)s.cnt[(turn - 1) & 1][q];
        return min(all, kList);
    };
    // The collected elements in order, element e in thread e: each counts those before it.
    auto sorted = [&](int n) {
        unsigned long long* const list = s.list[(turn - 1) & 1];
        const int n8 = (n + 7) / 8 * 8;
        if (tid < kList) {  // side by side, and full to a multiple of 8
            const int c0 = tid >> slot_bits, e0 = tid & (slot - 1);
            if ((uint32_t)e0 < s.cnt[(turn - 1) & 1][c0]) {
                int to = e0;
                for (int c = 0; c < c0; ++c) to += (int)s.cnt[(turn - 1) & 1][c];
                if (to < kList) s.tmp[to] = list[tid];
            }
            if (tid >= n && tid < n8) s.tmp[tid] = ~0ull;
        }
        __syncthreads();
        // the comparisons of an element are shared by as many neighbouring threads as there are to spare
        const int p_bits = min(5, max(0, __clz(n - 1 | 1) - __clz(kThreads / 2))), P = 1 << p_bits;  // P n <= kThreads
        if (warp * 32 < P * n) {
            const int e = tid >> p_bits;
            const unsigned long long k = e < n ? s.tmp[e] : ~0ull;
            int before = 0;
            for (int q = 8 * (tid & (P - 1)); q < n8; q += 8 * P) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const ulonglong2 v = reinterpret_cast<const ulonglong2*>(s.tmp + q)[i];
                    before += (v.x < k) + (v.y < k);
                }
            }
            for (int o = 1; o < P; o <<= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
            if (e < n && (tid & (P - 1)) == 0) list[before] = k;
        }
        __syncthreads();
        return tid < n ? list[tid] : ~0ull;
    };
    // Running sum of the elements' weights, on top of `before`.
    auto summed = [&](int n, unsigned long long k, double before) {
        double run = 0.0;
        if (warp * 32 < n) {
            if (tid < n) {
                const float x = value_of((uint32_t)(k >> 32));
                const int bin = r.bin(x);
                run = s.W[bin] * (double)r.units(x, r.end_of((float)bin));
            }
            run = warp_scan(run, lane);
            if (lane == 31) s.scan[warp] = run;
        }
        __syncthreads();
        if (warp * 32 < n)
            for (int v = 0; v < warp; ++v) before += s.scan[v];
        return before + run;
    };
    // The first of the elements 0..n-1 whose running sum is above (strict) or at least t; the last one if none is.
    auto first_at = [&](int n, unsigned long long k, double run, double t, bool strict) {
        if (tid == 0) s.hit = max(n - 1, 0);
        __syncthreads();
        const unsigned ok = warp * 32 < n ? __ballot_sync(0xffffffffu, tid < n && (strict ? run > t : run >= t)) : 0u;
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
    const int k = p.top_k ? p.top_k[b] : 0;

    // Three searches at most: the k-th candidate, the border of the nucleus, the drawn token.  The first warp of every CTA
    // takes the decisions, from the same numbers.
    unsigned long long t = 0;            // (first warp) weight, or candidates, of bin `lane`
    double w0 = 0.0, run0 = 0.0;         // of the same bin, and of all up to it
    float most = 0.f, most_upto = 0.f;   // of the same two, the largest CTA's share (in units, at most)
    float t_upto = 0.f;                  // t of the bin and all before it
    double Z = 0.0;                      // weight of what is kept (once weighed)
    bool weighed = false;
    for (int stage = k > 0 && k < p.V ? 0 : 1; stage < 3; ++stage) {
        if (stage == 1 && !nucleus) continue;
        const bool by_rank = stage == 0, strict = stage == 2;
        const float per = by_rank ? 1.f : kPerUnit;
        const bool fresh = !weighed;
        if (fresh) {
            level0(!by_rank);
            weighed = !by_rank;
        }
        if (warp == 0) {
            if (fresh) {
                t = total(most);
                w0 = by_rank ? (double)t : s.W[lane] * (double)t;
                run0 = w0;
                most_upto = most;
                t_upto = (float)t;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {  // (three scans side by side: one alone waits for its own steps)
                    const double a = __shfl_up_sync(0xffffffffu, run0, o);
                    const float c = __shfl_up_sync(0xffffffffu, most_upto, o), e = __shfl_up_sync(0xffffffffu, t_upto, o);
                    if (lane >= o) {
                        run0 += a;
                        most_upto += c;
                        t_upto += e;
                    }
                }
                Z = __shfl_sync(0xffffffffu, run0, 31);
            }
            Search f;
            f.target = by_rank ? (double)k : (stage == 1 ? tp : u) * Z;
            // the bin that holds the target
            const unsigned ok = __ballot_sync(0xffffffffu, t > 0 && (strict ? run0 > f.target : run0 >= f.target));
            const unsigned any = __ballot_sync(0xffffffffu, t > 0);
            f.j = ok ? __ffs(ok) - 1 : 31 - __clz(any | 1u);
            f.before = __shfl_sync(0xffffffffu, run0 - w0, f.j);
            f.tot = per * __shfl_sync(0xffffffffu, (float)t, f.j);
            f.part = per * __shfl_sync(0xffffffffu, most, f.j);
            f.upto = per * __shfl_sync(0xffffffffu, most_upto, f.j);
            f.all = per * __shfl_sync(0xffffffffu, t_upto, f.j);
            f.g = range_of_bin(f.j);
            if (by_rank && Z <= (double)k) f.j = -1;  // no more candidates than that
            if (lane == 0) s.at = f;
        }
        __syncthreads();
        const int j = s.at.j;
        const double target = s.at.target;
        Range g = s.at.g;
        float tot = s.at.tot, part = solo ? tot : s.at.part;
        if (j < 0) {
            __syncthreads();
            continue;
        }
        const bool open = !by_rank && j == kBins - 1;  // (weights in the last bin may be anything down to 0: they count nothing)
        bool local = g.ka >= have.ka && g.kb <= have.kb && have.ia == 0 && have.ib == kAll;
        // Narrow the range around the target until its elements can be collected.
        int n = 0;
        bool rest = false;  // few enough from the top down: all that is left to do happens in the list
        for (int level = 0; level < 16; ++level) {
            if (open) {
                uint32_t c = 0;
                visit(g, local, [&](uint32_t, int) { ++c; });
                red_add(my_hist, c);
                totals();
                have_totals();
                __syncthreads();  // (the histograms are counted into again: every warp has cleared its bins)
                tot = part = 0.f;
                for (int q = 0; q < C; ++q) {
                    const float v = (float)s.xch[(turn - 1) & 1][q][0];
                    tot += v;
                    part = fmaxf(part, v);
                }
            }
            if (!local && part <= kLocal) {
                // everything from the top down if it fits: then the other searches find their elements there too
                const bool top = level == 0 && !open && s.at.upto <= kLocal;
                compact(top ? Range{key_of(r.m), g.kb, 0, kAll} : g);
                local = true;
                if (top && !solo && C > 1 && s.at.all <= (float)p.move_max) {
                    // few enough for one CTA: they go to the place of its row, and the others are done
                    const uint32_t n = s.nloc;
                    expect(C * 4);
                    if (tid < C) send(in_cta(shared_addr(&s.moved[rank]), tid), in_cta(bars + 8 * (turn & 1), tid), n);
                    wait_for(turn);  // (and all have done with their rows)
                    ++turn;
                    uint32_t at = 0, all_n = 0;
                    for (int c = 0; c < C; ++c) {
                        at += c < rank ? s.moved[c] : 0;
                        all_n += s.moved[c];
                    }
                    all_n = min(all_n, (uint32_t)kMoved);
                    if (rank) {
                        const uint32_t to = in_cta(shared_addr(&s.row[0]), 0), bar = in_cta(bars + 8 * (turn & 1), 0);
                        for (uint32_t e = tid; e < n && at + e < kMoved; e += kThreads)
                            send(to + 8 * (at + e), bar, *reinterpret_cast<const unsigned long long*>(&s.loc[e]));
                        __syncthreads();
                        if (s.late) cluster.sync();
                        return;
                    }
                    for (uint32_t e = tid; e < n; e += kThreads) reinterpret_cast<uint2*>(&s.row[0])[e] = s.loc[e];
                    expect((all_n - n) * 8);
                    wait_for(turn);
                    ++turn;
                    __syncthreads();  // (every warp has read its CTA's own count: the waits above are for other CTAs only)
                    if (tid == 0) s.nloc = all_n;
                    __syncthreads();
                    loc = reinterpret_cast<uint2*>(&s.row[0]);
                    solo = true;
                    C = 1;
                    slot_bits = __ffs(kList) - 1;
                    slot = kList;
                    part = tot;
                }
                if (top && by_rank) {
                    have_all = true;
                    rest = s.at.all <= kSorted && (solo ? s.at.all : s.at.upto) <= slot;
                    if (rest) g = have;
                }
            }
            if (local && (rest || (part <= slot && tot <= kSorted))) {
                n = gather(g);
                break;
            }
            // 32 parts of its values, or of its indices where there is only one value
            const bool by_value = g.ka != g.kb;
            if (!by_value && g.ib == kAll) g.ib = p.V - 1;
            const uint32_t lo = by_value ? g.ka : (uint32_t)g.ia, span = by_value ? g.kb - g.ka : (uint32_t)(g.ib - g.ia);
            const int sh = max(0, 32 - __clz(span) - 5);
            const float X = r.end_of((float)j);
            visit(g, local, [&](uint32_t key, int i) {
                red_add(my_hist + (((by_value ? key : (uint32_t)i) - lo) >> sh) * 128u, by_rank ? 1u : r.units(value_of(key), X));
            });
            totals();
            if (warp == 0) {
                float share;
                const unsigned long long tt = total(share);
                const double before = s.at.before, w = by_rank ? (double)tt : s.W[j] * (double)tt, run = warp_scan(w, lane);
                const unsigned yes = __ballot_sync(0xffffffffu, tt > 0 && (strict ? before + run > target : before + run >= target));
                const unsigned some = __ballot_sync(0xffffffffu, tt > 0);
                const int cut = yes ? __ffs(yes) - 1 : 31 - __clz(some | 1u);
                const double step = __shfl_sync(0xffffffffu, run - w, cut);
                const uint32_t a = lo + ((uint32_t)cut << sh), last = (uint32_t)min((unsigned long long)a + (1u << sh) - 1, (unsigned long long)lo + span);
                if (by_value) { g.ka = a; g.kb = last; }
                else { g.ia = (int)a; g.ib = (int)last; }
                const float total_of = __shfl_sync(0xffffffffu, (float)tt, cut), share_of = __shfl_sync(0xffffffffu, share, cut);
                if (lane == 0) {
                    s.at.before = before + step;
                    s.at.tot = per * total_of;
                    s.at.part = per * share_of;
                    s.at.g = g;
                }
            }
            __syncthreads();
            g = s.at.g;
            tot = s.at.tot;
            part = s.at.part;
        }
        const unsigned long long e = sorted(n);
        if (by_rank && !rest) {
            if (tid == max(0, min(n, k - (int)s.at.before) - 1)) s.res = Result{value_of((uint32_t)(e >> 32)), (int)(uint32_t)e, 0.0};
            __syncthreads();
        } else {
            const double cum = summed(n, e, rest ? 0.0 : s.at.before);
            int kept = n;
            double at = target;
            bool over = strict;
            if (rest) {
                kept = min(k, n);
                if (tid == kept - 1) s.res.mass = cum;
                __syncthreads();
                double z = s.res.mass;
                if (nucleus) {
                    kept = 1 + first_at(kept, e, cum, tp * z, false);
                    z = s.res.mass;
                }
                at = u * z;
                over = true;
            }
            first_at(kept, e, cum, at, over);
            if (rest) break;
        }
        lim_x = s.res.x;
        lim_i = s.res.i;
        if (stage == 1) Z = s.res.mass;
    }
    __syncthreads();
    if (s.late) cluster.sync();
    if (rank == 0 && tid == 0) p.tokens[b] = s.late ? -1 : s.res.i;
}

}  // namespace

cudaError_t sample_launch(const SampleArgs& a, cudaStream_t st, bool pdl) {
    // as many CTAs per row as hold it in shared memory (a power of two, eight at most: 131072 elements)
    int C = 1;
    while (C < kCluster && (int64_t)C * kHeld < a.V) C *= 2;
    const bool held = (int64_t)C * kHeld >= a.V;
    const int chunk = ((a.V + C - 1) / C + 3) / 4 * 4, block = kBlock * kThreads;
    SampleArgs p = a;
    // One CTA is slower with a long list than eight, but leaves seven places to other rows: where the grid is several
    // times what the GPU holds, it is given more (256 rows: 4 % less time; 128 rows: 89 against 85; 32 rows: 34 against 31).
    p.move_max = a.B * C > 4 * kResident ? kMoved : kMoved / 2;
    const size_t smem = sizeof(Smem) + (C == 1 ? (size_t)(chunk + block - 1) / block * block * 4 : (size_t)kHeld * 4);
    const bool vec = reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 && (a.B == 1 || a.ld % 4 == 0);
    auto kern = held ? (vec ? sample_rows<true, true> : sample_rows<true, false>) : (vec ? sample_rows<false, true> : sample_rows<false, false>);
    // (always the same value: calls of other threads rely on it)
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(sizeof(Smem) + kHeld * 4));
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(a.B * C);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
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
    return cudaLaunchKernelEx(&cfg, kern, p);
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
