// Verification of drafted tokens against the target's probabilities, from given random numbers.
#include <cfloat>

#include <cooperative_groups.h>

#include "common.cuh"
#include "first.h"
#include "ops.h"

using namespace first;
namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;  // that count; one more warp copies
constexpr int kMaxCluster = 16, kMaxRound = 8, kSums = 5;

struct VerifyArgs {
    const float *target, *draft;  // draft NULL: each drafted token had probability 1
    int64_t t_seq, t_row, d_seq, d_row;
    const int32_t* drafted;
    const float *u, *draws, *temperature;
    int32_t *tokens, *accepted;
    int B, K, V;
    bool probs;
    int C, R;  // CTAs of a cluster, positions a round
};

// One row's sum over some of its tokens, relative to their largest logit; greedy rows: value and lowest index of the largest.
struct Part {
    float top, sum;
    int32_t at;
};

// Logits as they count: NaN as -inf, +inf as the largest float32.
__device__ __forceinline__ float logit(float x) { return x > FLT_MAX ? FLT_MAX : (x == x ? x : -INFINITY); }
// Uniform draws as they count.
__device__ __forceinline__ double draw(float u) { return u < 1.f ? (double)fmaxf(u, 0.f) : (double)0x1.fffffep-1f; }

struct Scale {
    float hi, lo, floor;  // log2(e) / T in two parts; differences below `floor` weigh nothing
    double steps;         // 32 log2(e) / T
};

// exp((x - top) / T) in float32, of logits that count.
__device__ __forceinline__ float weight32(float x, float top, const Scale& sc) {
    const float t = fmaxf(x - top, sc.floor);
    float w;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(fmaf(t, sc.hi, t * sc.lo)));
    return w;
}
// The same in 64 bits, to 2^-39: which token a draw falls on hangs on the sums of these.  2^(k / 32) from a table for the nearest k, the
// rest by its Taylor series: |g| <= ln 2 / 64, g^5 / 120 < 2^-39.
template <typename Table>
__device__ __forceinline__ double weight64(float x, float top, const Scale& sc, Table&& pow32) {
    x = logit(x);
    const double a = ((double)x - (double)top) * sc.steps;
    constexpr double kMagic = 6755399441055744.0;  // 1.5 2^52: adding it leaves the nearest whole number in the low bits
    const double m = a + kMagic, g = (a - (m - kMagic)) * (0.69314718055994530942 / 32);
    const int k = __double2loint(m);
    const double s = fma(fma(fma(fma(g, 1.0 / 24, 1.0 / 6), g, 0.5), g, 1.0), g, 1.0) * pow32(k & 31);
    return a > -32000.0 ? __hiloint2double(__double2hiint(s) + (k >> 5) * (1 << 20), __double2loint(s)) : 0.0;
}

__device__ __forceinline__ double warp_sum64(double x) {
#pragma unroll 1
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
__device__ __forceinline__ double warp_scan64(double x) {
#pragma unroll 1
    for (int o = 1; o < 32; o *= 2) {
        const double v = __shfl_up_sync(0xffffffffu, x, o);
        if ((int)(threadIdx.x & 31) >= o) x += v;
    }
    return x;
}
__device__ __forceinline__ Part warp_join(Part p, const Scale& sc, bool greedy) {
    const float top = warp_max(p.top);
    if (greedy) p.at = __reduce_min_sync(0xffffffffu, p.top == top ? p.at : 0x7fffffff);
    else p.sum = top > -INFINITY ? warp_sum(p.sum * weight32(p.top, top, sc)) : 0.f;
    p.top = top;
    return p;
}

// A row's part [lo, hi) comes in pieces of kPiece tokens through a ring in shared memory, by copies of its whole 16 bytes of memory; the up to three
// tokens at either end that share theirs with others are fetched one by one (nothing outside the row is read).
constexpr int kPiece = 8192, kRing = 3, kEach = kPiece / (4 * kThreads);
struct Span {
    const float* from;  // 16-byte aligned
    int off, n, pieces; // tokens of it before the part, of the part, pieces
};
__device__ __forceinline__ Span span_of(const float* row, int lo, int hi) {
    Span s;
    s.off = (int)(reinterpret_cast<uintptr_t>(row + lo) >> 2 & 3);
    s.from = row + lo - s.off;
    s.n = hi - lo;
    s.pieces = s.n > 0 ? (s.off + s.n + kPiece - 1) / kPiece : 1;
    return s;
}
constexpr uint32_t kPolls = 1u << 22;
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {  // bounded: false after kPolls tries
    for (uint32_t i = 0; i < kPolls; ++i) {
        uint32_t ok;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
    }
    return false;
}
// The tokens of piece q that are not copied, one by one (out of line: few rows have any).
__device__ __noinline__ void edges(uint32_t dst, const float* from, int off, int all, int q) {
    const int head = q == 0 && off ? min(4, all) : off, tail = max(all & ~3, head);  // [off, head) and [tail, all) of the span
#pragma unroll 1
    for (int i = off; i < head; ++i) asm volatile("st.shared.f32 [%0], %1;" ::"r"(dst + 4 * i), "f"(__ldg(from + i)) : "memory");
#pragma unroll 1
    for (int i = tail; i < all && tail / kPiece == q; ++i) asm volatile("st.shared.f32 [%0], %1;" ::"r"(dst + 4 * (i % kPiece)), "f"(__ldg(from + i)) : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // (the place is copied into again later)
}
// (One thread's.)  What it stores itself is there when the barrier completes, like what is copied.
__device__ __forceinline__ void copy_piece(uint32_t dst, uint32_t bar, const Span& s, int q) {
    if ((s.off && q == 0) || ((s.off + s.n) & 3)) edges(dst, s.from, s.off, s.off + s.n, q);
    const int first = q * (kPiece / 4), b0 = max(first, s.off ? 1 : 0), b1 = min(first + kPiece / 4, (s.off + s.n) / 4);  // whole 16 bytes
    const uint32_t bytes = 16 * max(b1 - b0, 0);
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
    if (bytes)
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                     ::"r"(dst + 16 * (b0 - first)), "l"(s.from + 4 * (int64_t)b0), "r"(bytes), "r"(bar) : "memory");
}
template <bool GREEDY>
__device__ __forceinline__ void add(Part& p, const float4* piece, const Span& s, int q, int lo, const Scale& sc) {
    float f[4 * kEach];
    const int first = q * kPiece - s.off + 4 * (int)threadIdx.x;  // of the part
    const bool whole = q * kPiece >= s.off && (q + 1) * kPiece <= s.off + s.n;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const float4 v = piece[j * kThreads + threadIdx.x];
        f[4 * j] = v.x; f[4 * j + 1] = v.y; f[4 * j + 2] = v.z; f[4 * j + 3] = v.w;
    }
    if (!whole)
#pragma unroll
        for (int i = 0; i < 4 * kEach; ++i)
            if ((unsigned)(first + i / 4 * 4 * kThreads + i % 4) >= (unsigned)s.n) f[i] = -INFINITY;
    float big = -INFINITY;  // (a maximum passes over NaN, and so does weight32)
#pragma unroll
    for (int i = 0; i < 4 * kEach; ++i) big = fmaxf(big, f[i]);
    if (big > FLT_MAX) {
        big = FLT_MAX;
#pragma unroll
        for (int i = 0; i < 4 * kEach; ++i) f[i] = logit(f[i]);
    }
    if (GREEDY) {
        if (big < p.top || big == -INFINITY) return;
        int at = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < 4 * kEach; ++i)
            if (f[i] == big) at = min(at, lo + first + i / 4 * 4 * kThreads + i % 4);
        p.at = big > p.top ? at : min(at, p.at);
        p.top = big;
        return;
    }
    if (big == -INFINITY) return;
    if (big > p.top) {
        p.sum *= weight32(p.top, big, sc);
        p.top = big;
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4 * kEach; ++i) sum += weight32(f[i], p.top, sc);
    p.sum += sum;
}

// One cluster a sequence.  Rounds of R positions, then 2 R and so on: every row's sum and largest logit, then the decisions (taken by every
// CTA alike), until one is refused or all are accepted; the rows of later positions are not read.  Then the new token's
// distribution, in 64 bits, over the one row (or two) that it comes from: those rows are in L2 by now.
// 64 sequences x 7 drafts of 128256 tokens, a draft model's logits too: 136 us; the rows up to the refusals (225 MB of 493) would take 34 at
// the copy's rate, the rest, and the 29-31 us of small batches, is latency: a round's copies, the cluster's joins, the decision, and the 64-bit pass.
__global__ void __launch_bounds__(kThreads + 32, 2) verify_rows(const VerifyArgs p) {
    __shared__ Part s_warp[2 * kMaxRound][kWarps], s_part[2][2 * kMaxRound];
    __shared__ double s_sum[kSums][kWarps], s_all[kSums][kMaxCluster * kWarps], s_run[kWarps], s_pow[32], s_seg;
    __shared__ int s_ok[kMaxRound], s_hit, s_found, s_at;
    __shared__ float s_tops[kMaxRound][2], s_top[2];
    extern __shared__ __align__(128) float4 s_ring[];  // [kRing][kPiece] tokens
    __shared__ uint64_t s_bar[2 * kRing];  // pieces that are there, pieces that have been read
    __shared__ int s_gave;
    cg::cluster_group cluster = cg::this_cluster();
    const int C = p.C, b = blockIdx.x / C, rank = blockIdx.x % C, tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);  // (so that the compiler knows it as the warp's)
    const float temp = p.temperature ? p.temperature[b] : 1.f;
    const bool greedy = !p.probs && !(temp > 0.f);
    // (at most 32 drafts: a lane each; the first that is no token ends them)
    const int32_t* drafted = p.drafted + (int64_t)b * p.K;
    const int mine = lane < p.K ? drafted[lane] : -1;
    const double my_u = lane < p.K ? draw(p.u[(int64_t)b * p.K + lane]) : 0.0;
    const uint32_t closed = ~__ballot_sync(0xffffffffu, mine >= 0 && mine < p.V);
    const int valid = closed ? __ffs(closed) - 1 : 32;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s_ring), bars = (uint32_t)__cvta_generic_to_shared(s_bar);
    const double my_pow = exp2((double)lane / 32);
    if (tid < 32) s_pow[tid] = my_pow;
    // 2^(k/32): from shared memory, or, where the whole warp asks, from its lanes (random places of a small table meet in its banks)
    auto from_table = [&](int k) { return s_pow[k]; };
    auto from_lanes = [&](int k) { return __shfl_sync(0xffffffffu, my_pow, k); };
    if (tid == 32) {
        s_gave = 0;
        for (int i = 0; i < 2 * kRing; ++i)
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bars + 8 * i), "r"(i < kRing ? 1 : kWarps) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    int slot = 0;  // of the ring, next
    uint32_t phase = 0;
    Scale sc;
    const double t64 = (double)fminf(fmaxf(temp, 1e-37f), 1e30f);
    sc.hi = (float)(1.4426950408889634 / t64);
    sc.lo = (float)(1.4426950408889634 / t64 - (double)sc.hi);
    sc.floor = (float)(-200.0 * t64);
    sc.steps = 32 * 1.4426950408889634 / t64;
    const int per = ((p.V + C - 1) / C + 3) & ~3, lo = min(rank * per, p.V), hi = min(lo + per, p.V);
    auto t_of = [&](int i) { return p.target + b * p.t_seq + i * p.t_row; };
    auto d_of = [&](int i) { return p.draft + b * p.d_seq + i * p.d_row; };
    int j = 0;  // the position whose token is new
    if (p.probs) {
        bool ok = false;
        if (lane < valid) {
            const double pd = fmax((double)t_of(lane)[mine], 0.0), qd = p.draft ? fmax((double)d_of(lane)[mine], 0.0) : 1.0;
            ok = my_u * qd < pd;
        }
        const uint32_t refused = ~__ballot_sync(0xffffffffu, ok);
        j = refused ? __ffs(refused) - 1 : 32;
        __syncthreads();
    } else {
        const int sides = p.draft && !greedy ? 2 : 1;
        bool open = true;
        for (int i0 = 0, round = 0, n = 0; open; i0 += n, ++round) {
            n = min(min(p.R << round, kMaxRound), valid + 1 - i0);  // (what survives a round is likely to survive the next)
            // the drafted tokens' own logits and draws, for the decisions below
            const int my_i = i0 + min(warp, n - 1), my_d = __shfl_sync(0xffffffffu, mine, my_i & 31);
            const double u_i = __shfl_sync(0xffffffffu, my_u, my_i & 31);
            float own[2] = {0.f, 0.f};
            if (warp < n && my_i < valid && !greedy) {
                own[0] = __ldg(t_of(my_i) + my_d);
                if (p.draft) own[1] = __ldg(d_of(my_i) + my_d);
            }
            // the round's rows (target and draft in turns), piece after piece; the last warp copies them
            const int rows = n * sides - (sides == 2 && i0 + n - 1 == valid ? 1 : 0);
            for (int r = 0; r < rows; ++r) {
                const Span sp = span_of(sides == 2 ? (r & 1 ? d_of(i0 + r / 2) : t_of(i0 + r / 2)) : t_of(i0 + r), lo, hi);
                Part part{-INFINITY, 0.f, 0x7fffffff};
                for (int q = 0; q < sp.pieces; ++q) {
                    const uint32_t bar = bars + 8 * slot;
                    if (warp < kWarps) {
                        if (!bar_wait(bar, phase)) s_gave = 1;  // (the sequence's result is void)
                        const float4* piece = s_ring + slot * (kPiece / 4);
                        if (greedy) add<true>(part, piece, sp, q, lo, sc);
                        else add<false>(part, piece, sp, q, lo, sc);
                        __syncwarp();
                        if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar + 8 * kRing) : "memory");
                    } else if (lane == 0) {
                        if (!bar_wait(bar + 8 * kRing, phase ^ 1)) s_gave = 1;
                        copy_piece(ring + slot * (kPiece * 4), bar, sp, q);
                    }
                    if (++slot == kRing) { slot = 0; phase ^= 1; }
                }
                if (warp < kWarps) {
                    part = warp_join(part, sc, greedy);
                    if (lane == 0) s_warp[r][warp] = part;
                }
            }
            __syncwarp();
            __syncthreads();
            for (int r = warp; r < rows; r += kWarps) {
                const Part q = warp_join(lane < kWarps ? s_warp[r][lane] : Part{-INFINITY, 0.f, 0x7fffffff}, sc, greedy);
                if (lane == 0) s_part[round & 1][r] = q;
            }
            cluster.sync();
            if (warp < n) {  // one warp a position, half of it a side
                const bool drafts = my_i < valid;
                const int side = lane >> 4, k = lane & 15;
                Part q{-INFINITY, 0.f, 0x7fffffff};
                if (k < C && (side == 0 || (sides == 2 && drafts))) q = *cluster.map_shared_rank(&s_part[round & 1][warp * sides + side], k);
                float top = q.top;
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                float sum = greedy || !(top > -INFINITY) ? 0.f : q.sum * weight32(q.top, top, sc);
                int at = q.top == top ? q.at : 0x7fffffff;
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) {
                    sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    at = min(at, __shfl_xor_sync(0xffffffffu, at, o));
                }
                // u q < p with both sums multiplied out
                const double w = sum > 0.f && drafts ? weight64(own[side], top, sc, from_table) : 0.0;
                const float other = __shfl_down_sync(0xffffffffu, sum, 16);
                const double w_q = __shfl_down_sync(0xffffffffu, w, 16);
                const float top_q = __shfl_down_sync(0xffffffffu, top, 16);
                if (lane == 0) {
                    if (!drafts) s_ok[warp] = 0;
                    else if (greedy) s_ok[warp] = my_d == at && top > -INFINITY;
                    else if (!p.draft) s_ok[warp] = u_i * sum < w;
                    else s_ok[warp] = other > 0.f ? u_i * w_q * sum < w * other : w > 0.0;
                    s_tops[warp][0] = top;
                    s_tops[warp][1] = sides == 2 ? top_q : -INFINITY;
                    s_warp[0][warp] = Part{top, sum, at};
                    s_warp[1][warp] = Part{top_q, sides == 2 ? other : 0.f, 0};
                }
            }
            __syncthreads();
            int i = 0;
            while (i < n && s_ok[i]) ++i;
            if (i < n) {
                j = i0 + i;
                if (tid == 0) { s_top[0] = s_tops[i][0]; s_top[1] = s_tops[i][1]; s_at = s_warp[0][i].at; s_run[0] = s_warp[0][i].sum; s_run[1] = s_warp[1][i].sum; }
                open = false;
            }
            __syncthreads();
        }
    }
    // ---- the new token
    int token = -1;
    if (greedy) {
        if (s_top[0] > -INFINITY) token = s_at;
    } else {
        const float* t = t_of(j);
        const bool refused = j < valid;
        const float* d = refused && p.draft ? d_of(j) : nullptr;
        const int skip = refused && !p.draft ? __shfl_sync(0xffffffffu, mine, j & 31) : -1;
        const float tp = p.probs ? 0.f : s_top[0], td = p.probs ? 0.f : s_top[1];
        const bool none = !p.probs && tp == -INFINITY;
        auto of_p = [&](float x, auto& pow32) { return p.probs ? fmax((double)x, 0.0) : weight64(x, tp, sc, pow32); };
        auto of_q = [&](float x, auto& pow32) { return p.probs ? fmax((double)x, 0.0) : td > -INFINITY ? weight64(x, td, sc, pow32) : 0.0; };
        // p - ratio q, ratio = sum of p / sum of q.  Which tokens have something left hardly hangs on it: those of a ratio good to float32
        // are taken, whose sums, p's and q's apart, then give what is left with the 64-bit ratio.  A token on the wrong side is one whose p and
        // rough q are within the ratios' difference of each other, and is off by that difference times its q: the sum of such q's says whether it
        // matters (2^-36 of what is left); then the tokens are taken anew by the 64-bit ratio.
        double rough = p.probs ? 1.0 : d && s_run[1] > 0.0 ? s_run[0] / s_run[1] : 0.0;
        double ratio = rough;
        bool sure = p.probs;
        for (int again = 0; again < 2 && !none;) {  // (a second time, from p itself, if nothing is left of p - q)
            const bool two = d && !again;
            // every warp of the cluster sums a run of tokens
            constexpr int kDeep = 4;
            constexpr double kNear = 0x1p-19;
            const int span = ((hi - lo + kWarps - 1) / kWarps + 31) & ~31, w0 = min(lo + warp * span, hi), w1 = min(w0 + span, hi);
            double sums[4] = {0.0, 0.0, 0.0, 0.0};  // p and q of the tokens that have something left, of all
            float close = 0.f;                      // q of those next to the border
#pragma unroll 1
            for (int base = w0; base < w1; base += 32 * kDeep) {
                const int e0 = base + lane;
                float x[kDeep], y[kDeep];
#pragma unroll
                for (int i = 0; i < kDeep; ++i) {
                    const int e = e0 + 32 * i;
                    x[i] = e < w1 ? __ldg(t + e) : p.probs ? 0.f : -INFINITY;
                    y[i] = two && e < w1 ? __ldg(d + e) : p.probs ? 0.f : -INFINITY;
                }
#pragma unroll
                for (int i = 0; i < kDeep; ++i) {
                    const double vx = of_p(x[i], from_lanes), vy = two ? of_q(y[i], from_lanes) : 0.0;
                    sums[2] += vx;
                    sums[3] += vy;
                    const double border = rough * vy;
                    if (two && (unsigned)(__double2hiint(vx) - __double2hiint(border) + 4) <= 8u) close += (float)vy;  // (within 4 steps of 2^-20 or finer)
                    if (two ? vx > border : e0 + 32 * i != skip || again) {
                        sums[0] += vx;
                        sums[1] += vy;
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) sums[k] = warp_sum64(sums[k]);
            close = warp_sum(close);
            __syncthreads();
            if (lane == 0 && warp < kWarps) {
                for (int k = 0; k < 4; ++k) s_sum[k][warp] = sums[k];
                s_sum[4][warp] = close;
            }
            cluster.sync();
            const int each_run = (C * kWarps + 31) / 32;
            for (int r = tid; r < C * kWarps; r += kThreads + 32) {
                const double* from = cluster.map_shared_rank(&s_sum[0][0], r / kWarps) + r % kWarps;
#pragma unroll
                for (int k = 0; k < kSums; ++k) s_all[k][r % each_run * 32 + r / each_run] = from[k * kWarps];  // (a lane's runs a row apart: other banks)
            }
            __syncthreads();
            // which run: the last one that is not empty and starts at or before the target, a lane some neighbouring runs.  (What runs
            // once is kept short: fetching instructions is what takes the time here.)
            if (warp == 0) {
                const int n = max(0, min(each_run, C * kWarps - lane * each_run));  // of the lane
                double zp = 0.0, zq = 0.0, near = 0.0;
                if (two && !p.probs) {
#pragma unroll 1
                    for (int r = 0; r < n; ++r) {
                        zp += s_all[2][r * 32 + lane];
                        zq += s_all[3][r * 32 + lane];
                        near += s_all[4][r * 32 + lane];
                    }
                    zp = warp_sum64(zp);
                    zq = warp_sum64(zq);
                    near = warp_sum64(near);
                    ratio = zq > 0.0 ? zp / zq : 0.0;
                }
                auto left = [&](int r) {
                    const double x = s_all[0][r * 32 + lane];
                    return two ? fmax(x - ratio * s_all[1][r * 32 + lane], 0.0) : x;
                };
                double part = 0.0;
#pragma unroll 1
                for (int r = 0; r < n; ++r) part += left(r);
                const double run = warp_scan64(part);
                const double total = __shfl_sync(0xffffffffu, run, 31), want = draw(p.draws[b]) * total;
                double before = run - part, start = 0.0;
                int found = -1;
#pragma unroll 1
                for (int r = 0; r < n; ++r) {
                    const double x = left(r);
                    if (x > 0.0 && before <= want) { found = lane * each_run + r; start = before; }
                    before += x;
                }
                const int last = __reduce_max_sync(0xffffffffu, found);
                if (last >= 0 && found == last) s_seg = want - start;
                if (lane == 0) {
                    const double off = fabs(rough - ratio);
                    s_found = two && !sure && (off > kNear * rough || off * near > 0x1p-36 * total) ? -2 : last;
                    s_run[2] = ratio;
                }
            }
            __syncthreads();
            const int found = s_found;
            ratio = s_run[2];
            if (found == -2) {
                rough = ratio;
                sure = true;
                cluster.sync();  // (the sums are read before they change)
                continue;
            }
            if (found >= 0) {
                if (found / kWarps == rank) {  // this CTA has the run: its threads take neighbouring tokens
                    const int f0 = min(lo + found % kWarps * span, hi), f1 = min(f0 + span, hi);
                    const int each = (span + kThreads - 1) / kThreads;
                    const int e0 = min(f0 + tid * each, f1), e1 = min(e0 + each, f1);
                    auto left = [&](int e) {
                        const double x = of_p(__ldg(t + e), from_table);
                        if (!two) return e == skip && !again ? 0.0 : x;
                        const double y = of_q(__ldg(d + e), from_table);
                        return x > rough * y ? fmax(x - ratio * y, 0.0) : 0.0;
                    };
                    double mine64 = 0.0;
#pragma unroll 1
                    for (int e = e0; e < e1; ++e) mine64 += left(e);
                    const double run = warp_scan64(mine64);
                    __syncthreads();
                    if (lane == 31 && warp < kWarps) s_run[warp] = run;
                    if (tid == 0) s_at = -1, s_hit = 0x7fffffff;
                    __syncthreads();
                    double cum = run - mine64;
#pragma unroll 1
                    for (int w = 0; w < warp; ++w) cum += s_run[w];
                    int hit = 0x7fffffff, last = -1;
#pragma unroll 1
                    for (int e = e0; e < e1; ++e) {
                        const double x = left(e);
                        cum += x;
                        if (x > 0.0) {
                            last = e;
                            if (cum > s_seg && hit == 0x7fffffff) hit = e;
                        }
                    }
                    hit = __reduce_min_sync(0xffffffffu, hit);
                    last = __reduce_max_sync(0xffffffffu, last);
                    if (lane == 0) { atomicMin(&s_hit, hit); atomicMax(&s_at, last); }
                    __syncthreads();
                    if (tid == 0) p.tokens[(int64_t)b * (p.K + 1) + j] = s_hit != 0x7fffffff ? s_hit : s_at;
                }
                token = -2;  // (written above)
                break;
            }
            cluster.sync();
            ++again;
        }
    }
    if (rank == 0 && tid == 0) {
        int32_t* out = p.tokens + (int64_t)b * (p.K + 1);
        for (int i = 0; i < j; ++i) out[i] = drafted[i];
        if (token != -2) out[j] = token;
        for (int i = j + 1; i <= p.K; ++i) out[i] = -1;
        p.accepted[b] = j;
    }
    cluster.sync();  // (shared memory stays until everybody has read it)
    if (tid == 0 && s_gave) p.accepted[b] = -1;
}

}  // namespace

extern "C" int first_verify(const float* target, int64_t target_seq_stride, int64_t target_row_stride, const float* draft,
                            int64_t draft_seq_stride, int64_t draft_row_stride, int32_t probs, const int32_t* drafted,
                            int32_t B, int32_t n_draft, int32_t vocab, const float* temperature, const float* uniforms,
                            const float* draws, int32_t* tokens, int32_t* accepted, void* stream) {
    if (B < 0 || n_draft < 0 || vocab <= 0) return FIRST_E_ARG;
    if (n_draft > FIRST_VERIFY_MAX_DRAFTS || vocab > FIRST_SAMPLE_MAX_VOCAB) return FIRST_E_UNSUPPORTED;
    if (target_seq_stride < 0 || target_row_stride < 0 || draft_seq_stride < 0 || draft_row_stride < 0) return FIRST_E_SHAPE;
    if (B == 0) return FIRST_OK;
    if (!target || !draws || !tokens || !accepted || (n_draft > 0 && (!drafted || !uniforms))) return FIRST_E_ARG;
    if ((n_draft > 0 && target_row_stride < vocab) || (draft && n_draft > 1 && draft_row_stride < vocab)) return FIRST_E_SHAPE;
    if (B > 1 && (target_seq_stride < vocab || (draft && n_draft > 0 && draft_seq_stride < vocab))) return FIRST_E_SHAPE;
    if (!words_ok({target, draft, drafted, temperature, uniforms, draws, tokens, accepted})) return FIRST_E_UNSUPPORTED;
    VerifyArgs a{};
    a.target = target; a.draft = n_draft > 0 ? draft : nullptr;
    a.t_seq = target_seq_stride; a.t_row = target_row_stride; a.d_seq = draft_seq_stride; a.d_row = draft_row_stride;
    a.drafted = drafted;
    a.u = uniforms; a.draws = draws; a.temperature = probs ? nullptr : temperature;
    a.tokens = tokens; a.accepted = accepted;
    a.B = B; a.K = n_draft; a.V = vocab;
    a.probs = probs != 0;
    // CTAs a sequence: two a multiprocessor in all, what that has room for (24 x 5 of 50257: 8 each 37 us, 16 each 49), or up to three while clusters are
    // small, as many sequences end early and the next ones shorten the last (180 x 4 of 64000: one each 186 us, two each 121; 80 x 3 of 32000: 57, 49).
    // Positions of the first round: several where there are few sequences and a round's latency is the time, one where there are many and the rows
    // behind a refusal cost more (5 drafts of 128256, most of them accepted | half: 1 sequence in rounds of 1, 2, 4, 8: 43, 41, 35, 39 | 27, 29, 35, 39 us;
    // 8: 51, 51, 49, 49 | 43, 45, 45, 51; 16: 57, 55, 59, 63 | 55, 55, 55, 64; 48: 127, 125, 125, 125 | 123, 121, 117, 127; 64: 127, 129, 123, 133 |
    // 109, 117, 135, 152; 100: 168, 173, 201, 219 | 152, 170, 203, 238; 24 x 5 looked up of 50257: 39, 38, 37, 37; 48 of them 47, 51, 47, 49 | 41, 37, 43, 49).
    a.C = 1;
    while (a.C < kMaxCluster && (int64_t)B * a.C * 2 <= (a.C < 4 ? 3 : 2) * kSMs && vocab > 4096 * a.C) a.C *= 2;
    a.R = B <= 8 ? 4 : B <= 48 ? 2 : 1;
    constexpr int kSmem = kRing * kPiece * 4;
    static std::atomic<uint64_t> done{0};
    if (allow_launch(verify_rows, kSmem, true, done) != cudaSuccess) return FIRST_E_CUDA;
    if (B > 0x7fffffff / kMaxCluster) return FIRST_E_CAPACITY;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)B * a.C);
    cfg.blockDim = dim3(kThreads + 32);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = a.C;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, verify_rows, a) == cudaSuccess ? FIRST_OK : FIRST_E_CUDA;
}
