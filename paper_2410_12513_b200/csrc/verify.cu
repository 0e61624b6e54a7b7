// Verification of drafted tokens against the target's probabilities, from given random numbers.
#include <cfloat>

#include <cooperative_groups.h>

#include "common.cuh"
#include "first.h"
#include "ops.h"

using namespace first;
namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 16, kMaxRound = 8;

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

// One row's sum over one CTA's part, relative to the part's largest value; greedy rows: value and lowest index of the largest.
struct Part {
    double sum;
    float top;
    int32_t at;
};

// Logits as they count: NaN as -inf, +inf as the largest float32.
__device__ __forceinline__ float logit(float x) { return x > FLT_MAX ? FLT_MAX : (x == x ? x : -INFINITY); }
// Uniform draws as they count.
__device__ __forceinline__ double draw(float u) { return u < 1.f ? (double)fmaxf(u, 0.f) : (double)0x1.fffffep-1f; }

// exp((x - top) / T) in 64 bits: which token a draw falls on hangs on the sums of these.
__device__ __forceinline__ double weight(float x, float top, double inv_t) {
    x = logit(x);
    return x == -INFINITY ? 0.0 : exp(((double)x - (double)top) * inv_t);
}

struct Scale {
    float hi, lo, floor;  // log2(e) / T in two parts; differences below `floor` weigh nothing
    double inv_t;
};

// Sum of a row's weights over [lo, hi) by one block; float32 weights (their sum only decides about acceptance, where a
// relative error of 2^-22 moves the border of a draw by that much).
__device__ Part row_part(const float* row, int lo, int hi, const Scale& sc, bool greedy, Part* red) {
    const int tid = threadIdx.x;
    float top = -INFINITY;
    double sum = 0.0;
    int at = 0x7fffffff;
    auto batch = [&](const float* x, int n, const int* idx) {
        float big = -INFINITY;
        for (int i = 0; i < n; ++i) big = fmaxf(big, x[i]);
        if (greedy) {
            if (big > top || at == 0x7fffffff) {
                for (int i = n - 1; i >= 0; --i)
                    if (x[i] == big) at = idx[i];
                top = big;
            }
            return;
        }
        if (big > top) {
            sum *= top == -INFINITY ? 0.0 : exp(((double)top - (double)big) * sc.inv_t);
            top = big;
        }
        float part = 0.f;
        for (int i = 0; i < n; ++i) {
            const float t = fmaxf(x[i] - top, sc.floor);
            float w;
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(fmaf(t, sc.hi, t * sc.lo)));
            part += w;
        }
        sum += (double)part;
    };
    // head: up to the first 16-byte border, tail: after the last
    const int head = min(hi - lo, (int)((4 - ((reinterpret_cast<uintptr_t>(row + lo) >> 2) & 3)) & 3));
    const int body = (hi - lo - head) / 4, tail = lo + head + body * 4;
    if (tid < head || (tid >= 32 && tid - 32 < hi - tail)) {
        const int e = tid < head ? lo + tid : tail + tid - 32;
        const float x = logit(row[e]);
        batch(&x, 1, &e);
    }
    const float4* v = reinterpret_cast<const float4*>(row + lo + head);
    constexpr int kUnroll = 4;
    for (int i = tid; i < body; i += kUnroll * kThreads) {
        float x[4 * kUnroll];
        int idx[4 * kUnroll];
#pragma unroll
        for (int j = 0; j < kUnroll; ++j) {
            const int k = i + j * kThreads;
            const float4 f = k < body ? __ldg(v + k) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            x[4 * j] = logit(f.x); x[4 * j + 1] = logit(f.y); x[4 * j + 2] = logit(f.z); x[4 * j + 3] = logit(f.w);
#pragma unroll
            for (int e = 0; e < 4; ++e) idx[4 * j + e] = lo + head + 4 * k + e;
        }
        batch(x, 4 * kUnroll, idx);
    }
    // the warp's, then the block's
    float big = warp_max(top);
    if (greedy) {
        at = __reduce_min_sync(0xffffffffu, top == big ? at : 0x7fffffff);
    } else {
        sum *= top == -INFINITY ? 0.0 : (top == big ? 1.0 : exp(((double)top - (double)big) * sc.inv_t));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    }
    __syncthreads();  // (red may still be read)
    if ((tid & 31) == 0) red[tid >> 5] = Part{sum, big, at};
    __syncthreads();
    Part all{0.0, -INFINITY, 0x7fffffff};
    if (tid < 32) {
        const Part q = tid < kWarps ? red[tid] : Part{0.0, -INFINITY, 0x7fffffff};
        big = warp_max(q.top);
        all.top = big;
        all.at = __reduce_min_sync(0xffffffffu, q.top == big ? q.at : 0x7fffffff);
        all.sum = greedy || q.top == -INFINITY ? 0.0 : q.sum * (q.top == big ? 1.0 : exp(((double)q.top - (double)big) * sc.inv_t));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) all.sum += __shfl_xor_sync(0xffffffffu, all.sum, o);
    }
    return all;  // (threads 0..31)
}

__device__ __forceinline__ double block_sum(double x, double* red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < kWarps; ++w) s += red[w];
    return s;
}

// One cluster a sequence.  Rounds of R positions: every row's sum and largest logit, then the decisions (taken by every
// CTA alike), until one is refused or all are accepted; the rows of later positions are not read.  Then the new token's
// distribution, in 64 bits, over the one row (or two) that it comes from: those rows are in L2 by now.
__global__ void __launch_bounds__(kThreads) verify_rows(const VerifyArgs p) {
    __shared__ Part s_part[2][kMaxRound][2], s_red[kWarps];
    __shared__ double s_sum[kWarps], s_z[2], s_seg;
    __shared__ int s_ok[kMaxRound], s_hit, s_found;
    __shared__ float s_top[2];
    __shared__ int s_at;
    cg::cluster_group cluster = cg::this_cluster();
    const int C = p.C, b = blockIdx.x / C, rank = blockIdx.x % C, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const float temp = p.temperature ? p.temperature[b] : 1.f;
    const bool greedy = !p.probs && !(temp > 0.f);
    Scale sc;
    const double t64 = (double)fminf(fmaxf(temp, 1e-37f), 1e30f);
    sc.inv_t = 1.0 / t64;
    sc.hi = (float)(1.4426950408889634 / t64);
    sc.lo = (float)(1.4426950408889634 / t64 - (double)sc.hi);
    sc.floor = (float)(-200.0 * t64);
    const int32_t* drafted = p.drafted + (int64_t)b * p.K;
    // (at most 32 drafts: a lane each; the first that is no token ends them)
    const int mine = lane < p.K ? drafted[lane] : -1;
    const uint32_t closed = ~__ballot_sync(0xffffffffu, mine >= 0 && mine < p.V);
    const int valid = closed ? __ffs(closed) - 1 : 32;
    const int per = ((p.V + C - 1) / C + 3) & ~3, lo = min(rank * per, p.V), hi = min(lo + per, p.V);
    auto t_of = [&](int i) { return p.target + b * p.t_seq + i * p.t_row; };
    auto d_of = [&](int i) { return p.draft + b * p.d_seq + i * p.d_row; };
    int j = 0;  // the position whose token is new
    if (p.probs) {
        bool ok = false;
        if (lane < valid) {
            const double pd = fmax((double)t_of(lane)[mine], 0.0), qd = p.draft ? fmax((double)d_of(lane)[mine], 0.0) : 1.0;
            ok = draw(p.u[(int64_t)b * p.K + lane]) * qd < pd;
        }
        const uint32_t refused = ~__ballot_sync(0xffffffffu, ok);
        j = refused ? __ffs(refused) - 1 : 32;
    } else {
        bool open = true;
        for (int i0 = 0, round = 0; open; i0 += p.R, ++round) {
            const int n = min(p.R, valid + 1 - i0);
            for (int i = 0; i < n; ++i) {
                Part a = row_part(t_of(i0 + i), lo, hi, sc, greedy, s_red);
                if (tid == 0) s_part[round & 1][i][0] = a;
                if (p.draft && !greedy && i0 + i < valid) {
                    a = row_part(d_of(i0 + i), lo, hi, sc, false, s_red);
                    if (tid == 0) s_part[round & 1][i][1] = a;
                }
            }
            cluster.sync();
            if (warp < n) {  // one warp a position
                const int i = i0 + warp;
                double z[2] = {0.0, 0.0};
                float top[2] = {-INFINITY, -INFINITY};
                int at = 0x7fffffff;
                for (int side = 0; side < (p.draft && !greedy && i < valid ? 2 : 1); ++side) {
                    const Part q = lane < C ? *cluster.map_shared_rank(&s_part[round & 1][warp][side], lane) : Part{0.0, -INFINITY, 0x7fffffff};
                    top[side] = warp_max(q.top);
                    if (side == 0) at = __reduce_min_sync(0xffffffffu, q.top == top[0] ? q.at : 0x7fffffff);
                    z[side] = q.top == -INFINITY ? 0.0 : q.sum * exp(((double)q.top - (double)top[side]) * sc.inv_t);
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) z[side] += __shfl_xor_sync(0xffffffffu, z[side], o);
                }
                if (lane == 0) {
                    bool ok = false;
                    if (i < valid) {
                        const int d = drafted[i];
                        if (greedy) {
                            ok = d == at && top[0] > -INFINITY;
                        } else {
                            const double pd = z[0] > 0.0 ? weight(t_of(i)[d], top[0], sc.inv_t) / z[0] : 0.0;
                            const double qd = !p.draft ? 1.0 : z[1] > 0.0 ? weight(d_of(i)[d], top[1], sc.inv_t) / z[1] : 0.0;
                            ok = draw(p.u[(int64_t)b * p.K + i]) * qd < pd;
                        }
                    }
                    s_ok[warp] = ok;
                }
                __syncwarp();
                if (lane == 0) {  // (kept for the position that turns out to be the last)
                    s_red[warp] = Part{0.0, top[0], at};
                    s_sum[warp] = top[1];
                }
            }
            __syncthreads();
            int i = 0;
            while (i < n && s_ok[i]) ++i;
            if (i < n) {
                j = i0 + i;
                if (tid == 0) { s_top[0] = s_red[i].top; s_top[1] = (float)s_sum[i]; s_at = s_red[i].at; }
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
        const int skip = refused && !p.draft ? drafted[j] : -1;
        const float tp = p.probs ? 0.f : s_top[0], td = p.probs ? 0.f : s_top[1];
        const bool none = !p.probs && tp == -INFINITY;
        double ratio = 1.0;
        if (d && !p.probs && !none) {  // both rows' sums
            double zp = 0.0, zq = 0.0;
            for (int e = lo + tid; e < hi; e += kThreads) {
                zp += weight(t[e], tp, sc.inv_t);
                if (td > -INFINITY) zq += weight(d[e], td, sc.inv_t);
            }
            zp = block_sum(zp, s_sum);
            zq = block_sum(zq, s_sum);
            if (tid == 0) { s_z[0] = zp; s_z[1] = zq; }
            cluster.sync();
            zp = zq = 0.0;
            for (int k = 0; k < C; ++k) {
                zp += cluster.map_shared_rank(s_z, k)[0];
                zq += cluster.map_shared_rank(s_z, k)[1];
            }
            ratio = zq > 0.0 ? zp / zq : 0.0;
        }
        for (int again = 0; again < 2 && !none; ++again) {  // (a second time, from p itself, if nothing is left of p - q)
            auto left = [&](int e) {
                if (p.probs) {
                    const double a = fmax((double)t[e], 0.0);
                    if (again || !refused) return a;
                    return d ? fmax(a - fmax((double)d[e], 0.0), 0.0) : (e == skip ? 0.0 : a);
                }
                const double a = weight(t[e], tp, sc.inv_t);
                if (again || !refused) return a;
                return d ? fmax(a - (td > -INFINITY ? ratio * weight(d[e], td, sc.inv_t) : 0.0), 0.0) : (e == skip ? 0.0 : a);
            };
            // every warp of the cluster sums a run of tokens
            const int span = ((hi - lo + kWarps - 1) / kWarps + 31) & ~31, w0 = min(lo + warp * span, hi), w1 = min(w0 + span, hi);
            double sum = 0.0;
            for (int e = w0 + lane; e < w1; e += 32) sum += left(e);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            __syncthreads();
            if (lane == 0) s_sum[warp] = sum;
            cluster.sync();
            // which run: the last one that is not empty and starts at or before the target, a lane some neighbouring runs
            if (warp == 0) {
                const int n = C * kWarps, each = (n + 31) / 32;
                double x[kMaxCluster * kWarps / 32], part = 0.0;
#pragma unroll
                for (int i = 0; i < kMaxCluster * kWarps / 32; ++i) {
                    const int r = lane * each + i;
                    x[i] = i < each && r < n ? cluster.map_shared_rank(s_sum, r / kWarps)[r % kWarps] : 0.0;
                    part += x[i];
                }
                double run = part;
#pragma unroll
                for (int o = 1; o < 32; o *= 2) {
                    const double y = __shfl_up_sync(0xffffffffu, run, o);
                    if (lane >= o) run += y;
                }
                const double want = draw(p.draws[b]) * __shfl_sync(0xffffffffu, run, 31);
                double before = __shfl_up_sync(0xffffffffu, run, 1), start = 0.0;
                if (lane == 0) before = 0.0;
                int found = -1;
#pragma unroll
                for (int i = 0; i < kMaxCluster * kWarps / 32; ++i) {
                    if (x[i] > 0.0 && before <= want) { found = lane * each + i; start = before; }
                    before += x[i];
                }
                const int last = __reduce_max_sync(0xffffffffu, found);
                if (last >= 0 && found == last) s_seg = want - start;
                if (lane == 0) s_found = last;
            }
            __syncthreads();
            const int found = s_found;
            if (found >= 0) {
                if (found / kWarps == rank) {  // this CTA has the run: its threads take neighbouring tokens
                    const int f0 = min(lo + found % kWarps * span, hi), f1 = min(f0 + span, hi);
                    const int each = (span + kThreads - 1) / kThreads;
                    const int e0 = min(f0 + tid * each, f1), e1 = min(e0 + each, f1);
                    double mine = 0.0;
                    for (int e = e0; e < e1; ++e) mine += left(e);
                    double run = mine;
#pragma unroll
                    for (int o = 1; o < 32; o *= 2) {
                        const double y = __shfl_up_sync(0xffffffffu, run, o);
                        if (lane >= o) run += y;
                    }
                    __syncthreads();
                    if (lane == 31) s_red[warp].sum = run;
                    if (tid == 0) s_at = -1, s_hit = 0x7fffffff;
                    __syncthreads();
                    double cum = run - mine;
                    for (int w = 0; w < warp; ++w) cum += s_red[w].sum;
                    int hit = 0x7fffffff, last = -1;
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
            cluster.sync();  // (the sums are read before they change)
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
    VerifyArgs a{};
    a.target = target; a.draft = n_draft > 0 ? draft : nullptr;
    a.t_seq = target_seq_stride; a.t_row = target_row_stride; a.d_seq = draft_seq_stride; a.d_row = draft_row_stride;
    a.drafted = drafted;
    a.u = uniforms; a.draws = draws; a.temperature = probs ? nullptr : temperature;
    a.tokens = tokens; a.accepted = accepted;
    a.B = B; a.K = n_draft; a.V = vocab;
    a.probs = probs != 0;
    // CTAs a sequence: two a multiprocessor in all (more where that leaves most idle); positions a round: all where there are few sequences, as the
    // GPU has room for them at once, else one, so that rows behind a refusal are not read
    a.C = 1;
    while (a.C < kMaxCluster && (int64_t)B * a.C * 2 <= 2 * kSMs && vocab > 4096 * a.C) a.C *= 2;
    a.R = B <= 8 ? kMaxRound : B <= 24 ? 2 : 1;
    static const cudaError_t once = cudaFuncSetAttribute(verify_rows, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (once != cudaSuccess) return FIRST_E_CUDA;
    if (B > 0x7fffffff / kMaxCluster) return FIRST_E_CAPACITY;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)B * a.C);
    cfg.blockDim = dim3(kThreads);
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
