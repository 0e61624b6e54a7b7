// Next tokens of a batch with generation settings of its own for every request (the paper samples with temperature
// 0.8 and top-k 10, appendix "Training and Inference Setup"; requests of one batch need not agree on that).
//
// A row's candidates stand in descending order of their logits, equal ones by index.  Every filter keeps a prefix of
// that order, and so does a draw: the token is the first candidate whose cumulative weight exceeds u times the sum.
// All three are the same question -- where does a running sum (of ones, or of weights) reach a target -- and it is
// answered without sorting, by a digit-wise search: the keys' top digit is counted into a histogram, the digit
// that holds the target is found, and the search goes on among the elements with that digit.  Weights are integers
// (multiples of 2^-43 of the largest), so sums are exact whatever their order and the result is reproducible.
#include "common.cuh"
#include "first.h"
#include "ops.h"

namespace first {
namespace {

constexpr int kThreads = 1024, kBins = 2048;
constexpr double kUnit = 8796093022208.0;  // 2^43: sums of 2^19 weights stay below 2^63

struct RowParams {
    float m;
    double inv_T_div;  // the temperature
    float min_p;
};

// descending: the largest logit has the smallest key; -0 equals +0
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return (b & 0x80000000u) ? b : ~(b | 0x80000000u);
}
__device__ __forceinline__ float clean(float x) { return x != x ? -INFINITY : x; }

// weight in units of 2^-43, or -1 when the element is no candidate
__device__ __forceinline__ long long weight_of(float x, const RowParams& r) {
    if (!(x > -INFINITY)) return -1;
    const double w = x == r.m ? 1.0 : exp(((double)x - (double)r.m) / r.inv_T_div);
    if (!(w >= (double)r.min_p)) return -1;
    return __double2ll_rn(w * kUnit);
}

struct Shared {
    unsigned long long mass[kBins];
    unsigned int cnt[kBins];
    unsigned long long pre, hit;
    unsigned long long total_mass, total_cnt;
    float red[32];
    int redi[32];
};

// First element, in key order, at which the running sum (of weights, or of ones with by_rank) reaches target >= 1,
// among the candidates whose composite key is at most `limit`; the total is at least target.  Returns its composite key
// (value key << 20 | index); *incl = the sum of WEIGHTS up to and with it.
__device__ unsigned long long search(const float* row, int V, const RowParams& rp, unsigned long long limit,
                                     unsigned long long target, bool by_rank, Shared& s, unsigned long long* incl) {
    unsigned long long prefix = 0, before = 0, before_mass = 0;
    int bits = 52;
    while (bits > 0) {
        const int d = bits >= 11 ? 11 : bits, shift = bits - d;
        for (int i = threadIdx.x; i < kBins; i += kThreads) { s.mass[i] = 0; s.cnt[i] = 0; }
        __syncthreads();
        for (int i = threadIdx.x; i < V; i += kThreads) {
            const float x = clean(row[i]);
            const unsigned long long key = ((unsigned long long)key_of(x) << 20) | (unsigned)i;
            if (key > limit || (bits < 52 && (key >> bits) != prefix)) continue;
            const long long w = weight_of(x, rp);
            if (w < 0) continue;
            const int bin = (int)((key >> shift) & ((1u << d) - 1u));
            atomicAdd(&s.mass[bin], (unsigned long long)w);
            atomicAdd(&s.cnt[bin], 1u);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            unsigned long long run = before, runm = before_mass;
            int b = 0;
            for (; b < (1 << d); ++b) {
                const unsigned long long a = by_rank ? s.cnt[b] : s.mass[b];
                if (run + a >= target) break;
                run += a;
                runm += s.mass[b];
            }
            s.hit = (unsigned)b;
            s.pre = run;
            s.total_mass = runm;
            s.total_cnt = b < (1 << d) ? s.mass[b] : 0;
        }
        __syncthreads();
        prefix = (prefix << d) | s.hit;
        before = s.pre;
        before_mass = s.total_mass;
        *incl = before_mass + s.total_cnt;
        bits = shift;
        __syncthreads();
    }
    return prefix;
}

__global__ void __launch_bounds__(kThreads) sample_rows(const SampleArgs p) {
    const Stamp stamp_guard(p.stamp);
    __shared__ Shared s;
    pdl_trigger();
    pdl_wait();
    const int b = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float* row = p.logits + (int64_t)b * p.ld;
    float best = -INFINITY;
    int at = 0x7fffffff;
    for (int i = threadIdx.x; i < p.V; i += kThreads) {
        const float x = clean(row[i]);
        if (x > best) { best = x; at = i; }
    }
    for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const float v = __shfl_xor_sync(0xffffffffu, best, o);
            const int j = __shfl_xor_sync(0xffffffffu, at, o);
            if (v > best || (v == best && j < at)) { best = v; at = j; }
        }
        if (r == 0) {
            if (lane == 0) { s.red[warp] = best; s.redi[warp] = at; }
            __syncthreads();
            best = s.red[lane];
            at = s.redi[lane];
        }
    }
    if (threadIdx.x == 0 && p.pos) p.pos[b] += 1;
    const float T = p.temperature ? p.temperature[b] : 1.f;
    if (best == -INFINITY || !(T > 0.f)) {  // nothing to choose from, or greedy
        if (threadIdx.x == 0) p.tokens[b] = best == -INFINITY ? -1 : at;
        return;
    }
    RowParams rp;
    rp.m = best;
    rp.inv_T_div = (double)T;
    const float mp = p.min_p ? p.min_p[b] : 0.f;
    rp.min_p = mp > 0.f ? fminf(mp, 1.f) : 0.f;
    // candidates and their weight
    if (threadIdx.x == 0) { s.total_mass = 0; s.total_cnt = 0; }
    __syncthreads();
    unsigned long long mass = 0;
    unsigned cnt = 0;
    for (int i = threadIdx.x; i < p.V; i += kThreads) {
        const long long w = weight_of(clean(row[i]), rp);
        if (w >= 0) { mass += (unsigned long long)w; ++cnt; }
    }
    atomicAdd(&s.total_mass, mass);
    atomicAdd(&s.total_cnt, (unsigned long long)cnt);
    __syncthreads();
    unsigned long long Z = s.total_mass, n = s.total_cnt, limit = ~0ull;
    __syncthreads();
    const int k = p.top_k ? p.top_k[b] : 0;
    if (k > 0 && (unsigned long long)k < n) limit = search(row, p.V, rp, limit, (unsigned long long)k, true, s, &Z);
    const float tp = p.top_p ? p.top_p[b] : 1.f;
    if (tp < 1.f) {
        const double want = ceil((double)fmaxf(tp, 0.f) * (double)Z);
        unsigned long long t = want < 1.0 ? 1ull : (unsigned long long)want;
        limit = search(row, p.V, rp, limit, t < Z ? t : Z, false, s, &Z);
    }
    const float u0 = p.u[b], u = u0 >= 0.f ? fminf(u0, 0.99999994f) : (u0 < 0.f ? 0.f : 0.99999994f);
    const unsigned long long t = (unsigned long long)floor((double)u * (double)Z) + 1ull;
    unsigned long long unused;
    const unsigned long long key = search(row, p.V, rp, limit, t < Z ? t : Z, false, s, &unused);
    if (threadIdx.x == 0) p.tokens[b] = (int)(key & 0xfffffull);
}

}  // namespace

cudaError_t sample_launch(const SampleArgs& a, cudaStream_t st, bool pdl) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(a.B);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, sample_rows, a);
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
