// Rotary positions on caller-owned queries and keys, in place, and the frequencies of the usual long-context
// scalings.  (The paper names LLaMA-3 models and leaves the block to them; the step rotates by itself, see step_begin.)
#include <cmath>

#include "common.cuh"
#include "first.h"
#include "ops.h"

using namespace first;

namespace {

constexpr double kPi = 3.14159265358979323846;

struct RopeArgs {
    void *q, *k;
    int64_t q_tok, q_head, k_tok, k_head;  // strides in elements
    int Hq, H;                             // query heads, query + key heads
    int64_t tokens;
    int half;                              // rotated pairs per head
    int nv, hg;                            // vectors of pairs per head, head groups per token
    const int32_t* pos;
    const double* inv_freq;
    double factor;
    bool shared;                           // the block's cosines and sines are computed once for all its threads
};

// One pair: (a, b) -> (a c - b s, b c + a s).
template <typename T>
__device__ __forceinline__ void rotate(T& a, T& b, float2 cs) {
    const float x = to_f32(a), y = to_f32(b);
    a = from_f32<T>(x * cs.x - y * cs.y);
    b = from_f32<T>(y * cs.x + x * cs.y);
}

// An angle less its whole turns, to 64 bits (of angles up to 2^31; the sine's own way with large ones is a slow one).
__device__ __forceinline__ double turned(double angle) {
    constexpr double kTurn = 2.0 * kPi, kTurnLow = 2.4492935982947064e-16;  // 2 pi = their sum
    const double n = rint(angle * (1.0 / kTurn));
    return fma(-n, kTurnLow, fma(-n, kTurn, angle));
}
__device__ __forceinline__ float2 cos_sin(const RopeArgs& p, int64_t t, int i) {
    double s, c;
    sincos(turned((double)p.pos[t] * p.inv_freq[i]), &s, &c);
    return make_float2((float)(p.factor * c), (float)(p.factor * s));
}

// A thread takes V pairs of one token and every hg-th head of them.  Their cosines and sines are those of the step, bit for bit:
// formed in 64 bits and cut to 32 at the end.  That is some hundred instructions a pair, so a block computes those of its
// tokens once, into shared memory.  V = 16 bytes' worth of elements where the layout allows it, else 1.
// Bound by HBM: 32768 tokens of 32 + 8 heads of 128 in bfloat16 110.6 us, 6.1 TB/s (93 % of a copy); 32 tokens: launch.
template <typename T, int V, bool IL>
__global__ void __launch_bounds__(256) rope_rows(const RopeArgs p) {
    extern __shared__ __align__(16) float2 table[];
    const int64_t w0 = (int64_t)blockIdx.x * blockDim.x;
    const unsigned per = (unsigned)p.nv * p.hg;  // threads a token (2^31 at most)
    const int64_t t0 = w0 / per;
    const unsigned off = (unsigned)(w0 - t0 * per), at = off + threadIdx.x, in = at % per;
    const int dt = (int)(at / per), g = (int)(in / p.nv), v = (int)(in % p.nv);
    const int64_t t = t0 + dt;
    const float2* mine;
    if (p.shared) {
        const int n = (int)min(p.tokens - t0, (int64_t)((off + blockDim.x - 1) / per) + 1);
        for (int e = threadIdx.x; e < n * p.half; e += blockDim.x) table[e] = cos_sin(p, t0 + e / p.half, e % p.half);
        mine = table + dt * p.half + v * V;
        __syncthreads();
    } else {
        for (int i = 0; t < p.tokens && i < V; ++i) table[threadIdx.x * V + i] = cos_sin(p, t, v * V + i);
        mine = table + threadIdx.x * V;
    }
    if (t >= p.tokens) return;
    float2 cs[V];
#pragma unroll
    for (int i = 0; i < V; ++i) cs[i] = mine[i];
    struct alignas(sizeof(T) * V) Vec { T e[V]; };
    // halves: V first members at v*V, V second members half elements on; interleaved: 2V consecutive elements
    const int o0 = IL ? 2 * v * V : v * V, o1 = IL ? o0 + V : o0 + p.half;
    for (int h = g; h < p.H; h += p.hg) {
        T* row = h < p.Hq ? static_cast<T*>(p.q) + t * p.q_tok + h * p.q_head
                          : static_cast<T*>(p.k) + t * p.k_tok + (h - p.Hq) * p.k_head;
        Vec a = *reinterpret_cast<const Vec*>(row + o0), b = *reinterpret_cast<const Vec*>(row + o1);
        if constexpr (IL) {
            if constexpr (V == 1) {
                rotate(a.e[0], b.e[0], cs[0]);
            } else {
#pragma unroll
                for (int i = 0; i < V / 2; ++i) {
                    rotate(a.e[2 * i], a.e[2 * i + 1], cs[i]);
                    rotate(b.e[2 * i], b.e[2 * i + 1], cs[V / 2 + i]);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) rotate(a.e[i], b.e[i], cs[i]);
        }
        *reinterpret_cast<Vec*>(row + o0) = a;
        *reinterpret_cast<Vec*>(row + o1) = b;
    }
}

template <typename T, int V>
cudaError_t launch(RopeArgs p, bool interleaved, cudaStream_t st) {
    p.nv = p.half / V;
    // Heads per thread: one while the launch is small, more once the threads fill the GPU anyway.
    const int64_t one = p.tokens * p.nv * p.H, full = kSMs * 2048;
    const int per = (int)(one <= full ? 1 : one / full < 8 ? one / full : 8);
    p.hg = (p.H + per - 1) / per;
    // If an equal share of up to half as many fills whole blocks with whole tokens (or tokens with blocks), that one: a block's
    // cosines are then all its own (the large launch: 8 groups of 5 heads 110.6 us, 5 of 8 118.7).
    for (int h = p.hg; h <= 2 * p.hg && h <= p.H; ++h)
        if (p.H % h == 0 && (256 % ((int64_t)p.nv * h) == 0 || (int64_t)p.nv * h % 256 == 0)) {
            p.hg = h;
            break;
        }
    const int64_t blocks = (p.tokens * p.nv * p.hg + 255) / 256;
    // tokens that a block's threads can belong to; very wide heads (from 2048 pairs on) have a block within one head
    const int64_t most = (255 / ((int64_t)p.nv * p.hg) + 2) * p.half;
    p.shared = most <= 4096;
    const size_t smem = (p.shared ? most : 256 * V) * sizeof(float2);
    if (interleaved) rope_rows<T, V, true><<<(unsigned)blocks, 256, smem, st>>>(p);
    else rope_rows<T, V, false><<<(unsigned)blocks, 256, smem, st>>>(p);
    return cudaGetLastError();
}

// In-place rotation wants every element to belong to one (token, head): rows may not overlap.
bool strides_ok(int64_t tokens, int64_t heads, int64_t hd, int64_t ts, int64_t hs) {
    if (heads == 0) return true;
    if (ts < 0 || hs < 0) return false;
    if (heads > 1 && hs < hd) return false;
    if (tokens <= 1) return true;
    if (heads <= 1) return ts >= hd;
    return ts >= (heads - 1) * hs + hd || (ts >= hd && hs >= (tokens - 1) * ts + hd);
}

}  // namespace

extern "C" int first_rope_freqs(const first_rope_spec* s, double* inv_freq, double* factor) {
    if (!s || !inv_freq || !factor) return FIRST_E_ARG;
    if (s->rot_dim <= 0 || s->rot_dim % 2 || !(s->base > 0.0) || !std::isfinite(s->base)) return FIRST_E_ARG;
    if (s->scaling < FIRST_ROPE_NONE || s->scaling > FIRST_ROPE_YARN) return FIRST_E_ARG;
    const bool scaled = s->scaling != FIRST_ROPE_NONE;
    if (scaled && (!(s->factor >= 1.0) || !std::isfinite(s->factor))) return FIRST_E_ARG;
    if (s->scaling == FIRST_ROPE_LLAMA3 || s->scaling == FIRST_ROPE_YARN)
        if (s->trained_len <= 0 || !(s->low > 0.0) || !(s->high > s->low) || !std::isfinite(s->high)) return FIRST_E_ARG;
    if (s->scaling == FIRST_ROPE_YARN && !(s->base > 1.0)) return FIRST_E_ARG;
    const int half = s->rot_dim / 2;
    const double len = (double)s->trained_len;
    // YaRN ramps between the (fractional) dimensions that turn `high` and `low` times over the trained length
    auto dim = [&](double turns) { return s->rot_dim * std::log(len / (turns * 2.0 * kPi)) / (2.0 * std::log(s->base)); };
    double lo = 0.0, hi = 0.0;
    if (s->scaling == FIRST_ROPE_YARN) {
        lo = std::fmax(std::floor(dim(s->high)), 0.0);
        hi = std::fmin(std::ceil(dim(s->low)), s->rot_dim - 1.0);
    }
    for (int i = 0; i < half; ++i) {
        const double f = std::pow(s->base, -2.0 * i / (double)s->rot_dim);
        double keep = 1.0;  // share of the unscaled frequency; the rest is divided by the factor
        if (s->scaling == FIRST_ROPE_LINEAR) keep = 0.0;
        if (s->scaling == FIRST_ROPE_LLAMA3) keep = std::fmin(1.0, std::fmax(0.0, (len * f / (2.0 * kPi) - s->low) / (s->high - s->low)));
        if (s->scaling == FIRST_ROPE_YARN) keep = 1.0 - std::fmin(1.0, std::fmax(0.0, (i - lo) / std::fmax(hi - lo, 0.001)));
        inv_freq[i] = scaled ? keep * f + (1.0 - keep) * f / s->factor : f;
    }
    *factor = s->scaling == FIRST_ROPE_YARN ? 0.1 * std::log(s->factor) + 1.0 : 1.0;
    return FIRST_OK;
}

extern "C" int first_rope(void* q, int64_t q_token_stride, int64_t q_head_stride, int32_t n_q_heads, void* k,
                          int64_t k_token_stride, int64_t k_head_stride, int32_t n_kv_heads, int32_t dtype, int64_t tokens,
                          int32_t head_dim, int32_t rot_dim, const int32_t* pos, const double* inv_freq, float factor,
                          int32_t interleaved, void* stream) {
    if (tokens < 0 || n_q_heads < 0 || n_kv_heads < 0 || n_q_heads + (int64_t)n_kv_heads > 65536) return FIRST_E_ARG;
    if (dtype != FIRST_DTYPE_F32 && dtype != FIRST_DTYPE_BF16) return FIRST_E_ARG;
    if (head_dim <= 0 || rot_dim <= 0 || rot_dim % 2 || rot_dim > head_dim) return FIRST_E_SHAPE;
    if (head_dim > 65536) return FIRST_E_UNSUPPORTED;
    if (!strides_ok(tokens, n_q_heads, head_dim, q_token_stride, q_head_stride) ||
        !strides_ok(tokens, n_kv_heads, head_dim, k_token_stride, k_head_stride))
        return FIRST_E_SHAPE;
    if (tokens == 0 || n_q_heads + n_kv_heads == 0) return FIRST_OK;  // (an empty tensor's address may be NULL)
    if ((n_q_heads > 0 && !q) || (n_kv_heads > 0 && !k) || !pos || !inv_freq) return FIRST_E_ARG;
    RopeArgs p{};
    p.q = q; p.k = k;
    p.q_tok = q_token_stride; p.q_head = q_head_stride; p.k_tok = k_token_stride; p.k_head = k_head_stride;
    p.Hq = n_q_heads; p.H = n_q_heads + n_kv_heads;
    p.tokens = tokens;
    p.half = rot_dim / 2;
    p.pos = pos; p.inv_freq = inv_freq; p.factor = factor;
    if ((__int128)tokens * p.half * p.H > ((__int128)1 << 38)) return FIRST_E_CAPACITY;  // (grid size; 2^38 pairs = 1 TB of bfloat16)
    const int es = dtype == FIRST_DTYPE_BF16 ? 2 : 4, V = 16 / es;
    for (const void* ptr : {n_q_heads > 0 ? q : nullptr, n_kv_heads > 0 ? k : nullptr})
        if (reinterpret_cast<uintptr_t>(ptr) % es) return FIRST_E_UNSUPPORTED;
    auto aligned = [&](const void* ptr, int64_t ts, int64_t hs, int heads) {
        return !heads || ((reinterpret_cast<uintptr_t>(ptr) % 16) == 0 && (tokens == 1 || ts % V == 0) && (heads == 1 || hs % V == 0));
    };
    const bool wide = p.half % V == 0 && aligned(q, p.q_tok, p.q_head, n_q_heads) && aligned(k, p.k_tok, p.k_head, n_kv_heads);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (dtype == FIRST_DTYPE_BF16) e = wide ? launch<__nv_bfloat16, 8>(p, interleaved, st) : launch<__nv_bfloat16, 1>(p, interleaved, st);
    else e = wide ? launch<float, 4>(p, interleaved, st) : launch<float, 1>(p, interleaved, st);
    return e == cudaSuccess ? FIRST_OK : FIRST_E_CUDA;
}
