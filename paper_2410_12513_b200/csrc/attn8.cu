// Attention of a sequence's newest tokens over a paged 8-bit cache.
#include <algorithm>

#include <cooperative_groups.h>

#include "cache8.cuh"

using namespace first;
namespace cg = cooperative_groups;

namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kMaxCluster = 16;
constexpr float kLift = 7.f, kSlack = 8.f;  // weights are 2^(z - reference + kLift), the reference lags by kSlack at most

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// N 32-bit words that are read once (N = 1, 2 or 4).
template <int N>
__device__ __forceinline__ void stream_words(const uint8_t* p, uint32_t* w) {
    if constexpr (N == 4)
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
    else if constexpr (N == 2)
        asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
    else
        asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(w[0]) : "l"(p));
}

// A cluster takes a tile of query rows (tokens x query heads of a KV head) of one sequence; its CTAs and their warps cut
// the sequence's tokens among them, and join (maximum, sum, output) at the end, over shared memory and then over the
// cluster's.  The tensor cores see tokens as rows: S[16 tokens][8 columns] = K q, O[16 of hd][8 columns] += V' P.  A
// column is a query row, or with SPLIT (float32 queries) one half of a row: q = hi + lo and P = hi + lo, both halves'
// products added in float32, so that nothing is rounded to 11 bits.  8-bit values are halves exactly; q is scaled by a
// power of two into the halves' range; the pages' scales act on the float32 products.
// Fragments come straight from global memory: the order of hd within a product and the order of hd in O's rows are free,
// so a thread's share of a K row is 16 adjacent bytes, and of V rows too.
template <int HD, int NT, bool SPLIT, bool E4M3>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 3 : 2) attn8(const Attn8Args p, const int S) {
    constexpr int kRows = NT * 8 / (SPLIT ? 2 : 1), kCols = NT * 8, kSteps = HD / 16;
    constexpr int kRowWords = HD / 16;   // words of a K row that a thread holds (a quarter of the row)
    constexpr int kVWords = HD / 32;     // words of a V row that a thread holds (an eighth)
    constexpr int U = NT <= 2 ? 2 : 1;   // groups of 16 tokens a step
    constexpr int kPer = SPLIT ? 1 : 2;  // query rows a thread sees of 8 columns
    constexpr int kStride = HD + 16;     // of O in shared memory
    __shared__ __align__(16) __half s_q[kCols][HD + 8];
    __shared__ __align__(16) uint2 s_frag[NT > 2 ? kSteps * NT * 32 : 1];
    __shared__ __align__(16) float s_o[kRows * kStride];
    __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows], s_rs[kRows];
    __shared__ float s_cm[kRows], s_cl[kRows];            // this CTA's, read by the cluster
    __shared__ float s_w[kMaxCluster][kRows], s_inv[kRows];
    const Stamp stamp_guard(p.s.stamp);
    pdl_trigger();
    pdl_wait();
    const int rank = blockIdx.x % S, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    const int h = blockIdx.y;
    Seq8 q;
    if (!find_seq(p.s, blockIdx.x / S, q)) return;  // (the whole cluster)
    const int r0 = blockIdx.z * kRows, rows = min(kRows, q.n * p.G - r0);
    if (rows <= 0) return;
    const int64_t cap = p.s.width << p.c.shift;
    const int tok0 = r0 / p.G;
    const int first_lim = (int)min((int64_t)q.before + tok0 + 1, cap);
    const int end = (int)min((int64_t)q.before + (r0 + rows - 1) / p.G + 1, cap);  // tokens that any row sees
    const int groups = (end + 15) / 16, per = ((groups + S - 1) / S + U - 1) / U * U;
    const int t0 = min(rank * per, groups), t1 = min(t0 + per, groups);

    // ---- query rows as halves
    for (int r = warp; r < kRows; r += kWarps) {
        float f[HD / 32];
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) f[i] = 0.f;
        if (r < rows) {
            const int tok = (r0 + r) / p.G, head = h * p.G + (r0 + r) % p.G;
            const int64_t at = (q.start + tok) * p.q.tok + head * p.q.head;
            auto get = [&](int d) {
                return p.q.f32 ? static_cast<const float*>(p.q.p)[at + d] : to_f32(static_cast<const __nv_bfloat16*>(p.q.p)[at + d]);
            };
#pragma unroll
            for (int i = 0; i < HD / 32; ++i) {
                const int d = i * 32 + lane;
                f[i] = get(d);
                if (p.s.cs) {
                    constexpr int half = HD / 2;
                    const bool up = d >= half;
                    const float2 t = p.s.cs[(int64_t)q.seq * half + (up ? d - half : d)];
                    const float o = get(up ? d - half : d + half);
                    f[i] = up ? f[i] * t.x + o * t.y : f[i] * t.x - o * t.y;
                }
                const uint32_t m = __float_as_uint(f[i]) & 0x7fffffffu;
                amax = max(amax, m < 0x7f800000u ? m : 0u);
            }
        }
        amax = __reduce_max_sync(0xffffffffu, amax);
        // the row's largest magnitude goes to [2^13, 2^14); 2^126 at most, and its inverse is a float32 too
        const int e = max(min(140 - (int)(amax >> 23), 126), -126);
        const float up = __int_as_float((e + 127) << 23);
        if (lane == 0) s_rs[r] = __int_as_float((127 - e) << 23);
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) {
            const float x = f[i] * up;
            const __half hi = __float2half_rn(x);
            if constexpr (SPLIT) {
                s_q[2 * r][i * 32 + lane] = hi;
                s_q[2 * r + 1][i * 32 + lane] = __float2half_rn(x - __half2float(hi));
            } else {
                s_q[r][i * 32 + lane] = hi;
            }
        }
    }
    __syncthreads();
    // word w of a thread's share of a K row covers elements dim(w) .. dim(w) + 3
    auto dim = [&](int w) { return HD >= 64 ? (w / 4) * 64 + c * 16 + (w % 4) * 4 : c * 8 + w * 4; };
    uint2 qf[NT <= 2 ? kSteps * NT : 1];
    if constexpr (NT <= 2) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int n = 0; n < NT; ++n) qf[s * NT + n] = *reinterpret_cast<const uint2*>(&s_q[n * 8 + g][dim(s)]);
    } else {
        for (int i = warp; i < kSteps * NT; i += kWarps)
            s_frag[i * 32 + lane] = *reinterpret_cast<const uint2*>(&s_q[i % NT * 8 + g][dim(i / NT)]);
        __syncthreads();
    }
    int lim[NT][kPer];    // tokens that the thread's query rows see
    float rs[NT][kPer];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int r = n * (8 / (SPLIT ? 2 : 1)) + kPer * c + j;
            lim[n][j] = r < rows ? (int)min((int64_t)q.before + (r0 + r) / p.G + 1, cap) : end;
            rs[n][j] = s_rs[r] * p.scale * 1.44269504088896341f;
        }

    float o[NT][kSteps][4];
    float m[NT][kPer], l[NT][kPer];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][s][e] = 0.f;
#pragma unroll
        for (int j = 0; j < kPer; ++j) { m[n][j] = -INFINITY; l[n][j] = 0.f; }
    }

    uint32_t kw[U][2][kRowWords], vw[U][4][kVWords];
    // Step i of a warp covers groups t0 + (i * kWarps + warp) * U ..  Their pages and scales are looked up for 32 / U
    // steps at a time, one group a lane.
    int my_page = -1;
    float my_ks = 0.f, my_vs = 0.f;
    const int steps = t1 > t0 ? ((t1 - t0 + U - 1) / U - warp + kWarps - 1) / kWarps : 0;
    auto look_up = [&](int i) {
        const int t = t0 + ((i + lane / U) * kWarps + warp) * U + lane % U;
        my_page = -1;
        my_ks = my_vs = 0.f;
        if (t < t1) {
            my_page = find_page(p.s, p.c.n_pages, q.seq, t >> (p.c.shift - 4));
            if (my_page >= 0) {
                my_ks = p.c.ks[(int64_t)my_page * p.c.H + h];
                my_vs = p.c.vs[(int64_t)my_page * p.c.H + h];
            }
        }
    };
    auto row_of = [&](int i, int u) {  // first byte of group u's tokens of step i, -1: none
        const int pg = __shfl_sync(0xffffffffu, my_page, (i % (32 / U)) * U + u);
        const int t = t0 + (i * kWarps + warp) * U + u;
        return pg < 0 ? (int64_t)-1 : ((((int64_t)pg * p.c.H + h) << p.c.shift) + ((t * 16) & ((1 << p.c.shift) - 1))) * HD;
    };
    auto load_k = [&](int64_t at, uint32_t (&w)[2][kRowWords]) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (at < 0) {
#pragma unroll
                for (int i = 0; i < kRowWords; ++i) w[r][i] = 0;
                continue;
            }
            const uint8_t* a = p.c.k + at + (g + 8 * r) * HD;
            if constexpr (HD == 32) {
                stream_words<2>(a + c * 8, w[r]);
            } else {
#pragma unroll
                for (int i = 0; i < HD / 64; ++i) stream_words<4>(a + i * 64 + c * 16, w[r] + 4 * i);
            }
        }
    };
    auto load_v = [&](int64_t at, uint32_t (&w)[4][kVWords]) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (at < 0) {
#pragma unroll
                for (int i = 0; i < kVWords; ++i) w[r][i] = 0;
            } else {
                stream_words<kVWords>(p.c.v + at + (2 * c + (r & 1) + 8 * (r >> 1)) * HD + g * (HD / 8), w[r]);
            }
        }
    };
    int64_t at[U];
    float ks[U], vs[U];
    auto fetch_info = [&](int i, float (&a)[U], float (&b)[U], int64_t (&r)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            r[u] = row_of(i, u);
            a[u] = __shfl_sync(0xffffffffu, my_ks, (i % (32 / U)) * U + u);
            b[u] = __shfl_sync(0xffffffffu, my_vs, (i % (32 / U)) * U + u);
        }
    };
    if (steps > 0) {
        look_up(0);
        fetch_info(0, ks, vs, at);
#pragma unroll
        for (int u = 0; u < U; ++u) load_k(at[u], kw[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) load_v(at[u], vw[u]);
    }
    for (int i = 0; i < steps; ++i) {
        const int tb = (t0 + (i * kWarps + warp) * U) * 16;  // the step's first token
        float s[U][NT][4];
        // ---- S = K q
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[u][n][e] = 0.f;
#pragma unroll
            for (int w = 0; w < kSteps; ++w) {
                uint32_t a0, a1, a2, a3;
                to_halves<E4M3>(kw[u][0][w], a0, a2);
                to_halves<E4M3>(kw[u][1][w], a1, a3);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint2 b = NT <= 2 ? qf[NT <= 2 ? w * NT + n : 0] : s_frag[NT > 2 ? (w * NT + n) * 32 + lane : 0];
                    mma(s[u][n], a0, a1, a2, a3, b.x, b.y);
                }
            }
        }
        // ---- the next step's K
        int64_t at_n[U];
        float ks_n[U], vs_n[U];
        const bool more = i + 1 < steps;
        if (more) {
            if ((i + 1) % (32 / U) == 0) look_up(i + 1);
            fetch_info(i + 1, ks_n, vs_n, at_n);
#pragma unroll
            for (int u = 0; u < U; ++u) load_k(at_n[u], kw[u]);
        }
        // ---- weights
        const bool edge = tb + 16 * U > first_lim;  // some row does not see all of the step's tokens
        float z[U][NT][kPer][2];                    // [..][tokens g, g + 8]
        bool over = false;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const float f = ks[u] * rs[n][j];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        float v = (SPLIT ? s[u][n][2 * x] + s[u][n][2 * x + 1] : s[u][n][2 * x + j]) * f;
                        if (edge && tb + 16 * u + g + 8 * x >= lim[n][j]) v = -INFINITY;
                        if (at[u] < 0) v = -INFINITY;  // (no page: its tokens are not there)
                        z[u][n][j][x] = v;
                        over |= v > m[n][j] + kSlack;
                    }
                }
        if (__any_sync(0xffffffffu, over)) {  // the references move: to the maximum so far
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    float top = m[n][j];
#pragma unroll
                    for (int u = 0; u < U; ++u) top = fmaxf(top, fmaxf(z[u][n][j][0], z[u][n][j][1]));
#pragma unroll
                    for (int d = 4; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                    const float f = top == -INFINITY ? 1.f : exp2_fast(m[n][j] - top);
                    m[n][j] = top;
                    l[n][j] *= f;
#pragma unroll
                    for (int w = 0; w < kSteps; ++w) {
                        if constexpr (SPLIT) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[n][w][e] *= f;
                        } else {
                            o[n][w][j] *= f;
                            o[n][w][2 + j] *= f;
                        }
                    }
                }
        }
        uint32_t pb[U][NT][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    float w[kPer];
#pragma unroll
                    for (int j = 0; j < kPer; ++j) {
                        w[j] = exp2_fast(z[u][n][j][x] - (m[n][j] == -INFINITY ? 0.f : m[n][j]) + kLift);
                        l[n][j] += w[j];
                    }
                    __half2 v;
                    if constexpr (SPLIT) {
                        const __half hi = __float2half_rn(w[0]);
                        v = __halves2half2(hi, __float2half_rn(w[0] - __half2float(hi)));
                    } else {
                        v = __floats2half2_rn(w[0], w[kPer - 1]);
                    }
                    pb[u][n][x] = transpose8(*reinterpret_cast<uint32_t*>(&v));
                }
        // ---- O += V' P; what lies behind the last token is not a value
        if (tb + 16 * U > end) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (tb + 16 * u + 2 * c + (r & 1) + 8 * (r >> 1) >= end)
#pragma unroll
                        for (int w = 0; w < kVWords; ++w) vw[u][r][w] = 0;
        }
#pragma unroll
        for (int w = 0; w < kVWords; ++w) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                uint32_t a[2][2][2];  // [bytes 0,1 | 2,3][tokens 0.. | 8..][element]
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    to_halves<E4M3>(__byte_perm(vw[u][2 * x][w], vw[u][2 * x + 1][w], 0x5140), a[0][x][0], a[0][x][1]);
                    to_halves<E4M3>(__byte_perm(vw[u][2 * x][w], vw[u][2 * x + 1][w], 0x7362), a[1][x][0], a[1][x][1]);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        float t[4] = {0.f, 0.f, 0.f, 0.f};
                        mma(t, a[x][0][0], a[x][0][1], a[x][1][0], a[x][1][1], pb[u][n][0], pb[u][n][1]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[n][2 * w + x][e] = fmaf(t[e], vs[u], o[n][2 * w + x][e]);
                    }
            }
        }
        if (more) {
#pragma unroll
            for (int u = 0; u < U; ++u) load_v(at_n[u], vw[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) { at[u] = at_n[u]; ks[u] = ks_n[u]; vs[u] = vs_n[u]; }
        }
    }

    // ---- join the warps
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
#pragma unroll
            for (int d = 4; d < 32; d *= 2) l[n][j] += __shfl_xor_sync(0xffffffffu, l[n][j], d);
            if (g == 0) {
                const int r = n * (8 / (SPLIT ? 2 : 1)) + kPer * c + j;
                s_m[warp][r] = m[n][j];
                s_l[warp][r] = l[n][j];
            }
        }
    __syncthreads();
    for (int turn = 0; turn < kWarps; ++turn) {
        if (warp == turn) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const int r = n * (8 / (SPLIT ? 2 : 1)) + kPer * c + j;
                    float top = -INFINITY;
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_m[w][r]);
                    const float f = m[n][j] == -INFINITY ? 0.f : exp2_fast(m[n][j] - top);
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) {
                        // elements g * HD/8 + 2s and the next, kept at [s][g][2]
                        float2* dst = reinterpret_cast<float2*>(&s_o[r * kStride + s * 16 + g * 2]);
                        float2 v;
                        if constexpr (SPLIT) v = make_float2((o[n][s][0] + o[n][s][1]) * f, (o[n][s][2] + o[n][s][3]) * f);
                        else v = make_float2(o[n][s][j] * f, o[n][s][2 + j] * f);
                        if (turn > 0) {
                            const float2 had = *dst;
                            v.x += had.x;
                            v.y += had.y;
                        }
                        *dst = v;
                    }
                }
        }
        __syncthreads();
    }
    for (int r = tid; r < kRows; r += kThreads) {
        float top = -INFINITY, sum = 0.f;
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_m[w][r]);
        for (int w = 0; w < kWarps; ++w) sum += s_m[w][r] == -INFINITY ? (s_l[w][r] == s_l[w][r] ? 0.f : s_l[w][r]) : s_l[w][r] * exp2_fast(s_m[w][r] - top);
        s_cm[r] = top;
        s_cl[r] = sum;
    }
    // ---- join the cluster
    cg::cluster_group cluster = cg::this_cluster();
    if (S > 1) cluster.sync(); else __syncthreads();
    for (int r = tid; r < rows; r += kThreads) {
        float top = -INFINITY, sum = 0.f;
        for (int k = 0; k < S; ++k) top = fmaxf(top, S > 1 ? *cluster.map_shared_rank(&s_cm[r], k) : s_cm[r]);
        for (int k = 0; k < S; ++k) {
            const float cm = S > 1 ? *cluster.map_shared_rank(&s_cm[r], k) : s_cm[r];
            const float cl = S > 1 ? *cluster.map_shared_rank(&s_cl[r], k) : s_cl[r];
            const float f = cm == -INFINITY ? 0.f : exp2_fast(cm - top);
            s_w[k][r] = f;
            sum += cm == -INFINITY ? (cl == cl ? 0.f : cl) : cl * f;
        }
        s_inv[r] = sum == 0.f ? 0.f : 1.f / sum;  // (a row that sees nothing gives zeros)
    }
    __syncthreads();
    for (int e = rank * kThreads + tid; e < rows * HD; e += S * kThreads) {
        const int r = e / HD, d = e % HD;
        const int in = r * kStride + (d % (HD / 8)) / 2 * 16 + d / (HD / 8) * 2 + (d & 1);
        float v = 0.f;
        for (int k = 0; k < S; ++k) v = fmaf(S > 1 ? *cluster.map_shared_rank(&s_o[in], k) : s_o[in], s_w[k][r], v);
        v *= s_inv[r];
        const int tok = (r0 + r) / p.G, head = h * p.G + (r0 + r) % p.G;
        const int64_t to = (q.start + tok) * p.out.tok + head * p.out.head + d;
        if (p.out.p) {
            if (p.out.f32) static_cast<float*>(p.out.p)[to] = v;
            else static_cast<__nv_bfloat16*>(p.out.p)[to] = __float2bfloat16_rn(v);
        } else {
            const __nv_bfloat16 hi = __float2bfloat16_rn(v);
            p.out_hi[to] = hi;
            p.out_lo[to] = __float2bfloat16_rn(v - __bfloat162float(hi));
        }
    }
    if (S > 1) cluster.sync();  // (the others still read this CTA's part)
}

template <int HD, int NT, bool SPLIT, bool E4M3>
cudaError_t launch(const Attn8Args& a, int S, cudaStream_t st, bool pdl) {
    constexpr int kRows = NT * 8 / (SPLIT ? 2 : 1);
    auto kern = attn8<HD, NT, SPLIT, E4M3>;
    if (S > 8) {
        static const cudaError_t once = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (once != cudaSuccess) return once;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)a.s.B * S, a.c.H, (unsigned)(((int64_t)a.s.max_new * a.G + kRows - 1) / kRows));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = S;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, a, S);
}

template <int HD, bool SPLIT, bool E4M3>
cudaError_t launch_nt(const Attn8Args& a, cudaStream_t st, bool pdl, int n_sm) {
    const int64_t cols = (int64_t)a.s.max_new * a.G * (SPLIT ? 2 : 1);
    const int nt = cols <= 8 ? 1 : cols <= 16 ? 2 : 4;
    const int64_t tiles = (cols + 8 * nt - 1) / (8 * nt), items = (int64_t)a.s.B * a.c.H * tiles;
    // CTAs of a cluster: as many as keep some 8 waves of CTAs, at least 256 tokens of the longest possible sequence each
    const int64_t longest = a.s.width << a.c.shift;
    int S = 1;
    while (S < kMaxCluster && items * S < (int64_t)n_sm * 8 && longest > (int64_t)S * 256) S *= 2;
    switch (nt) {
        case 1: return launch<HD, 1, SPLIT, E4M3>(a, S, st, pdl);
        case 2: return launch<HD, 2, SPLIT, E4M3>(a, S, st, pdl);
        default: return launch<HD, 4, SPLIT, E4M3>(a, S, st, pdl);
    }
}

}  // namespace

namespace first {

cudaError_t attn8_launch(const Attn8Args& a, cudaStream_t st, bool pdl, int n_sm) {
#define FIRST_ATTN8(HD)                                                                                          \
    case HD:                                                                                                     \
        if (a.q.f32) return a.c.e4m3 ? launch_nt<HD, true, true>(a, st, pdl, n_sm) : launch_nt<HD, true, false>(a, st, pdl, n_sm); \
        return a.c.e4m3 ? launch_nt<HD, false, true>(a, st, pdl, n_sm) : launch_nt<HD, false, false>(a, st, pdl, n_sm);
    switch (a.c.hd) {
        FIRST_ATTN8(32)
        FIRST_ATTN8(64)
        default:
        FIRST_ATTN8(128)
    }
#undef FIRST_ATTN8
}

}  // namespace first

extern "C" int first_attn8(const first_cache8* cache, const void* q, int64_t q_token_stride, int64_t q_head_stride,
                           int32_t n_q_heads, int32_t dtype, float scale, const int32_t* cu_new, int32_t total,
                           const int32_t* pages, int32_t max_pages, const int32_t* len, int32_t B, int32_t max_new, void* out,
                           int64_t out_token_stride, int64_t out_head_stride, uint32_t* flags, void* stream) {
    int rc = check_cache8(cache);
    if (rc) return rc;
    const int hd = cache->head_dim;
    if ((rc = check_seqs8(pages, max_pages, len, cu_new, B, total, max_new))) return rc;
    if (n_q_heads <= 0) return FIRST_E_ARG;
    if (n_q_heads % cache->n_kv_heads) return FIRST_E_SHAPE;
    if ((rc = check_rows8(q, q_token_stride, q_head_stride, n_q_heads, hd, dtype, total, false)) ||
        (rc = check_rows8(out, out_token_stride, out_head_stride, n_q_heads, hd, dtype, total, true)))
        return rc;
    if (B == 0 || total == 0 || max_new == 0) return FIRST_OK;
    Attn8Args a;
    a.c = cache8_of(*cache);
    a.s.pages = pages; a.s.width = max_pages; a.s.len = len; a.s.cu = cu_new;
    a.s.B = B; a.s.total = total; a.s.max_new = std::min(max_new, total); a.s.flags = flags;
    a.G = n_q_heads / cache->n_kv_heads;
    if ((int64_t)max_pages * cache->page > (1 << 30) || (int64_t)a.s.max_new * a.G > (1 << 18) || B > (1 << 26)) return FIRST_E_CAPACITY;
    const bool f32 = dtype == FIRST_DTYPE_F32;
    a.q = Rows8{const_cast<void*>(q), q_token_stride, q_head_stride, f32};
    a.out = Rows8{out, out_token_stride, out_head_stride, f32};
    a.scale = scale;
    return attn8_launch(a, static_cast<cudaStream_t>(stream), false, kSMs) == cudaSuccess ? FIRST_OK : FIRST_E_CUDA;
}
