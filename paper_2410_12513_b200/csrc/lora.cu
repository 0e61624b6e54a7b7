// Low-rank adapters of many requests beside a shared projection (the paper's "LoRA Compensation Module" keeps one
// adapter merged into the weights; here every row of a batch may have its own):
//   y[r] += scale[a] * B_a (A_a x[r]),  a = adapter of row r.
//
// Bound by the adapters' bytes at few rows, by y's (read and written) at many; the products are small.  One launch does both:
// rows of one adapter are taken together, up to TR of them (a tile), so that its A and B are read once for all of
// them; a cluster of eight CTAs works on a tile:
//   shrink   h = A x on the tensor cores (mma.sync m16n8k16, rank rows x batch rows: the products are far too small for
//            128-row tcgen05 tiles), the input features split over the CTAs and their warps
//   combine  every CTA adds the eight partial sums up from the cluster's shared memory, in a fixed order
//   expand   y += B h, the output features split over the CTAs (and over several clusters when tiles are few; each of
//            those computes h again, from L2)
// All operands enter exactly: float32 values as three bfloat16 terms (8 bits each), h too; of their products those
// below 2^-26 are left out.  Infinities, and float32 values that round to one in bfloat16, meet terms of zero there: a sum that
// is not finite is formed again in plain float32.  How the sums are ordered depends on the sizes k, n, rank alone, so a row's result does not depend on
// the rows around it.
//
// Measured (on the device; adapters, x and y larger than L2 in turn): 1 row of q|k|v at rank 8 6.3 us, 32 rows of 16 adapters 9.9 us (1.1 TB/s),
// 256 rows of 64 adapters at the down projection 34.0 us (2.9 TB/s; the shrink, which streams A, is more than half of it), 1024 rows of 8
// adapters at gate|up 46.1 us (2.7 TB/s; y begins to move after 12 us of plan, shrink and meeting; 44.8 without the look for
// sums that are not finite).
#include <algorithm>
#include <type_traits>

#include <cooperative_groups.h>

#include "common.cuh"
#include "first.h"
#include "ops.h"

namespace first {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256, kWarps = 8, kCluster = 8;
constexpr int kParts = 8;           // (16-row tile of A, share of the input features) pairs a CTA cuts its part of the shrink into, about
constexpr int kMaxRows = 1024;      // rows of a launch (the ids are sorted into tiles by every CTA)
constexpr int kMaxSize = 1 << 30;   // input, output features (numbers of them are rounded up to tiles in 32 bits)
constexpr int kMaxIds = 4096;       // adapters that can be; with more, every row is a tile of its own

// (x, y) -> packed bfloat16 pairs: term 0 the nearest bfloat16, the others what is left (nothing, of an infinity or NaN)
template <int N>
__device__ __forceinline__ void split(float x, float y, uint32_t (&t)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
        t[i] = *reinterpret_cast<const uint32_t*>(&h);
        const float xh = bf_lo(t[i]), yh = bf_hi(t[i]);
        x = fabsf(xh) < INFINITY ? x - xh : 0.f;
        y = fabsf(yh) < INFINITY ? y - yh : 0.f;
    }
}
// The same of one value, the largest among them: a finite one has finite terms.
__device__ __forceinline__ void split_one(float x, uint16_t (&t)[3]) {
    constexpr float kMost = 3.3895313892515355e38f;  // of bfloat16
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const float c = fabsf(x) < INFINITY ? fminf(fmaxf(x, -kMost), kMost) : x;
        const __nv_bfloat16 h = __float2bfloat16_rn(c);
        t[i] = __bfloat16_as_ushort(h);
        const float v = __bfloat162float(h);
        x = fabsf(v) < INFINITY ? x - v : 0.f;
    }
}
__device__ __forceinline__ float largest(float a, float b, float c) {  // of the absolute values; NaN where one is
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight (or four) consecutive elements as pairs of bfloat16, in N terms.
template <int N, int E>
struct Frag {
    uint32_t t[N][E / 2];
    __device__ __forceinline__ void keep_if(bool live) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < E / 2; ++e) t[i][e] = live ? t[i][e] : 0;
    }
};
template <typename T, int E>
__device__ __forceinline__ Frag<sizeof(T) == 2 ? 1 : 3, E> load_frag(const T* p) {
    Frag<sizeof(T) == 2 ? 1 : 3, E> f;
    if constexpr (sizeof(T) == 2) {
        if constexpr (E == 8) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
            f.t[0][0] = v.x; f.t[0][1] = v.y; f.t[0][2] = v.z; f.t[0][3] = v.w;
        } else {
            const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
            f.t[0][0] = v.x; f.t[0][1] = v.y;
        }
    } else {
#pragma unroll
        for (int q = 0; q < E / 4; ++q) {
            const float4 v = __ldg(reinterpret_cast<const float4*>(p) + q);
            uint32_t t[3];
            split(v.x, v.y, t);
#pragma unroll
            for (int i = 0; i < 3; ++i) f.t[i][2 * q] = t[i];
            split(v.z, v.w, t);
#pragma unroll
            for (int i = 0; i < 3; ++i) f.t[i][2 * q + 1] = t[i];
        }
    }
    return f;
}

// Four elements of a thread's own copy.
template <typename WT>
__device__ __forceinline__ Frag<sizeof(WT) == 2 ? 1 : 3, 4> shared_frag(const void* p) {
    Frag<sizeof(WT) == 2 ? 1 : 3, 4> f;
    if constexpr (sizeof(WT) == 2) {
        const uint2 v = *static_cast<const uint2*>(p);
        f.t[0][0] = v.x;
        f.t[0][1] = v.y;
    } else {
        const float4 v = *static_cast<const float4*>(p);
        uint32_t a[3], b[3];
        split(v.x, v.y, a);
        split(v.z, v.w, b);
#pragma unroll
        for (int i = 0; i < 3; ++i) { f.t[i][0] = a[i]; f.t[i][1] = b[i]; }
    }
    return f;
}

// 16 (8) bytes from global to shared memory in the background; with live = false zeros
template <int N>
__device__ __forceinline__ void copy_async(void* to, const void* from, bool live) {
    const uint32_t a = (uint32_t)__cvta_generic_to_shared(to);
    const int n = live ? N : 0;
    if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(a), "l"(from), "r"(n) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(a), "l"(from), "r"(n) : "memory");
}
__device__ __forceinline__ void copy_word(void* to, int word, const void* from, bool live) {
    const uint32_t a = (uint32_t)__cvta_generic_to_shared(to) + 4 * word;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(a), "l"(from), "r"(live ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The tensor cores and the cluster's barriers want whole warps, so nothing between them branches on a lane's own values:
// what a lane has no element for is loaded from an address that is good and dropped, or is a predicated instruction.
__device__ __forceinline__ void prefetch_if(const void* p, bool live) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %1, 0;\n @p prefetch.global.L2 [%0];\n}" ::"l"(p), "r"((uint32_t)live));
}
template <typename T>
__device__ __forceinline__ T load_if(const T* p, bool live) {
    T v;
    if constexpr (sizeof(T) == 4) {
        uint32_t u;
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %2, 0;\n mov.b32 %0, 0;\n @p ld.global.b32 %0, [%1];\n}" : "=r"(u) : "l"(p), "r"((uint32_t)live) : "memory");
        memcpy(&v, &u, 4);
    } else {
        uint16_t u;
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %2, 0;\n mov.b16 %0, 0;\n @p ld.global.b16 %0, [%1];\n}" : "=h"(u) : "l"(p), "r"((uint32_t)live) : "memory");
        memcpy(&v, &u, 2);
    }
    return v;
}
template <typename T>
__device__ __forceinline__ void store_if(T* p, T v, bool live) {
    if constexpr (sizeof(T) == 4) {
        uint32_t u;
        memcpy(&u, &v, 4);
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %2, 0;\n @p st.global.b32 [%0], %1;\n}" ::"l"(p), "r"(u), "r"((uint32_t)live) : "memory");
    } else {
        uint16_t u;
        memcpy(&u, &v, 2);
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %2, 0;\n @p st.global.b16 [%0], %1;\n}" ::"l"(p), "h"(u), "r"((uint32_t)live) : "memory");
    }
}
__device__ __forceinline__ void store16_if(void* p, const uint4& v, bool live) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %5, 0;\n @p st.global.v4.b32 [%0], {%1, %2, %3, %4};\n}" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z),
                 "r"(v.w), "r"((uint32_t)live) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

__host__ __device__ constexpr int steps_ahead(int rows) { return rows == 8 ? 2 : 3; }

template <int XK>
__device__ __forceinline__ float x_at(const LoraArgs& p, int64_t i) {
    if constexpr (XK == kLoraXF32) return static_cast<const float*>(p.x)[i];
    const float v = __bfloat162float(static_cast<const __nv_bfloat16*>(p.x)[i]);
    if constexpr (XK == kLoraXPair) return fabsf(v) < INFINITY ? v + __bfloat162float(static_cast<const __nv_bfloat16*>(p.x_lo)[i]) : v;
    return v;
}

struct Plan {
    int tiles;          // clusters = tiles * slices
    int slices;         // parts of the output features
    int direct;         // 1: tile t is row t
    int mt, ks;         // 16-row tiles of A; shares that the input features of one are cut into
    int h_stride;       // of a batch row's h, in bfloat16
    int h_bytes;        // of all of h
    int y_vec;          // y's rows are 16-byte aligned
};

// XK: LoraX.  WT: type of the adapters.  TR: rows of a tile (8 or 32).  OCC: CTAs a
// multiprocessor has room for (2: 128 registers a thread; 4: 64, for grids that want the room).
template <int XK, typename WT, typename YT, int TR, int OCC>
__global__ void __launch_bounds__(kThreads, OCC) lora_tiles(const LoraArgs p, const Plan pl) {
    const Stamp stamp_guard(p.stamp);
    constexpr int NT = TR / 8, NX = XK == kLoraXBf16 ? 1 : XK == kLoraXPair ? 2 : 3, NW = sizeof(WT) == 2 ? 1 : 3;
    using XT = typename std::conditional<XK == kLoraXF32, float, __nv_bfloat16>::type;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int rows_s[TR];     // the tile's rows
    __shared__ int tile_s[2];      // adapter, rows
    __shared__ int warp_s[kWarps];
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), lane = threadIdx.x & 31, tid = threadIdx.x;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);  // (the same in every lane, for the compiler too)
    const int g = lane >> 2, t = lane & 3;
    const int tile = (int)(blockIdx.x / kCluster) % pl.tiles, slice = (int)(blockIdx.x / kCluster) / pl.tiles;
    pdl_trigger();
    pdl_wait();
    const int m = p.m_dev ? max(0, min(p.m, *p.m_dev - p.row0)) : p.m;
    auto id_of = [&](int i) {
        const int a = p.adapter[p.idx ? p.idx[i] : i];
        return a >= 0 && a < p.n ? a : -1;
    };

    // ---- the tile: which adapter, which rows
    if (pl.direct) {
        if (tid == 0) {
            tile_s[0] = tile < m ? id_of(tile) : -1;
            tile_s[1] = 1;
        }
        if (tid < TR) rows_s[tid] = tile;
        __syncthreads();
    } else if (p.m <= 32) {
        // one warp sees all rows: every TR-th row of an adapter opens a tile, tile t belongs to the t-th of those
        if (warp == 0) {
            const int id = lane < m ? id_of(lane) : -1;
            const unsigned same = __match_any_sync(0xffffffffu, id);
            const int nth = __popc(same & ((1u << lane) - 1u));  // among its adapter's rows
            const unsigned opens = __ballot_sync(0xffffffffu, id >= 0 && nth % TR == 0);
            const int lead = tile < __popc(opens) ? (int)__fns(opens, 0, tile + 1) : -1;
            if (lead < 0) {
                if (lane == 0) tile_s[0] = -1;
            } else {
                const int a = __shfl_sync(0xffffffffu, id, lead), n0 = __shfl_sync(0xffffffffu, nth, lead);
                const unsigned mine = __ballot_sync(0xffffffffu, id == a && nth >= n0 && nth < n0 + TR);
                if (lane < TR) rows_s[lane] = lead;  // (columns beyond the tile's rows: read, never written)
                __syncwarp();
                if (id == a && nth >= n0 && nth < n0 + TR) rows_s[nth - n0] = lane;
                if (lane == 0) {
                    tile_s[0] = a;
                    tile_s[1] = __popc(mine);
                }
            }
        }
        __syncthreads();
    } else {
        // rows per adapter; adapter a then has ceil(rows / TR) tiles, in the order of the ids
        int* cnt = reinterpret_cast<int*>(smem);                    // [n]
        int* ids = cnt + ((p.n + 3) & ~3);                          // [m]
        int own[kMaxRows / kThreads];
#pragma unroll
        for (int q = 0; q < kMaxRows / kThreads; ++q) own[q] = tid + q * kThreads < m ? id_of(tid + q * kThreads) : -1;
        for (int i = tid; i < p.n; i += kThreads) cnt[i] = 0;
        __syncthreads();
#pragma unroll
        for (int q = 0; q < kMaxRows / kThreads; ++q) {
            if (tid + q * kThreads < m) ids[tid + q * kThreads] = own[q];
            if (own[q] >= 0) atomicAdd(&cnt[own[q]], 1);
        }
        __syncthreads();
        // every warp finds the tile's adapter by itself: lane l looks at adapters 32 i + l
        int a = -1, nth = 0, rows = 0;
        for (int a0 = 0, before = 0; a0 < p.n; a0 += 32) {
            const int c = a0 + lane < p.n ? cnt[a0 + lane] : 0, n = (c + TR - 1) / TR;
            int upto = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += v;
            }
            const int all = __shfl_sync(0xffffffffu, upto, 31);
            if (tile < before + all) {
                const int l = __ffs(__ballot_sync(0xffffffffu, tile < before + upto)) - 1;
                a = a0 + l;
                nth = (tile - before - __shfl_sync(0xffffffffu, upto - n, l)) * TR;
                rows = min(TR, __shfl_sync(0xffffffffu, c, l) - nth);
                break;
            }
            before += all;
        }
        // its rows: those of the adapter, in order, number nth and on
        if (a >= 0) {
            const int seg = (m + kWarps * 32 - 1) / (kWarps * 32) * 32, i0 = warp * seg;  // rows of a warp
            int c = 0;
            for (int i = i0; i < min(m, i0 + seg); i += 32) c += __popc(__ballot_sync(0xffffffffu, i + lane < m && ids[i + lane] == a));
            if (lane == 0) warp_s[warp] = c;
            __syncthreads();
            int r = -nth;
            for (int w = 0; w < warp; ++w) r += warp_s[w];
            for (int i = i0; i < min(m, i0 + seg); i += 32) {
                const bool is = i + lane < m && ids[i + lane] == a;
                const unsigned who = __ballot_sync(0xffffffffu, is);
                const int at = r + __popc(who & ((1u << lane) - 1u));
                if (is && at >= 0 && at < TR) rows_s[at] = i + lane;
                if (is && at == 0)
                    for (int q = rows; q < TR; ++q) rows_s[q] = i + lane;  // (columns beyond its rows: read, never written)
                r += __popc(who);
            }
        }
        if (tid == 0) {
            tile_s[0] = a;
            tile_s[1] = rows;
        }
        __syncthreads();
    }
    const int ad = tile_s[0], live = tile_s[1];
    if (ad < 0) return;  // (the whole cluster: nothing has been shared yet)

    // ---- shrink: partial h of this CTA's input features
    const int M = p.S * p.R, MP = pl.mt * 16;
    float* part = reinterpret_cast<float*>(smem);                              // [MP][TR]: the CTA's sum, of its first share at first
    __nv_bfloat16* hs = reinterpret_cast<__nv_bfloat16*>(part + MP * TR);      // [S][3][TR][h_stride]
    uint8_t* pool = reinterpret_cast<uint8_t*>(hs) + pl.h_bytes;               // the other shares, [ks - 1][MP][TR]; then the copies in flight
    float* more = reinterpret_cast<float*>(pool);
    const int blocks = (p.K + 31) / 32;
    const int c0 = (int)((int64_t)blocks * rank / kCluster), c1 = (int)((int64_t)blocks * (rank + 1) / kCluster);
    for (int u = warp; u < pl.mt * pl.ks; u += kWarps) {
        const int mt = u / pl.ks, ks = u % pl.ks;
        const int b0 = c0 + (c1 - c0) * ks / pl.ks, b1 = c0 + (c1 - c0) * (ks + 1) / pl.ks;
        const WT* A = static_cast<const WT*>(p.a) + (int64_t)ad * M * p.K;
        const WT *A0 = A + (int64_t)min(mt * 16 + g, M - 1) * p.K, *A1 = A + (int64_t)min(mt * 16 + g + 8, M - 1) * p.K;
        const XT *X[NT], *XL[NT];
#pragma unroll
        for (int q = 0; q < NT; ++q) {
            const int64_t o = (int64_t)rows_s[q * 8 + g] * p.ldx;
            X[q] = static_cast<const XT*>(p.x) + o;
            XL[q] = XK == kLoraXPair ? static_cast<const XT*>(p.x_lo) + o : nullptr;
        }
        float acc[NT][4] = {};
        constexpr int kUnroll = TR == 8 && OCC == 2 ? 4 : 2;
#pragma unroll kUnroll
        for (int b = b0; b < b1; ++b) {
            const bool ragged = b * 32 + 32 > p.K, in = b * 32 + 8 * t < p.K;  // (what is behind the features' end: zeros)
            const int at = min(b * 32 + 8 * t, p.K - 8);
            auto f0 = load_frag<WT, 8>(A0 + at), f1 = load_frag<WT, 8>(A1 + at);
            if (ragged) {
                f0.keep_if(in);
                f1.keep_if(in);
            }
#pragma unroll
            for (int q = 0; q < NT; ++q) {
                uint32_t xf[NX][4];
                auto v = load_frag<XT, 8>(X[q] + at);
                if (ragged) v.keep_if(in);
                if constexpr (XK == kLoraXPair) {
                    auto w = load_frag<XT, 8>(XL[q] + at);
                    if (ragged) w.keep_if(in);
#pragma unroll
                    for (int e = 0; e < 4; ++e) { xf[0][e] = v.t[0][e]; xf[1][e] = w.t[0][e]; }
                } else {
#pragma unroll
                    for (int i = 0; i < NX; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) xf[i][e] = v.t[i][e];
                }
                // (which input features a step takes is arbitrary: a lane's eight are the same in both operands.  The tensor
                // cores cut sums off instead of rounding them, so a chain of them stays short: 32 features, low terms first,
                // then a float32 addition.)
                float blk[4] = {};
#pragma unroll
                for (int i = NX - 1; i >= 0; --i)
#pragma unroll
                    for (int j = NW - 1; j >= 0; --j)
                        if (i + j < 3)
#pragma unroll
                            for (int st = 0; st < 2; ++st)
                                mma(blk, f0.t[j][2 * st], f1.t[j][2 * st], f0.t[j][2 * st + 1], f1.t[j][2 * st + 1],
                                    xf[i][2 * st], xf[i][2 * st + 1]);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[q][e] += blk[e];
            }
        }
        float* o = (ks ? more + (ks - 1) * MP * TR : part) + mt * 16 * TR;
#pragma unroll
        for (int q = 0; q < NT; ++q) {
            o[g * TR + q * 8 + 2 * t] = acc[q][0];
            o[g * TR + q * 8 + 2 * t + 1] = acc[q][1];
            o[(g + 8) * TR + q * 8 + 2 * t] = acc[q][2];
            o[(g + 8) * TR + q * 8 + 2 * t + 1] = acc[q][3];
        }
    }
    __syncthreads();
    if (pl.ks > 1) {
        for (int e = tid; e < MP * TR; e += kThreads) {
            float v = part[e];
            for (int q = 0; q + 1 < pl.ks; ++q) v += more[q * MP * TR + e];
            part[e] = v;
        }
        __syncthreads();
    }
    // ---- expand, set-up: a step = 32 output features of one segment and 16 rows of the tile; as the rows of B are dealt out to
    // the tensor cores' columns, a thread has eight consecutive features of the rows g and g + 8, so y moves 16 bytes at a
    // time.  Where y's rows are not aligned for that (`odd`; tiles of 8 rows only) it has the pairs 8j + 2t, so that a row's
    // four threads touch neighbours (half the time that eight apiece took).  The operands of a warp's next steps are copied to
    // shared memory (odd y partly to L2 only) in the background (each thread reads what it copied itself); the first ones are on
    // their way while the cluster meets.
    constexpr int HR = TR == 8 ? 1 : 2;  // 8-row halves of a 16-row tile that are used
    constexpr int D = steps_ahead(TR);   // steps in flight
    int steps = 0;                       // (of 32 features)
    for (int s = 0; s < p.S; ++s) steps += (p.seg[s + 1] - p.seg[s] + 31) / 32;
    const int per = (steps + pl.slices * kCluster - 1) / (pl.slices * kCluster);
    const int first = min(steps, (slice * kCluster + rank) * per), last = min(steps, first + per);
    // with a second 16-row tile in use every other warp has that one
    const bool two = live > 16;
    const bool odd = TR == 8 && !pl.y_vec;
    // odd y word by word, where there are registers for it (63 rows, 4096 -> 16793 in float32: 15.2 us, without 15.8; 77 rows of
    // 2040 -> 1000, which are aligned, pay for it: 10.6, without 9.9)
    constexpr bool kWords = TR == 8 && OCC == 2 && sizeof(YT) == 4;
    const int q = two ? warp & 1 : 0, stride = two ? kWarps / 2 : kWarps;
    const int mine = max(0, (last - first - (two ? warp >> 1 : warp) + stride - 1) / stride);  // this warp's steps
    struct Place {  // of a step: its features, the end of their segment, and the segment
        int f0, end, s;
    };
    auto ahead = [&](Place& at, int n) {  // n steps on
        while (at.s < p.S) {
            const int left = (at.end - at.f0 + 31) / 32;
            if (n < left) {
                at.f0 += 32 * n;
                return;
            }
            n -= left;
            if (++at.s < p.S) {
                at.f0 = at.end;
                at.end = p.seg[at.s + 1];
            }
        }
    };
    YT* y_row[HR];  // its rows
    bool has[HR];   // (a tile may have fewer: the row is its last one then, and is left alone)
#pragma unroll
    for (int h = 0; h < HR; ++h) {
        const int c = q * 16 + h * 8 + g, i = rows_s[c];
        has[h] = c < live;
        y_row[h] = static_cast<YT*>(p.y) + (int64_t)(p.scatter ? p.idx[i] : i) * p.ldy;
    }
    const int kbs = (p.R + 15) / 16;
    constexpr int YV = sizeof(YT) / 2;  // 16-byte words of eight elements
    struct Step {  // of one thread: y, and columns 0..15 of B (part j: features 2j, 2j+1 of every eight; odd: the j-th eight)
        uint4 y[HR * YV][32];
        typename std::conditional<sizeof(WT) == 2, uint2, uint4>::type w[4][32];
    };
    Step* const ring = reinterpret_cast<Step*>(pool) + warp * D;
    const WT* const B = static_cast<const WT*>(p.b) + (int64_t)ad * p.N * p.R;
    const int fw = odd ? g : (g >> 1) * 8 + (g & 1), fj = odd ? 8 : 2;  // this thread's row of B in part 0; from part to part
    const bool in0 = 4 * t < p.R;           // (a rank of 8 has no columns 8..15)
    const int c0w = min(4 * t, p.R - 4);
    auto w_row = [&](int f0, int j) { return B + (int64_t)min(f0 + fw + fj * j, p.N - 1) * p.R; };
    auto w_cols = [&](int f0, int j, int kb) {  // columns 16 kb + 4 t .. + 3 of part j's row; zeros behind the last
        auto f = load_frag<WT, 4>(w_row(f0, j) + min(kb * 16 + 4 * t, p.R - 4));
        if (kb * 16 + 16 > p.R) f.keep_if(kb * 16 + 4 * t < p.R);
        return f;
    };
    auto fetch = [&](const Place& at, Step& d) {
        if (pl.y_vec && at.f0 + 32 <= at.end) {
#pragma unroll
            for (int h = 0; h < HR; ++h)
#pragma unroll
                for (int v = 0; v < YV; ++v) copy_async<16>(&d.y[h * YV + v][lane], reinterpret_cast<const uint4*>(y_row[h] + at.f0 + 8 * t) + v, has[h]);
        }
        if constexpr (TR == 8) {
            if (odd) {
                if constexpr (kWords) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int f = at.f0 + 2 * t + (e >> 1) * 8 + (e & 1);
                        copy_word(&d.y[e >> 2][lane], e & 3, y_row[0] + min(f, at.end - 1), has[0] && f < at.end);
                    }
                } else {  // (the four threads' addresses are a quarter of the step apart)
                    prefetch_if(y_row[0] + at.f0 + 8 * t, has[0] && at.f0 + 8 * t < at.end);
                }
            }
        }
        if (at.f0 + 32 <= p.N) {
            const WT* w = B + (int64_t)(at.f0 + fw) * p.R + c0w;
#pragma unroll
            for (int j = 0; j < 4; ++j) copy_async<4 * sizeof(WT)>(&d.w[j][lane], w + fj * j * p.R, in0);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) copy_async<4 * sizeof(WT)>(&d.w[j][lane], w_row(at.f0, j) + c0w, in0);
        }
    };
    Place here{0, p.seg[1], 0}, next;
    if (mine > 0) ahead(here, first + (two ? warp >> 1 : warp));
    next = here;
#pragma unroll
    for (int d = 0; d < D; ++d) {
        if (d < mine) fetch(next, ring[d]);
        copy_commit();
        ahead(next, stride);
    }
    __syncwarp();
    cluster_arrive();
    cluster_wait();

    // ---- combine: h of the tile's rows, scaled, in three terms; columns up to the next multiple of 16 are zero
    const float sc = p.scales ? p.scales[ad] : 1.f;
    for (int e = tid; e < p.S * kbs * 16 * live; e += kThreads) {
        const int sj = e / live, col = e - sj * live, s = sj / (kbs * 16), j = sj - s * (kbs * 16);
        float v = 0.f;
        if (j < p.R) {
#pragma unroll
            for (int c = 0; c < kCluster; ++c) v += cluster.map_shared_rank(part, c)[(s * p.R + j) * TR + col];
            if (!(fabsf(v) < INFINITY)) {
                const WT* A = static_cast<const WT*>(p.a) + ((int64_t)ad * M + s * p.R + j) * p.K;
                const int64_t o = (int64_t)rows_s[col] * p.ldx;
                v = 0.f;
                for (int k = 0; k < p.K && v == v; k += 8)  // (a NaN stays one: rows full of them end at once)
#pragma unroll
                    for (int i = 0; i < 8; ++i) v = fmaf(to_f32(A[k + i]), x_at<XK>(p, o + k + i), v);
            }
        }
        uint16_t t3[3];
        split_one(v * sc, t3);
#pragma unroll
        for (int i = 0; i < 3; ++i) reinterpret_cast<uint16_t*>(hs)[((s * 3 + i) * TR + col) * pl.h_stride + j] = t3[i];
    }
    __syncthreads();
    cluster_arrive();  // (no CTA leaves before all have read its partial sums)

    // ---- expand
    for (int n = 0, at = 0; n < mine; ++n, at = at + 1 < D ? at + 1 : 0) {
        copy_wait<D - 1>();
        Step& cur = ring[at];
        const int f0 = here.f0, end = here.end;
        float acc[4][4] = {};
        const __nv_bfloat16* const h_tile = hs + (here.s * 3 * TR + q * 16 + g) * pl.h_stride + 4 * t;
        [[maybe_unused]] Frag<NW, 4> w_next[4];
        for (int kb = 0; kb < kbs; ++kb) {
            Frag<NW, 4> w[4];
            if constexpr (TR == 8 && OCC == 2) {  // (there are registers for the next columns: 9 rows, 4096 -> 4096 at rank 56 in float32: 14.7 us, without 15.9)
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = kb ? w_next[j] : shared_frag<WT>(&cur.w[j][lane]);
                if (kb + 1 < kbs)
#pragma unroll
                    for (int j = 0; j < 4; ++j) w_next[j] = w_cols(f0, j, kb + 1);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[j] = kb ? w_cols(f0, j, kb) : shared_frag<WT>(&cur.w[j][lane]);
            }
            float blk[4][4] = {};
#pragma unroll
            for (int k = 2; k >= 0; --k) {
                const __nv_bfloat16* hk = h_tile + k * TR * pl.h_stride + kb * 16;
                const uint2 h0 = *reinterpret_cast<const uint2*>(hk);
                const uint2 h1 = HR == 2 ? *reinterpret_cast<const uint2*>(hk + 8 * pl.h_stride) : make_uint2(0, 0);
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int i = NW - 1; i >= 0; --i)
                        if (k + i < 3) mma(blk[j], h0.x, h1.x, h0.y, h1.y, w[j].t[i][0], w[j].t[i][1]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][e] += blk[j][e];
        }
        // element e of row h is feature ft + (e >> 1) * fs + (e & 1), acc[e >> 1][2 h + (e & 1)]
        const int fs = TR == 8 && odd ? 8 : 2, ft = f0 + (TR == 8 && odd ? 2 : 8) * t;
        bool good[HR];  // a row that is not there, or a sum that is not finite: not stored here
#pragma unroll
        for (int h = 0; h < HR; ++h)
            good[h] = has[h] && largest(largest(largest(acc[0][2 * h], acc[0][2 * h + 1], acc[1][2 * h]), acc[1][2 * h + 1], acc[2][2 * h]),
                                        largest(acc[2][2 * h + 1], acc[3][2 * h], acc[3][2 * h + 1]), 0.f) < INFINITY;
        if (pl.y_vec && f0 + 32 <= end) {
#pragma unroll
            for (int h = 0; h < HR; ++h) {
                uint4 v[YV];
                if constexpr (sizeof(YT) == 4) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint4 o = cur.y[h * YV + i][lane];
                        v[i] = make_uint4(__float_as_uint(__uint_as_float(o.x) + acc[2 * i][2 * h]),
                                          __float_as_uint(__uint_as_float(o.y) + acc[2 * i][2 * h + 1]),
                                          __float_as_uint(__uint_as_float(o.z) + acc[2 * i + 1][2 * h]),
                                          __float_as_uint(__uint_as_float(o.w) + acc[2 * i + 1][2 * h + 1]));
                    }
                } else {
                    auto add = [&](uint32_t o, int j) {
                        const __nv_bfloat162 r = __floats2bfloat162_rn(bf_lo(o) + acc[j][2 * h], bf_hi(o) + acc[j][2 * h + 1]);
                        return *reinterpret_cast<const uint32_t*>(&r);
                    };
                    const uint4 o = cur.y[h][lane];
                    v[0] = make_uint4(add(o.x, 0), add(o.y, 1), add(o.z, 2), add(o.w, 3));
                }
#pragma unroll
                for (int i = 0; i < YV; ++i) store16_if(reinterpret_cast<uint4*>(y_row[h] + f0 + 8 * t) + i, v[i], good[h]);
            }
        } else {  // a segment's last features, or rows that are not aligned: one by one
#pragma unroll
            for (int h = 0; h < HR; ++h) {
                YT o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int f = ft + (e >> 1) * fs + (e & 1);
                    if (kWords && odd) o[e] = reinterpret_cast<const YT*>(&cur.y[(e >> 2) % (HR * YV)][lane])[e & 3];
                    else o[e] = load_if(y_row[h] + f, has[h] && f < end);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int f = ft + (e >> 1) * fs + (e & 1);
                    store_if(y_row[h] + f, from_f32<YT>(to_f32(o[e]) + acc[e >> 1][2 * h + (e & 1)]), good[h] && f < end);
                }
            }
        }
        if (n + D < mine) fetch(next, cur);
        copy_commit();
        bool again = has[0] && !good[0];
        if constexpr (HR == 2) again = again || (has[1] && !good[1]);
        if (__any_sync(0xffffffffu, again)) {  // (seldom: sums that are not finite, with h put together from its terms)
#pragma unroll 1
            for (int at_e = 0; at_e < 8 * HR; ++at_e) {
                float v = 0.f;
#pragma unroll
                for (int e = 0; e < 8 * HR; ++e) v = e == at_e ? acc[(e & 7) >> 1][2 * (e >> 3) + (e & 1)] : v;
                const int h = at_e >> 3, f = ft + ((at_e & 7) >> 1) * fs + (at_e & 1);
                if ((HR == 2 && h ? has[HR - 1] && !good[HR - 1] : has[0] && !good[0]) && f < end) {
                    if (!(fabsf(v) < INFINITY)) {
                        const __nv_bfloat16* hc = hs + (here.s * 3 * TR + q * 16 + h * 8 + g) * pl.h_stride;
                        v = 0.f;
                        for (int j0 = 0; j0 < p.R && v == v; j0 += 8)
#pragma unroll
                            for (int j = j0; j < j0 + 8; ++j) {
                                const float h0 = __bfloat162float(hc[j]), h1 = __bfloat162float(hc[TR * pl.h_stride + j]), h2 = __bfloat162float(hc[2 * TR * pl.h_stride + j]);
                                v = fmaf(to_f32(B[(int64_t)f * p.R + j]), h0 + (h1 + h2), v);
                            }
                    }
                    YT* const o = (HR == 2 && h ? y_row[HR - 1] : y_row[0]) + f;
                    *o = from_f32<YT>(to_f32(*o) + v);
                }
            }
            __syncwarp();
        }
        ahead(here, stride);
        ahead(next, stride);
    }
    copy_wait<0>();
    __syncwarp();
    cluster_wait();
}

constexpr size_t kMaxSmem = 226 * 1024;  // dynamic bytes of a CTA; the static ones (under 1 KB) come on top

// Launch shape of `rows`-row tiles; the shared memory it takes (see the kernel for the parts).
Plan plan_of(const LoraArgs& a, int rows, int tiles, int n_sm, size_t& smem) {
    Plan pl{};
    const int M = a.S * a.R, kbs = (a.R + 15) / 16, wt = a.w_f32 ? 4 : 2, yt = a.y_f32 ? 4 : 2;
    pl.direct = a.n > kMaxIds || a.m == 1;
    pl.tiles = tiles;
    // few tiles: several clusters share one's output features, while there is room for them and a step for each warp
    pl.slices = std::max(1, std::min(2 * n_sm / (tiles * kCluster), a.N / (32 * kCluster * kWarps)));
    pl.mt = (M + 15) / 16;
    pl.ks = std::max(1, kParts / pl.mt);
    pl.h_stride = 16 * (kbs | 1);  // an odd number of 32-byte units: eight batch rows' fragments meet no bank twice
    pl.y_vec = reinterpret_cast<uintptr_t>(a.y) % 16 == 0 && (a.m == 1 || a.ldy * yt % 16 == 0);
    pl.h_bytes = a.S * 3 * rows * pl.h_stride * 2;
    const size_t step = (rows == 8 ? 1 : 2) * yt / 2 * 512 + 4 * 32 * 4 * wt, shares = (size_t)(pl.ks - 1) * pl.mt * 16 * rows * 4;
    smem = (size_t)pl.mt * 16 * rows * 4 + pl.h_bytes + std::max(shares, kWarps * steps_ahead(rows) * step);
    if (!pl.direct) smem = std::max(smem, ((size_t)(a.n + 3) / 4 * 4 + a.m) * 4);
    return pl;
}

template <int XK, typename WT, typename YT, int TR, int OCC>
cudaError_t launch_tiles(const LoraArgs& a, const Plan& pl, size_t smem, cudaStream_t st, bool pdl) {
    auto kern = lora_tiles<XK, WT, YT, TR, OCC>;
    if (smem > 40 * 1024) {  // (always the same value: calls of other threads rely on it)
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMaxSmem);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(pl.tiles * pl.slices * kCluster);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = kCluster;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, a, pl);
}

template <int XK, typename WT, typename YT>
cudaError_t launch_rows(const LoraArgs& a, cudaStream_t st, bool pdl, int n_sm) {
    // At most as many tiles as: one for every row, or one ragged tile for every adapter and full ones for the rest.
    auto tiles_of = [&](int rows) { return a.n > kMaxIds || a.m == 1 ? a.m : (int)std::min<int64_t>(a.m, (int64_t)a.n + a.m / rows); };
    size_t smem;
    // Tiles of 32 rows once an adapter has 16 rows on average (1024 rows of 8 adapters, gate|up: 46.7 us against 83.5 with
    // tiles of 8) and they fill the GPU (362 rows of 8 adapters, 4096 -> 6144, 152 CTAs: 15.5 us against 13.6 with tiles of 8), if
    // their h fits (four segments of rank 128 do not) and y is aligned; else of 8.  Adapters are counted as they are resident: how
    // many of them the rows use is known on the device only.  (x in two halves comes from the step, whose batches and prompt
    // chunks have too few rows for them.)
    if constexpr (XK != kLoraXPair)
        if (a.m >= 16 * (int64_t)a.n && a.m > 32 && 2 * tiles_of(32) * kCluster > 3 * n_sm) {
            const Plan pl = plan_of(a, 32, tiles_of(32), n_sm, smem);
            if (smem <= kMaxSmem && pl.y_vec) return launch_tiles<XK, WT, YT, 32, 2>(a, pl, smem, st, pdl);
        }
    const int tiles = tiles_of(8);
    const Plan pl = plan_of(a, 8, tiles, n_sm, smem);
    // With 64 registers four CTAs fit on a multiprocessor instead of two, at the price of spills: 256 rows of 64 adapters
    // (768 CTAs) 33.7 us against 36.9 with two, 32 rows of 16 adapters (160 CTAs) 11.7 against 10.2.  float32 adapters take
    // three times the registers and stay at two.
    if constexpr (sizeof(WT) == 2)
        if (tiles * kCluster > 2 * n_sm) return launch_tiles<XK, WT, YT, 8, 4>(a, pl, smem, st, pdl);
    return launch_tiles<XK, WT, YT, 8, 2>(a, pl, smem, st, pdl);
}

template <typename WT, typename YT>
cudaError_t launch_x(const LoraArgs& a, cudaStream_t st, bool pdl, int n_sm) {
    switch (a.x_kind) {
        case kLoraXF32: return launch_rows<kLoraXF32, WT, YT>(a, st, pdl, n_sm);
        case kLoraXBf16: return launch_rows<kLoraXBf16, WT, YT>(a, st, pdl, n_sm);
        default: return launch_rows<kLoraXPair, WT, YT>(a, st, pdl, n_sm);
    }
}

}  // namespace

cudaError_t lora_launch(const LoraArgs& args, cudaStream_t st, bool pdl, int n_sm) {
    LoraArgs a = args;
    for (int64_t r0 = 0; r0 < args.m; r0 += kMaxRows) {
        a.m = (int)std::min<int64_t>(kMaxRows, args.m - r0);
        const size_t xe = args.x_kind == kLoraXF32 ? 4 : 2, ye = args.y_f32 ? 4 : 2;
        a.x = static_cast<const char*>(args.x) + (size_t)r0 * args.ldx * xe;
        a.x_lo = args.x_lo ? static_cast<const char*>(args.x_lo) + (size_t)r0 * args.ldx * xe : nullptr;
        if (args.idx) a.idx = args.idx + r0;
        else a.adapter = args.adapter + r0;
        if (!args.scatter) a.y = static_cast<char*>(args.y) + (size_t)r0 * args.ldy * ye;
        a.row0 = (int)r0;
        const cudaError_t e =
            a.w_f32 ? (a.y_f32 ? launch_x<float, float>(a, st, pdl, n_sm) : launch_x<float, __nv_bfloat16>(a, st, pdl, n_sm))
                    : (a.y_f32 ? launch_x<__nv_bfloat16, float>(a, st, pdl, n_sm) : launch_x<__nv_bfloat16, __nv_bfloat16>(a, st, pdl, n_sm));
        if (e != cudaSuccess) return e;
        pdl = false;
    }
    return cudaSuccess;
}

}  // namespace first

using namespace first;

extern "C" int first_lora(const void* x, int32_t x_dtype, int64_t x_stride, const void* a, const void* b,
                          int32_t w_dtype, const float* scales, const int32_t* row_adapter, int32_t n_adapters,
                          int32_t rank, int32_t n_segments, const int32_t* segments, int32_t rows, int32_t k, int32_t n,
                          void* y, int32_t y_dtype, int64_t y_stride, void* stream) {
    if (rows < 0 || n_adapters < 0 || k <= 0 || n <= 0 || rank <= 0 || n_segments <= 0) return FIRST_E_ARG;
    if (rows == 0 || n_adapters == 0) return FIRST_OK;
    if (!x || !a || !b || !row_adapter || !y || !segments) return FIRST_E_ARG;
    for (int32_t dt : {x_dtype, w_dtype, y_dtype})
        if (dt != FIRST_DTYPE_F32 && dt != FIRST_DTYPE_BF16) return FIRST_E_ARG;
    if (k > kMaxSize || n > kMaxSize) return FIRST_E_UNSUPPORTED;
    if (n_segments > FIRST_LORA_MAX_SEGMENTS || rank > FIRST_LORA_MAX_RANK || rank % 8 || k % 8) return FIRST_E_UNSUPPORTED;
    if (segments[0] != 0 || segments[n_segments] != n) return FIRST_E_SHAPE;
    for (int i = 0; i < n_segments; ++i) {
        if (segments[i + 1] <= segments[i]) return FIRST_E_SHAPE;
        if (segments[i] % 16) return FIRST_E_UNSUPPORTED;
    }
    if (rows > 1 && (x_stride < k || y_stride < n)) return FIRST_E_SHAPE;
    const int xe = x_dtype == FIRST_DTYPE_F32 ? 4 : 2;
    if (rows > 1 && (x_stride * xe) % 16) return FIRST_E_UNSUPPORTED;
    if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) % 16)
        return FIRST_E_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(y) % (y_dtype == FIRST_DTYPE_F32 ? 4 : 2)) return FIRST_E_UNSUPPORTED;
    LoraArgs p;
    p.x = x;
    p.x_kind = x_dtype == FIRST_DTYPE_F32 ? kLoraXF32 : kLoraXBf16;
    p.ldx = x_stride;
    p.a = a; p.b = b;
    p.w_f32 = w_dtype == FIRST_DTYPE_F32;
    p.scales = scales;
    p.adapter = row_adapter;
    p.n = n_adapters; p.S = n_segments; p.R = rank; p.K = k; p.N = n;
    for (int i = 0; i <= n_segments; ++i) p.seg[i] = segments[i];
    p.y = y; p.y_f32 = y_dtype == FIRST_DTYPE_F32; p.ldy = y_stride;
    p.m = rows;
    return lora_launch(p, static_cast<cudaStream_t>(stream), false, kSMs) == cudaSuccess ? FIRST_OK : FIRST_E_CUDA;
}
