// Attention of a sequence's newest tokens over a paged 8-bit cache.
#include <algorithm>

#include <cuda.h>

#include "cache8.cuh"

using namespace first;

namespace {

constexpr int kMaxCluster = 8, kMaxSorted = 256, kMaxSplits = 64;
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
// Products with 8-bit integer rows as they are: [16 rows][32] x [32][8 columns].  The sums here stay below 2^22: an
// accumulator that starts at kIntZero is, as a float32, 1.5 2^23 + the sum.
constexpr uint32_t kIntZero = 0x4b400000u;
__device__ __forceinline__ void mma_int(uint32_t (&d)[4], const uint32_t (&a)[4], uint2 b) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y));
}
// Four E4M3 numbers as halves, in order.
__device__ __forceinline__ void e4m3_halves(uint32_t w, uint32_t& a, uint32_t& b) {
    asm("{.reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}" : "=r"(a), "=r"(b) : "r"(w));
}
// Four 8-bit values as halves, in order.  Integers: 0x64 above a byte is 1024 + byte.
template <bool E4M3>
__device__ __forceinline__ void k_halves(uint32_t w, uint32_t& a, uint32_t& b) {
    if constexpr (E4M3) {
        e4m3_halves(w, a, b);
    } else {
        const __half2 bias = __half2half2(__ushort_as_half(0x6480));  // 1152
        w ^= 0x80808080u;
        uint32_t x = __byte_perm(w, 0x64646464u, 0x4140), y = __byte_perm(w, 0x64646464u, 0x4342);
        const __half2 p = __hsub2(*reinterpret_cast<__half2*>(&x), bias), q = __hsub2(*reinterpret_cast<__half2*>(&y), bias);
        a = *reinterpret_cast<const uint32_t*>(&p);
        b = *reinterpret_cast<const uint32_t*>(&q);
    }
}
// Four 8 x 16-byte blocks of shared memory, a row's address a lane (lanes 8 i .. 8 i + 7: block i), whole or with rows and
// 16-bit columns exchanged.
__device__ __forceinline__ void blocks(uint32_t at, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void blocks_turned(uint32_t at, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void bar_init(uint32_t bar) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Bounded: false after kPolls tries.
constexpr uint32_t kPolls = 1u << 22;
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
    for (uint32_t i = 0; i < kPolls; ++i) {
        uint32_t ok;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
    }
    return false;
}
__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap* map, uint32_t bar, int row) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(0), "r"(row) : "memory");
}
// A float into element `i` of an array in the shared memory of the cluster's CTA `k`.
__device__ __forceinline__ void remote_store(uint32_t array, int k, int i, float v) {
    asm volatile("{\n .reg .u32 a;\n mapa.shared::cluster.u32 a, %0, %1;\n st.shared::cluster.f32 [a], %2;\n}"
                 ::"r"(array + 4 * i), "r"(k), "f"(v) : "memory");
}
// Where 16-byte piece `x` of row `row` of a copied box lies: the copy swizzles a row's pieces by the row, so that eight rows'
// equal pieces are in different banks.
template <int HD>
__device__ __forceinline__ uint32_t in_box(int row, int x) {
    const int turn = HD == 128 ? row & 7 : HD == 64 ? row >> 1 & 3 : row >> 2 & 1;
    return row * HD + ((x ^ turn) << 4);
}
// Bytes (token, d), (token, d + 1), (token + 1, d), (token + 1, d + 1) -> halves of the two tokens, at d and at d + 1.  Exact:
// 0x64 above a byte is 1024 + byte.
template <bool E4M3>
__device__ __forceinline__ void v_halves(uint32_t w, uint32_t& a, uint32_t& b) {
    if constexpr (E4M3) {
        e4m3_halves(__byte_perm(w, 0, 0x3120), a, b);
    } else {
        const __half2 bias = __half2half2(__ushort_as_half(0x6480));  // 1152
        uint32_t x = (w & 0x00ff00ffu) ^ 0x64806480u, y = (w >> 8 & 0x00ff00ffu) ^ 0x64806480u;
        const __half2 p = __hsub2(*reinterpret_cast<__half2*>(&x), bias), q = __hsub2(*reinterpret_cast<__half2*>(&y), bias);
        a = *reinterpret_cast<const uint32_t*>(&p);
        b = *reinterpret_cast<const uint32_t*>(&q);
    }
}

// Element d of the result for a row of the caller's.
__device__ __forceinline__ void put(const Attn8Args& p, int64_t row, int head, int d, float v) {
    const int64_t to = row * p.out.tok + head * p.out.head + d;
    if (p.out.p) {
        if (p.out.f32) static_cast<float*>(p.out.p)[to] = v;
        else static_cast<__nv_bfloat16*>(p.out.p)[to] = __float2bfloat16_rn(v);
    } else {
        const __nv_bfloat16 hi = __float2bfloat16_rn(v);
        p.out_hi[to] = hi;
        p.out_lo[to] = __float2bfloat16_rn(v - __bfloat162float(hi));
    }
}
// Where a row's unfinished results are kept, in rows.
__device__ __forceinline__ int64_t part_of(int b, int h, int r, int rows, int H) { return ((int64_t)b * H + h) * rows + r; }

template <int NT>
constexpr int kGroups = NT <= 3 ? 2 : 1;  // groups of 16 tokens a step
template <int NT>
constexpr int kRing = 4 / kGroups<NT>;    // steps that a warp has room for: one in use, the others on their way
template <int HD, int NT>
constexpr int kStepBytes = 2 * 16 * kGroups<NT> * HD;

// How K is multiplied.  Integers with one query row a column pair (PER 1): as they are, a query element in 4 parts of 8 bits, base 256, a
// multiple of some 2^-30 of its row's largest.  (Two parts were enough for bfloat16's 8 bits only where all elements are of one size:
// beside a channel of 64 times the others the result was 2e-3 off, of 1024 times 4e-2.)  Otherwise as halves (exactly): E4M3 has no products of its
// own on this path, and integers with a query row a column take half as many products so (32 sequences x 8 drafts of 4 heads: in parts 164 us, as
// halves 127).  A query row is scaled by a power of two into their range and takes one (bfloat16's 8 bits fit, down to 2^-30 of the
// row's largest) or, PER 1, two (hi + lo).
template <bool E4M3, int PER>
constexpr bool kHalves = E4M3 || PER == 2;
constexpr int kParts = 4;

// A cluster takes a tile of query rows (tokens x query heads of a KV head) of one sequence; its CTAs and their warps take
// its tokens in turns and join (maximum, sum, output) at the end, over shared memory and then over the cluster's.  The
// tensor cores see tokens as rows: S[16 tokens][8 columns] = K q, O[16 of hd][8 columns] += V' P.
// S: by integers as they are a query row takes a column a part (above), added up in float32; by halves a column, or two.
// O: V in halves (exactly), P = hi + lo in halves: two columns a query row (PER 1), or one column and a second product (PER 2, where rows are many).
// (One half, 11 bits, was 2^-12 of the largest value off, visible in bfloat16 where values cancel; the second products cost 16 x 6 drafts 57 -> 63 us, launched alone.)
// K's page scales act on the float32 products, V's on the weights, relative to the largest that the warp has met (a page far below it, 2^-12, is added
// apart, so that its weights are not subnormal halves).
// Every warp copies its own tokens (TMA, a step ahead) and waits for nobody else until the end.
// Longer sequences come first, so that the last CTAs are short ones.
// 8 KV heads of 128, 4 query heads each: 32 sequences (277 MB, integers) 55 us, 5.0 TB/s; 128 (1220 MB, float32 queries) 216 to 233 us on several cards, 5.2 to
// 5.65 TB/s: the cache's bytes, and the start and join of each item.  16 sequences x 6 drafts (105 MB, E4M3) 59.5 us: conversions, the softmax of 24
// columns and two products with V, at 8 warps an SM.
template <int HD, int NT, int PER, bool F32, bool E4M3, int kWarps>
__global__ void __launch_bounds__(32 * kWarps, (NT == 1 ? (kWarps == 8 ? 16 : 12) : 8) / kWarps)
    attn8(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const Attn8Args p, const int S,
          const int Z) {
    constexpr int kThreads = 32 * kWarps;
    constexpr int kRows = NT * 4 * PER, kSteps = HD / 16, kLong = HD / 32;  // steps of 16 (halves) and of 32 (8 bits) along hd
    constexpr int P = kParts;
    constexpr bool kHalfK = kHalves<E4M3, PER>;
    constexpr int kTiles = kHalfK ? 1 : P / 2;  // S columns' tiles for a tile of O's: integers take two parts of four rows each
    constexpr int U = kGroups<NT>, kStages = kRing<NT>;
    constexpr int kStride = HD + 16;     // of O in shared memory
    constexpr bool kHeld = NT * kTiles * (kHalfK ? 2 : 1) <= 3;  // the queries' fragments fit into registers
    extern __shared__ __align__(16) uint8_t s_dynamic[];  // [warps][kStages][K | V of a step]; at the end [warps][rows][kStride] float32
    __shared__ uint64_t s_bar[kWarps][kStages];
    constexpr int kFrag = NT * kTiles * (kHalfK ? kSteps : kLong);  // fragments of the queries
    // The queries' parts, and, once this CTA has made fragments of them, what the cluster writes.
    using Parts = uint8_t[kRows][kHalfK ? 2 / PER : P][kHalfK ? 2 * HD + 16 : HD + 16];
    using Got = float[kRows * HD + kMaxCluster];
    __shared__ __align__(16) uint8_t s_both[sizeof(Parts) > sizeof(Got) ? sizeof(Parts) : sizeof(Got)];
    Parts& s_q = *reinterpret_cast<Parts*>(s_both);
    Got& s_got = *reinterpret_cast<Got*>(s_both);
    __shared__ __align__(16) uint2 s_frag[kHeld ? 1 : kFrag * 32];
    __shared__ float s_gm[kMaxCluster][kRows], s_gl[kMaxCluster][kRows];  // written by the cluster
    __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows], s_f[kMaxCluster > kWarps ? kMaxCluster : kWarps][kRows];
    __shared__ float s_rs[kRows], s_inv[kRows];
    __shared__ int s_len[kMaxSorted], s_mine;
    const Stamp stamp_guard(p.s.stamp);
    const int tid = threadIdx.x, lane = tid & 31, g = lane >> 2, c = lane & 3;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);  // (so that the compiler knows it, and what hangs on it, as the warp's)
    const int rank = blockIdx.x % S, z_of = blockIdx.x / S % Z, h = blockIdx.x / (S * Z);  // a sequence and head has Z clusters
    const uint32_t aligned = ((uint32_t)__cvta_generic_to_shared(s_dynamic) + 1023u) & ~1023u;
    float* const s_part = reinterpret_cast<float*>(s_dynamic + (aligned - (uint32_t)__cvta_generic_to_shared(s_dynamic)));
    const uint32_t ring = aligned + warp * kStages * kStepBytes<HD, NT>, bars = (uint32_t)__cvta_generic_to_shared(s_bar[warp]);
    if (lane == 0) {
        if (warp == 0) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
        }
#pragma unroll
        for (int i = 0; i < kStages; ++i) bar_init(bars + 8 * i);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    pdl_trigger();
    pdl_wait();
    // ---- which sequence: the blockIdx.y-th longest
    const int live = p.s.m_dev ? min(__ldg(p.s.m_dev), (int)gridDim.y) : gridDim.y;
    if ((int)blockIdx.y >= live) return;
    int mine = blockIdx.y;
    if (live > 1 && gridDim.y <= kMaxSorted) {
        for (int i = tid; i < live; i += kThreads) s_len[i] = p.s.len[p.s.idx ? p.s.idx[i] : i];
        __syncthreads();
        for (int i = tid; i < live; i += kThreads) {
            const int n = s_len[i];
            int before = 0;
            for (int j = 0; j < live; ++j) before += s_len[j] > n || (s_len[j] == n && j < i);
            if (before == mine) s_mine = i;
        }
        __syncthreads();
        mine = s_mine;
    }
    // Step i of a warp covers groups ((i * Z*S + its CTA's) * kWarps + warp) * U ..: in turns over the CTAs' warps, whatever
    // the length.  Their pages and scales are looked up for kBatch steps at a time, one group a lane.
    constexpr int kBatch = 32 / U;
    auto group_of = [&](int i) { return ((i * Z * S + z_of * S + rank) * kWarps + warp) * U; };
    int page0 = raw_page(p.s, p.s.idx ? p.s.idx[mine] : mine, (group_of(lane / U) + lane % U) >> (p.c.shift - 4));  // (needs no length)
    Seq8 q;
    if (!find_seq(p.s, mine, q)) return;  // (the whole cluster)
    const int r0 = blockIdx.z * kRows, rows = min(kRows, q.n * p.G - r0);
    if (rows <= 0) return;
    const int64_t cap = p.s.width << p.c.shift;
    const int tok0 = r0 / p.G;
    const int first_lim = (int)min((int64_t)q.before + tok0 + 1, cap);
    const int end = (int)min((int64_t)q.before + (r0 + rows - 1) / p.G + 1, cap);  // tokens that any row sees
    const int t1 = (end + 15) / 16;

    // ---- the first tokens' values are on their way while the queries are prepared
    const int steps = t1 > group_of(0) ? (t1 - group_of(0) + Z * S * kWarps * U - 1) / (Z * S * kWarps * U) : 0;
    struct Groups {
        int page;
        float ks, vs;
    };
    auto page_of = [&](int i) {
        const int t = group_of(i + lane / U) + lane % U;
        return t < t1 ? raw_page(p.s, q.seq, t >> (p.c.shift - 4)) : -1;
    };
    auto look_up = [&](int page) {
        Groups x{check_page(p.s, p.c.n_pages, page), 0.f, 0.f};
        if (x.page >= 0) {
            x.ks = p.c.ks[(int64_t)x.page * p.c.H + h];
            x.vs = p.c.vs[(int64_t)x.page * p.c.H + h];
        }
        return x;
    };
    auto fetch = [&](int i, int page_here) {  // step i's values, a group a lane (nothing where it has no page)
        const int pg = __shfl_sync(0xffffffffu, page_here, (i % kBatch) * U + lane % U);
        const uint32_t some = __ballot_sync(0xffffffffu, pg >= 0) & ((1u << U) - 1u), bar = bars + 8 * (i % kStages);
        if (lane == 0) bar_expect(bar, __popc(some) * 2 * 16 * HD);
        __syncwarp();
        if (some >> lane & 1u) {
            const int row = ((pg * p.c.H + h) << p.c.shift) + (((group_of(i) + lane) * 16) & ((1 << p.c.shift) - 1));
            const uint32_t to = ring + (i % kStages) * kStepBytes<HD, NT> + lane * 16 * HD;
            tma_rows(to, &map_k, bar, row);
            tma_rows(to + U * 16 * HD, &map_v, bar, row);
        }
    };
    Groups ahead{-1, 0.f, 0.f}, here{-1, 0.f, 0.f};  // of the batch that is being fetched, and of the one in use
    int next_page = -1;
    if (group_of(lane / U) + lane % U >= t1) page0 = -1;
    if (steps > 0) here = ahead = look_up(page0);
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i)
        if (i < steps) fetch(i, here.page);
    // V's scales relative to the largest that the warp has met; -> what O has to be scaled by
    float v_top = 0.f;
    bool apart = false;  // V's scale of one of the batch's groups is far below the largest
    auto settle = [&]() {
        const float top = fmaxf(v_top, warp_max(fabsf(here.vs)));
        here.vs = top > 0.f ? here.vs / top : here.vs;
        apart = __any_sync(0xffffffffu, fabsf(here.vs) < 0x1p-12f && here.vs != 0.f);
        const float f = top > 0.f ? v_top / top : 1.f;
        v_top = top;
        return f;
    };

    // ---- query rows in parts
    for (int r = warp; r < kRows; r += kWarps) {
        float f[HD / 32];
        uint32_t amax = 0;
        bool odd = false;
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) f[i] = 0.f;
        if (r < rows) {
            const int tok = (r0 + r) / p.G, head = h * p.G + (r0 + r) % p.G;
            const int64_t from = (q.start + tok) * p.q.tok + head * p.q.head;
            auto get = [&](int d) {
                if constexpr (F32) return static_cast<const float*>(p.q.p)[from + d];
                else return to_f32(static_cast<const __nv_bfloat16*>(p.q.p)[from + d]);
            };
#pragma unroll
            for (int i = 0; i < HD / 32; ++i) f[i] = get(i * 32 + lane);
            if (p.s.cs) {
                constexpr int half = HD / 2;
#pragma unroll
                for (int i = 0; i < HD / 32; ++i) {
                    const int d = i * 32 + lane;
                    const bool up = d >= half;
                    const float2 t = p.s.cs[(int64_t)q.seq * half + (up ? d - half : d)];
                    const float o = get(up ? d - half : d + half);
                    f[i] = up ? f[i] * t.x + o * t.y : f[i] * t.x - o * t.y;
                }
            }
#pragma unroll
            for (int i = 0; i < HD / 32; ++i) {
                const uint32_t m = __float_as_uint(f[i]) & 0x7fffffffu;
                odd |= m >= 0x7f800000u;
                amax = max(amax, m < 0x7f800000u ? m : 0u);
            }
        }
        amax = __reduce_max_sync(0xffffffffu, amax);
        odd = __any_sync(0xffffffffu, odd);  // (no number among the parts stands for infinities and NaN: the row is NaN)
        // the row's largest magnitude goes to [2^kTop, 2^(kTop+1)); 2^126 times at most, and the inverse is a float32 too
        constexpr int kTop = kHalfK ? 13 : 8 * P - 3;
        const int e = max(min(127 + kTop - (int)(amax >> 23), 126), -126);
        const float up = __int_as_float((e + 127) << 23);
        if (lane == 0) s_rs[r] = odd ? __int_as_float(0x7fc00000) : __int_as_float((127 - e) << 23) * (kHalfK ? 1.f : (float)(1 << 8 * (P - 1)));
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) {
            const float x = f[i] * up;
            if constexpr (kHalfK) {
                const __half hi = __float2half_rn(x);
                reinterpret_cast<__half*>(s_q[r][0])[i * 32 + lane] = hi;
                if constexpr (PER == 1) reinterpret_cast<__half*>(s_q[r][1])[i * 32 + lane] = __float2half_rn(x - __half2float(hi));
            } else {
                int n = odd ? 0 : __float2int_rn(x);  // |n| <= 2^(8 P - 2): its digits, -128 .. 127 each, fit
#pragma unroll
                for (int k = P - 1; k >= 0; --k) {
                    const int digit = k ? (int)(int8_t)(n & 255) : n;
                    s_q[r][k][i * 32 + lane] = (uint8_t)digit;
                    n = (n - digit) >> 8;
                }
            }
        }
    }
    __syncthreads();
    // Fragment of tile n's (k-th) tile of columns, step s.  In parts: column g is row (n, g/2), part 2k + g%2.
    // Halves: column g is row (n, g) or, PER 1, half g%2 of row (n, g/2).
    auto query = [&](int n, int k, int s) {
        const uint8_t* x;
        if constexpr (kHalfK) {
            x = &s_q[n * 4 * PER + (PER == 1 ? g >> 1 : g)][PER == 1 ? g & 1 : 0][(s * 16 + 4 * c) * 2];
            return *reinterpret_cast<const uint2*>(x);
        } else {
            x = &s_q[n * 4 + (g >> 1)][2 * k + (g & 1)][s * 32 + 4 * c];
            return make_uint2(*reinterpret_cast<const uint32_t*>(x), *reinterpret_cast<const uint32_t*>(x + 16));
        }
    };
    constexpr int kQSteps = kHalfK ? kSteps : kLong;
    uint2 qf[kHeld ? kFrag : 1];
    if constexpr (kHeld) {
#pragma unroll
        for (int i = 0; i < kFrag; ++i) qf[i] = query(i / (kTiles * kQSteps), i / kQSteps % kTiles, i % kQSteps);
    } else {
        for (int i = warp; i < kFrag; i += kWarps) s_frag[i * 32 + lane] = query(i / (kTiles * kQSteps), i / kQSteps % kTiles, i % kQSteps);
        __syncthreads();
    }
    if (S > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");  // (waited for before the first remote store)
    auto fragment = [&](int i) {
        if constexpr (kHeld) return qf[i];
        else return s_frag[i * 32 + lane];
    };
    float rs[NT][PER];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < PER; ++j) rs[n][j] = s_rs[n * 4 * PER + PER * c + j] * p.scale * 1.44269504088896341f;

    float o[NT][kSteps][4];
    float m[NT][PER], l[NT][PER], base[NT][PER];  // base: kLift - m, huge as long as there is no maximum
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][s][e] = 0.f;
#pragma unroll
        for (int j = 0; j < PER; ++j) { m[n][j] = -INFINITY; l[n][j] = 0.f; base[n][j] = 3e38f; }
    }
    auto scale_o = [&](int n, int j, float f) {
#pragma unroll
        for (int w = 0; w < kSteps; ++w) {
            if constexpr (PER == 1) {
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][w][e] *= f;
            } else {
                o[n][w][j] *= f;
                o[n][w][2 + j] *= f;
            }
        }
    };
    // The lane's row address of four blocks, two 16-byte pieces of 16 tokens: (tokens 0 .. 7 | 8 ..) x (piece 2s | 2s + 1).
    uint32_t k_off[kLong];
#pragma unroll
    for (int s = 0; s < kLong; ++s) k_off[s] = in_box<HD>((lane & 7) + (lane & 8), 2 * s + (lane >> 4));
    for (int i = 0; i < steps; ++i) {
        const int tb = group_of(i) * 16;  // the step's first token
        if (i % kBatch == 0) {
            if (i > 0) here = ahead;
            const float f = settle();
            if (i > 0 && f != 1.f) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < PER; ++j) scale_o(n, j, f);
            }
        }
        // pages and scales of the next batch, well ahead
        if (i % kBatch == kBatch / 4 && i - i % kBatch + kBatch < steps) next_page = page_of(i - i % kBatch + kBatch);
        if (i % kBatch == kBatch / 2 && i - i % kBatch + kBatch < steps) ahead = look_up(next_page);
        const int coming = i + kStages - 1;
        if (coming < steps) fetch(coming, coming / kBatch == i / kBatch ? here.page : ahead.page);
        float ks[U], vr[U];
        bool special = tb + 16 * U > first_lim;  // some row does not see all of the step's tokens
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int from = (i % kBatch) * U + u;
            ks[u] = __shfl_sync(0xffffffffu, here.ks, from);
            vr[u] = __shfl_sync(0xffffffffu, here.vs, from);
        }
        const uint32_t have = __ballot_sync(0xffffffffu, here.page >= 0) >> ((i % kBatch) * U) & ((1u << U) - 1u);
        special |= have != (1u << U) - 1u;
        if (!__all_sync(0xffffffffu, bar_wait(bars + 8 * (i % kStages), (i / kStages) & 1))) {  // (gave up: the result is undefined)
            if (p.s.flags && lane == 0) atomicOr(p.s.flags, FIRST_FLAG_WAIT_EXPIRED);
            for (int k = i + 1; k < i + kStages && k < steps; ++k) bar_wait(bars + 8 * (k % kStages), (k / kStages) & 1);  // (its other copies)
            break;
        }
        const uint32_t k_in = ring + (i % kStages) * kStepBytes<HD, NT>, v_in = k_in + U * 16 * HD;
        // ---- S = K q, the groups' products in turns
        float z[U][NT][PER][2];  // [..][token of row g, of row g + 8]
        uint32_t a[U][kLong][4];
#pragma unroll
        for (int s = 0; s < kLong; ++s)
#pragma unroll
            for (int u = 0; u < U; ++u) blocks(k_in + u * 16 * HD + k_off[s], a[u][s]);
        constexpr int kAhead = NT == 1 ? kSteps / 2 : 0;  // V's first blocks are read before they are needed
        uint32_t v0[kAhead ? kAhead : 1][4];
#pragma unroll
        for (int w = 0; w < kAhead; ++w) blocks_turned(v_in + k_off[w], v0[w]);
        if constexpr (kHalfK) {
            float d[U][NT][4];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[u][n][e] = 0.f;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                uint2 b[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) b[n] = fragment(n * kSteps + s);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    uint32_t x[4];
                    k_halves<E4M3>(a[u][s / 2][s % 2 * 2], x[0], x[2]);
                    k_halves<E4M3>(a[u][s / 2][s % 2 * 2 + 1], x[1], x[3]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma(d[u][n], x[0], x[1], x[2], x[3], b[n].x, b[n].y);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < PER; ++j)
#pragma unroll
                        for (int x = 0; x < 2; ++x)
                            z[u][n][j][x] = (PER == 1 ? d[u][n][2 * x] + d[u][n][2 * x + 1] : d[u][n][2 * x + j]) * (ks[u] * rs[n][j]);
        } else {
            constexpr int kPairs = P / 2;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                uint32_t d[U][kPairs][4];
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int k = 0; k < kPairs; ++k)
#pragma unroll
                        for (int e = 0; e < 4; ++e) d[u][k][e] = kIntZero;
#pragma unroll
                for (int s = 0; s < kLong; ++s)
#pragma unroll
                    for (int k = 0; k < kPairs; ++k) {
                        const uint2 b = fragment((n * kTiles + k) * kLong + s);
#pragma unroll
                        for (int u = 0; u < U; ++u) mma_int(d[u][k], a[u][s], b);
                    }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const float f = ks[u] * rs[n][0];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        float v = 0.f;
#pragma unroll
                        for (int k = P - 1; k >= 0; --k) v = fmaf(v, 0.00390625f, __uint_as_float(d[u][k / 2][2 * x + (k & 1)]) - 12582912.f);
                        z[u][n][0][x] = v * f;
                    }
                }
            }
        }
        // ---- weights
        if (special) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    const int r = n * 4 * PER + PER * c + j;
                    const int lim = r < rows ? (int)min((int64_t)q.before + (r0 + r) / p.G + 1, cap) : end;
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int x = 0; x < 2; ++x)
                            if (!(have >> u & 1u) || tb + 16 * u + g + 8 * x >= lim) z[u][n][j][x] = -INFINITY;
                }
        }
        bool over = false;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < PER; ++j) over |= fmaxf(z[u][n][j][0], z[u][n][j][1]) + base[n][j] > kLift + kSlack;
        if (__any_sync(0xffffffffu, over)) {  // the references move: to the maximum so far
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    float now = m[n][j];
#pragma unroll
                    for (int u = 0; u < U; ++u) now = fmaxf(now, fmaxf(z[u][n][j][0], z[u][n][j][1]));
#pragma unroll
                    for (int d = 4; d < 32; d *= 2) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, d));
                    if (now > -INFINITY) {
                        const float f = exp2_fast(m[n][j] - now);
                        m[n][j] = now;
                        base[n][j] = kLift - now;
                        l[n][j] *= f;
                        scale_o(n, j, f);
                    }
                }
        }
        uint32_t pb[U][NT][2], pl[U][NT][2];  // (pl: PER 2's low halves)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float f = apart ? 1.f : vr[u];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    float w[PER];
#pragma unroll
                    for (int j = 0; j < PER; ++j) {
                        w[j] = exp2_fast(z[u][n][j][x] + base[n][j]);
                        l[n][j] += w[j];
                        w[j] *= f;
                    }
                    __half2 v;
                    if constexpr (PER == 1) {
                        const __half hi = __float2half_rn(w[0]);
                        v = __halves2half2(hi, __float2half_rn(w[0] - __half2float(hi)));
                    } else {
                        v = __floats2half2_rn(w[0], w[PER - 1]);
                        const float2 hi = __half22float2(v);
                        const __half2 lo = __floats2half2_rn(w[0] - hi.x, w[PER - 1] - hi.y);
                        pl[u][n][x] = transpose8(*reinterpret_cast<const uint32_t*>(&lo));
                    }
                    pb[u][n][x] = transpose8(*reinterpret_cast<uint32_t*>(&v));
                }
        }
        // ---- O += V' P, two steps of 16 of hd at a time.  float32: a step's products are added up apart (the tensor cores cut what they add
        // to a long sum: 1.0e-6 of the result against 3e-7 at 8192 tokens); so are, scaled, those of a page whose scale is far below the largest.
        auto turned = [&](int u, int w, uint32_t (&x)[2][4]) {
            uint32_t v[4];  // [step][tokens 0.. | 8..]
            if (u == 0 && kAhead) {
#pragma unroll
                for (int y = 0; y < 4; ++y) v[y] = v0[kAhead ? w / 2 : 0][y];
            } else {
                blocks_turned(v_in + u * 16 * HD + k_off[w / 2], v);
            }
            if (special) {  // what lies behind the last token, or on no page, is not a value
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int t = tb + 16 * u + 2 * c + 8 * (y & 1);
                    if (!(have >> u & 1u) || t >= end) v[y] = 0u;
                    else if (t + 1 >= end) v[y] &= 0xffffu;
                }
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                v_halves<E4M3>(v[2 * y], x[y][0], x[y][1]);
                v_halves<E4M3>(v[2 * y + 1], x[y][2], x[y][3]);
            }
        };
        if (!F32 && !apart) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int w = 0; w < kSteps; w += 2) {
                    uint32_t x[2][4];
                    turned(u, w, x);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            mma(o[n][w + y], x[y][0], x[y][1], x[y][2], x[y][3], pb[u][n][0], pb[u][n][1]);
                            if constexpr (PER == 2) mma(o[n][w + y], x[y][0], x[y][1], x[y][2], x[y][3], pl[u][n][0], pl[u][n][1]);
                        }
                }
        } else {
#pragma unroll
            for (int w = 0; w < kSteps; w += 2) {
                float t[NT][2][4];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    uint32_t x[2][4];
                    turned(u, w, x);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            if (u == 0 || apart) t[n][y][0] = t[n][y][1] = t[n][y][2] = t[n][y][3] = 0.f;
                            mma(t[n][y], x[y][0], x[y][1], x[y][2], x[y][3], pb[u][n][0], pb[u][n][1]);
                            if constexpr (PER == 2) mma(t[n][y], x[y][0], x[y][1], x[y][2], x[y][3], pl[u][n][0], pl[u][n][1]);
                            if (apart || u == U - 1)
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[n][w + y][e] = apart ? fmaf(t[n][y][e], vr[u], o[n][w + y][e]) : o[n][w + y][e] + t[n][y][e];
                        }
                }
            }
        }
        __syncwarp();  // (the step's room is free)
    }
    __syncthreads();  // (the ring becomes O's)

    // ---- join the warps
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int r = n * 4 * PER + PER * c + j;
#pragma unroll
            for (int d = 4; d < 32; d *= 2) l[n][j] += __shfl_xor_sync(0xffffffffu, l[n][j], d);
            if (g == 0) {
                s_m[warp][r] = m[n][j];
                s_l[warp][r] = l[n][j];
            }
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                float2 v;  // elements 16 s + 2 g and the next
                if constexpr (PER == 1) v = make_float2((o[n][s][0] + o[n][s][1]) * v_top, (o[n][s][2] + o[n][s][3]) * v_top);
                else v = make_float2(o[n][s][j] * v_top, o[n][s][2 + j] * v_top);
                *reinterpret_cast<float2*>(&s_part[(warp * kRows + r) * kStride + s * 16 + g * 2]) = v;
            }
        }
    // Part k of the rows' elements is finished by CTA k: everybody sends it there, with its maxima and sums.
    const int slice = (rows * HD + S - 1) / S;
    const uint32_t got = (uint32_t)__cvta_generic_to_shared(s_got), gm = (uint32_t)__cvta_generic_to_shared(s_gm),
                   gl = (uint32_t)__cvta_generic_to_shared(s_gl);
    __syncthreads();
    if (S > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");  // (all have their fragments)
    for (int i = tid; i < S * rows; i += kThreads) {
        const int k = i / rows, r = i % rows;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_m[w][r]);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float f = s_m[w][r] == -INFINITY ? 1.f : exp2_fast(s_m[w][r] - top);  // (no maximum: no weight either, or a NaN)
            if (k == 0) s_f[w][r] = f;
            sum = fmaf(s_l[w][r], f, sum);
        }
        remote_store(gm, k, rank * kRows + r, top);
        remote_store(gl, k, rank * kRows + r, sum);
    }
    __syncthreads();
    for (int e = tid; e < rows * HD; e += kThreads) {
        const int r = e / HD, in = r * kStride + e % HD, k = S > 1 ? e / slice : 0;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v = fmaf(s_part[w * kRows * kStride + in], s_f[w][r], v);
        remote_store(got, k, rank * slice + e - k * slice, v);
    }
    if (S > 1) {
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    } else {
        __syncthreads();
    }
    // the CTAs' factors of a row, one a lane of a quarter of a warp
    for (int i = tid; i < (rows * 8 + 31) / 32 * 32; i += kThreads) {
        const int r = min(i / 8, rows - 1), k = i % 8;
        const float cm = k < S ? s_gm[k][r] : -INFINITY;
        float top = cm;
#pragma unroll
        for (int d = 1; d < 8; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float f = cm == -INFINITY ? 1.f : exp2_fast(cm - top);
        float sum = k < S ? s_gl[k][r] * f : 0.f;
#pragma unroll
        for (int d = 1; d < 8; d *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        s_f[k][r] = f;
        if (k == 0) s_inv[r] = Z > 1 ? 1.f : sum == 0.f ? 0.f : 1.f / sum;  // (a row that sees nothing gives zeros)
        if (Z > 1 && rank == 0 && k == 0 && i / 8 < rows) {
            float* ml = p.part_ml + 2 * (part_of(mine, h, r0 + r, p.s.max_new * p.G, p.c.H) * Z + z_of);
            ml[0] = top;
            ml[1] = sum;
        }
    }
    __syncthreads();
    for (int i = tid; i < slice; i += kThreads) {
        const int e = rank * slice + i;
        if (e >= rows * HD) break;
        const int r = e / HD, d = e % HD;
        float v = 0.f;
#pragma unroll 4
        for (int k = 0; k < S; ++k) v = fmaf(s_got[k * slice + i], s_f[k][r], v);
        if (Z > 1) p.part_o[(part_of(mine, h, r0 + r, p.s.max_new * p.G, p.c.H) * Z + z_of) * HD + d] = v;
        else put(p, q.start + (r0 + r) / p.G, h * p.G + (r0 + r) % p.G, d, v * s_inv[r]);
    }
}

// The last join, of the clusters that shared a row: one block a (sequence, KV head), a row a turn.
__global__ void __launch_bounds__(128) attn8_join(const Attn8Args p, const int Z) {
    pdl_trigger();
    pdl_wait();
    Seq8 q;
    if (!find_seq(p.s, blockIdx.y, q)) return;
    const int h = blockIdx.x, hd = p.c.hd;
    __shared__ float s_f[kMaxSplits], s_inv;
    for (int r = blockIdx.z; r < q.n * p.G; r += gridDim.z) {
        const int64_t part = part_of(blockIdx.y, h, r, p.s.max_new * p.G, p.c.H) * Z;
        if (threadIdx.x < 32) {  // kEach splits a lane
            constexpr int kEach = kMaxSplits / 32;
            static_assert(kMaxSplits % 32 == 0, "every split has a lane");
            float m[kEach], top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int k = threadIdx.x + 32 * i;
                m[i] = k < Z ? p.part_ml[2 * (part + k)] : -INFINITY;
                top = fmaxf(top, m[i]);
            }
            top = warp_max(top);
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int k = threadIdx.x + 32 * i;
                const float f = m[i] == -INFINITY ? 1.f : exp2_fast(m[i] - top);
                s_f[k] = f;
                if (k < Z) sum += p.part_ml[2 * (part + k) + 1] * f;
            }
            sum = warp_sum(sum);
            if (threadIdx.x == 0) s_inv = sum == 0.f ? 0.f : 1.f / sum;
        }
        __syncthreads();
        for (int d = threadIdx.x; d < hd; d += 128) {
            float v = 0.f;
#pragma unroll 8
            for (int k = 0; k < Z; ++k) v = fmaf(p.part_o[(part + k) * hd + d], s_f[k], v);
            put(p, q.start + r / p.G, h * p.G + r % p.G, d, v * s_inv);
        }
        __syncthreads();
    }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// All tokens of a cache's K (or V) as rows of hd bytes, copied 16 at a time, their 16-byte pieces swizzled.
bool make_map(CUtensorMap* m, const void* p, const Cache8& c) {
    static const EncodeTiledFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &r) != cudaSuccess) f = nullptr;
        return reinterpret_cast<EncodeTiledFn>(f);
    }();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)c.hd, ((cuuint64_t)c.n_pages * c.H) << c.shift};
    const cuuint64_t strides[1] = {(cuuint64_t)c.hd};
    const cuuint32_t box[2] = {(cuuint32_t)c.hd, 16}, unit[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
              c.hd == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : c.hd == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a call is cut, from its sizes alone (lengths are on the device; the page table's width bounds them).
struct Plan {
    int tile, W, S, Z;  // query rows a tile, warps a CTA, CTAs a cluster, clusters a tile
};
Plan plan_for(int64_t B, int64_t H, int64_t rows, int64_t longest, bool f32, int n_sm) {
    Plan p;
    p.tile = f32 ? (rows <= 4 ? 4 : rows <= 8 ? 8 : 16) : rows <= 4 ? 4 : rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 24 ? 24 : 32;
    const int64_t items = B * H * ((rows + p.tile - 1) / p.tile);
    const int most = p.tile <= (f32 ? 4 : 8) ? 12 : 8;  // warps that an SM holds, by their registers
    p.S = p.Z = 1;
    // Many items: small CTAs, three an SM, whose starts and ends overlap (1024 items: 229 us, in large CTAs 250).  Fewer: one large
    // CTA an SM, so that the longest item is not the last (256 items: 65.6 us, small CTAs 96).
    p.W = items >= 3 * n_sm ? 4 : most;
    if (items >= n_sm) return p;
    // Less than one an SM: clusters.  Two CTAs each as long as all of them fit twice (128 items of six rows: 57.4 us, one each 69.6, three 71.6), more
    // as long as they fit once.
    if (longest <= 2048) {  // short: small CTAs start sooner (1 x 700 tokens: 8 small ones 12.3 us, 4 large ones 14.3)
        p.W = 4;
        while (p.S < kMaxCluster && items * p.S < n_sm && longest > p.S * 128) p.S *= 2;
        return p;
    }
    p.S = 2;
    while (p.S < kMaxCluster && items * p.S * 2 <= n_sm) p.S *= 2;
    // Long and few: a cluster has 8 CTAs at most, and large clusters leave SMs empty: several pairs, joined by a second launch over the
    // workspace (8 items of 131072 tokens: 9 pairs each 69.8 us, one cluster of 8 each 84).
    if (items * kMaxCluster <= n_sm && longest > 8192) {
        p.S = 2;
        p.Z = (int)std::min<int64_t>(n_sm / (2 * items), kMaxSplits);
    }
    return p;
}

template <int HD, int NT, int PER, bool F32, bool E4M3, int kWarps>
cudaError_t launch(const Attn8Args& a, const Plan& plan, cudaStream_t st, bool pdl) {
    const int S = plan.S, Z = plan.Z;
    constexpr int kRows = NT * 4 * PER;
    constexpr int kSmem = kWarps * std::max(kRows * (HD + 16) * 4, kRing<NT> * kStepBytes<HD, NT>) + 1024;
    auto kern = attn8<HD, NT, PER, F32, E4M3, kWarps>;
    static std::atomic<uint64_t> done{0};
    const cudaError_t ready = allow_launch(kern, kSmem, false, done);
    if (ready != cudaSuccess) return ready;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(S * Z * a.c.H), (unsigned)a.s.B, (unsigned)(((int64_t)a.s.max_new * a.G + kRows - 1) / kRows));
    cfg.blockDim = dim3(32 * kWarps);
    cfg.dynamicSmemBytes = kSmem;
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
    CUtensorMap mk{}, mv{};
    if (a.c.n_pages > 0 && (!make_map(&mk, a.c.k, a.c) || !make_map(&mv, a.c.v, a.c))) return cudaErrorUnknown;  // (without pages nothing is copied)
    cudaError_t e = cudaLaunchKernelEx(&cfg, kern, mk, mv, a, S, Z);
    if (e != cudaSuccess || Z == 1) return e;
    cfg.gridDim = dim3(a.c.H, a.s.B, std::min(a.s.max_new * a.G, 64));
    cfg.blockDim = dim3(128);
    cfg.dynamicSmemBytes = 0;
    cfg.attrs = at + 1;  // (it may be set up while the last CTAs above still work)
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attn8_join, a, Z);
}

template <int HD, bool F32, bool E4M3>
cudaError_t launch_rows(const Attn8Args& a, cudaStream_t st, bool pdl, int n_sm) {
    Plan p = plan_for(a.s.B, a.c.H, (int64_t)a.s.max_new * a.G, a.s.width << a.c.shift, F32, n_sm);
    if (!a.part_o && p.Z > 1) {  // no room for them: one cluster each
        p.Z = 1;
        p.S = kMaxCluster;
    }
    if constexpr (F32) {
        if (p.W > 4) return p.tile == 4 ? launch<HD, 1, 1, F32, E4M3, 12>(a, p, st, pdl) : p.tile == 8 ? launch<HD, 2, 1, F32, E4M3, 8>(a, p, st, pdl)
                                                                                                  : launch<HD, 4, 1, F32, E4M3, 8>(a, p, st, pdl);
        return p.tile == 4 ? launch<HD, 1, 1, F32, E4M3, 4>(a, p, st, pdl) : p.tile == 8 ? launch<HD, 2, 1, F32, E4M3, 4>(a, p, st, pdl)
                                                                                    : launch<HD, 4, 1, F32, E4M3, 4>(a, p, st, pdl);
    } else {
        switch (p.tile) {
            case 4: return p.W > 4 ? launch<HD, 1, 1, F32, E4M3, 12>(a, p, st, pdl) : launch<HD, 1, 1, F32, E4M3, 4>(a, p, st, pdl);
            case 8: return p.W > 4 ? launch<HD, 1, 2, F32, E4M3, 12>(a, p, st, pdl) : launch<HD, 1, 2, F32, E4M3, 4>(a, p, st, pdl);
            case 16: return p.W > 4 ? launch<HD, 2, 2, F32, E4M3, 8>(a, p, st, pdl) : launch<HD, 2, 2, F32, E4M3, 4>(a, p, st, pdl);
            case 24: return p.W > 4 ? launch<HD, 3, 2, F32, E4M3, 8>(a, p, st, pdl) : launch<HD, 3, 2, F32, E4M3, 4>(a, p, st, pdl);
            default: return p.W > 4 ? launch<HD, 4, 2, F32, E4M3, 8>(a, p, st, pdl) : launch<HD, 4, 2, F32, E4M3, 4>(a, p, st, pdl);
        }
    }
}

}  // namespace

namespace first {

cudaError_t attn8_launch(const Attn8Args& a, cudaStream_t st, bool pdl, int n_sm) {
#define FIRST_ATTN8(HD)                                                                                                            \
    if (a.q.f32) return a.c.e4m3 ? launch_rows<HD, true, true>(a, st, pdl, n_sm) : launch_rows<HD, true, false>(a, st, pdl, n_sm); \
    return a.c.e4m3 ? launch_rows<HD, false, true>(a, st, pdl, n_sm) : launch_rows<HD, false, false>(a, st, pdl, n_sm)
    if (a.c.hd == 32) { FIRST_ATTN8(32); }
    if (a.c.hd == 64) { FIRST_ATTN8(64); }
    FIRST_ATTN8(128);
#undef FIRST_ATTN8
}

int64_t attn8_part_floats(int64_t B, int64_t H, int64_t rows, int hd, int64_t longest, bool f32, int n_sm) {
    const Plan p = plan_for(B, H, rows, longest, f32, n_sm);
    return p.Z > 1 ? B * H * rows * p.Z * (hd + 2) : 0;
}

}  // namespace first

extern "C" int first_attn8(const first_cache8* cache, const void* q, int64_t q_token_stride, int64_t q_head_stride,
                           int32_t n_q_heads, int32_t dtype, float scale, const int32_t* cu_new, int32_t total,
                           const int32_t* pages, int32_t max_pages, const int32_t* len, int32_t B, int32_t max_new, void* out,
                           int64_t out_token_stride, int64_t out_head_stride, void* workspace, int64_t workspace_bytes,
                           uint32_t* flags, void* stream) {
    int rc = check_cache8(cache);
    if (rc) return rc;
    const int hd = cache->head_dim;
    if ((rc = check_seqs8(pages, max_pages, len, cu_new, B, total, max_new, flags))) return rc;
    if (n_q_heads <= 0 || workspace_bytes < 0) return FIRST_E_ARG;
    if (!words_ok({workspace})) return FIRST_E_UNSUPPORTED;
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
    if ((int64_t)max_pages * cache->page > (1 << 30) || (int64_t)a.s.max_new * a.G > (1 << 18) || B > 65535) return FIRST_E_CAPACITY;
    const bool f32 = dtype == FIRST_DTYPE_F32;
    a.q = Rows8{const_cast<void*>(q), q_token_stride, q_head_stride, f32};
    a.out = Rows8{out, out_token_stride, out_head_stride, f32};
    a.scale = scale;
    const int64_t rows = (int64_t)a.s.max_new * a.G, need = attn8_part_floats(B, a.c.H, rows, hd, a.s.width << a.c.shift, f32, kSMs);
    if (workspace && need > 0 && workspace_bytes >= need * 4) {
        a.part_o = static_cast<float*>(workspace);
        a.part_ml = a.part_o + need / (hd + 2) * hd;
    }
    return attn8_launch(a, static_cast<cudaStream_t>(stream), false, kSMs) == cudaSuccess ? FIRST_OK : FIRST_E_CUDA;
}

extern "C" int64_t first_attn8_workspace(const first_cache8* cache, int32_t n_q_heads, int32_t dtype, int32_t total, int32_t max_pages,
                                         int32_t B, int32_t max_new) {
    if (check_cache8(cache) || n_q_heads <= 0 || n_q_heads % cache->n_kv_heads || total <= 0 || max_pages <= 0 || B <= 0 || max_new <= 0) return 0;
    const int64_t rows = (int64_t)std::min(max_new, total) * (n_q_heads / cache->n_kv_heads);
    return 4 * attn8_part_floats(B, cache->n_kv_heads, rows, cache->head_dim, (int64_t)max_pages * cache->page, dtype == FIRST_DTYPE_F32, kSMs);
}
