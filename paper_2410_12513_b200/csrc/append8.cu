// Paged 8-bit cache: new keys and values into pages, values back out of them, and pages from place to place.
#include <algorithm>

#include "cache8.cuh"

using namespace first;

namespace first {

int check_cache8(const first_cache8* c) {
    if (!c || c->n_pages < 0 || c->n_kv_heads <= 0) return FIRST_E_ARG;
    if (c->format != FIRST_CACHE_INT8 && c->format != FIRST_CACHE_E4M3) return FIRST_E_ARG;
    if (c->n_pages > 0 && (!c->k || !c->v || !c->k_scale || !c->v_scale)) return FIRST_E_ARG;
    if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return FIRST_E_UNSUPPORTED;
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return FIRST_E_UNSUPPORTED;
    if (c->n_kv_heads > 1024) return FIRST_E_UNSUPPORTED;
    if ((int64_t)c->n_pages * c->n_kv_heads * c->page > 0x7fffffff) return FIRST_E_CAPACITY;  // (rows are counted in 32 bits)
    if ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v)) % 16) return FIRST_E_UNSUPPORTED;
    if (!words_ok({c->k_scale, c->v_scale})) return FIRST_E_UNSUPPORTED;
    return FIRST_OK;
}

int check_seqs8(const int32_t* pages, int32_t max_pages, const int32_t* len, const int32_t* cu, int32_t B, int32_t total, int32_t max_new,
                const uint32_t* flags) {
    if (B < 0 || total < 0 || max_pages < 0 || max_new < 0) return FIRST_E_ARG;
    if (!cu && total != B) return FIRST_E_SHAPE;
    if (B > 0 && total > 0 && max_new > 0 && (!len || (max_pages > 0 && !pages))) return FIRST_E_ARG;
    return words_ok({pages, len, cu, flags}) ? FIRST_OK : FIRST_E_UNSUPPORTED;
}

// Rows that are written belong to one (token, head) each; rows that are read may repeat.
int check_rows8(const void* p, int64_t tok, int64_t head, int32_t heads, int32_t hd, int32_t dtype, int64_t total, bool written) {
    if (dtype != FIRST_DTYPE_F32 && dtype != FIRST_DTYPE_BF16) return FIRST_E_ARG;
    if (tok < 0 || head < 0) return FIRST_E_SHAPE;
    if (written && total > 0) {
        if (heads > 1 && head < hd) return FIRST_E_SHAPE;
        if (total > 1 && !(heads == 1 ? tok >= hd : tok >= (heads - 1) * head + hd || (tok >= hd && head >= (total - 1) * tok + hd)))
            return FIRST_E_SHAPE;
    }
    if (total > 0 && !p) return FIRST_E_ARG;
    if (reinterpret_cast<uintptr_t>(p) % (dtype == FIRST_DTYPE_F32 ? 4 : 2)) return FIRST_E_UNSUPPORTED;
    return FIRST_OK;
}

Cache8 cache8_of(const first_cache8& c) {
    Cache8 o;
    o.k = static_cast<uint8_t*>(c.k);
    o.v = static_cast<uint8_t*>(c.v);
    o.ks = c.k_scale;
    o.vs = c.v_scale;
    o.n_pages = c.n_pages;
    o.H = c.n_kv_heads;
    for (o.shift = 4; (1 << o.shift) < c.page;) ++o.shift;
    o.hd = c.head_dim;
    o.e4m3 = c.format == FIRST_CACHE_E4M3;
    return o;
}

}  // namespace first

namespace {

// The 8-bit value nearest to an exact quotient num / den (ties to even, saturated; NaN gives 0), in 64 bits: the quotient
// of two float32 is nearer to a tie than 64 bits resolve only where it is one.
template <bool E4M3>
__device__ __noinline__ uint32_t quotient_slow(double num, double den) {
    const double y = num / den;
    if (!(y == y)) return 0;
    if constexpr (E4M3) {
        const double a = fmin(fabs(y), 448.0);
        int e = 0;
        frexp(a, &e);  // a in [2^(e-1), 2^e)
        e = max(e, -5);
        const double step = ldexp(1.0, e - 4);
        const float r = (float)(rint(a / step) * step);
        return __nv_cvt_float_to_fp8(y < 0 ? -r : r, __NV_SATFINITE, __NV_E4M3);
    } else {
        return (uint32_t)(uint8_t)(int8_t)(int)rint(fmin(fmax(y, -127.0), 127.0));
    }
}

// Eight elements of a row, as they are in memory, and as float32.
template <typename T>
struct Eight {
    uint32_t w[2 * sizeof(T)];
};
template <typename T, bool WIDE>
__device__ __forceinline__ Eight<T> load8(const T* p) {
    Eight<T> r;
    if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const uint4 u = reinterpret_cast<const uint4*>(p)[i];
            r.w[4 * i] = u.x; r.w[4 * i + 1] = u.y; r.w[4 * i + 2] = u.z; r.w[4 * i + 3] = u.w;
        }
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.w[i] = reinterpret_cast<const uint32_t*>(p)[i];
    } else {
        const uint16_t* s = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = s[2 * i] | (uint32_t)s[2 * i + 1] << 16;
    }
    return r;
}
template <typename T>
__device__ __forceinline__ float value_of(const Eight<T>& r, int i) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(r.w[i]);
    else return i & 1 ? bf_hi(r.w[i / 2]) : bf_lo(r.w[i / 2]);
}
// Largest magnitude so far, as float32 bits (bfloat16: two 16-bit halves side by side): magnitudes are ordered like their bits.
template <typename T>
__device__ __forceinline__ uint32_t larger(uint32_t m, const Eight<T>& r) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, r.w[i] & 0x7fffffffu);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) m = __vmaxu2(m, r.w[i] & 0x7fff7fffu);
    }
    return m;
}
template <typename T>
__device__ __forceinline__ uint32_t largest(uint32_t m) {
    return sizeof(T) == 4 ? m : max(m & 0xffff0000u, m << 16);
}

// Eight finite values to 8 bits at once, if none is close to a tie: x * inv is within 2^-22 of the quotient.  (|x| is at most the
// scale's 127 or 448 times, so nothing saturates but by that much.)  false: some are.
template <bool E4M3, typename T>
__device__ __forceinline__ bool quotients(const Eight<T>& r, float inv, uint2& out) {
    uint32_t o[2];
    if constexpr (E4M3) {
        const float lo = inv * (1.f - 0x1p-20f), hi = inv * (1.f + 0x1p-20f);
        uint32_t diff = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t c[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float x = value_of(r, 4 * h + 2 * i), y = value_of(r, 4 * h + 2 * i + 1);
                c[i][0] = __nv_cvt_float2_to_fp8x2(make_float2(x * lo, y * lo), __NV_SATFINITE, __NV_E4M3);
                c[i][1] = __nv_cvt_float2_to_fp8x2(make_float2(x * hi, y * hi), __NV_SATFINITE, __NV_E4M3);
                diff |= c[i][0] ^ c[i][1];
            }
            o[h] = c[0][0] | c[1][0] << 16;
        }
        out = make_uint2(o[0], o[1]);
        return diff == 0;
    } else {
        float off = 0.f;
        uint32_t b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float y = value_of(r, i) * inv, m = y + 12582912.f;  // 1.5 2^23: the nearest whole number, in the low bits
            off = fmaxf(off, fabsf(y - (m - 12582912.f)));
            b[i] = __float_as_uint(m);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) o[h] = __byte_perm(__byte_perm(b[4 * h], b[4 * h + 1], 0x0040), __byte_perm(b[4 * h + 2], b[4 * h + 3], 0x0040), 0x5410);
        out = make_uint2(o[0], o[1]);
        return off < 0.4999f;
    }
}

// Eight finite values exactly (out of line): where a little more and a little less than x * inv have different neighbours, x is compared
// with the middle between the two, times the scale: a fused product and difference has the exact sign, as long as it cannot fall below the smallest
// float32 (a scale from 2^-100 up).  (bfloat16 values meet exact ties often: quotients of 8-bit numbers.)
template <bool E4M3, typename T>
__device__ __noinline__ uint2 quotients_exact(const Eight<T> r, float s, float inv) {
    uint32_t w[2] = {0, 0};
    const float lo = inv * (1.f - 0x1p-20f), hi = inv * (1.f + 0x1p-20f);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = value_of(r, e);
        uint32_t a, b;
        float va, vb;
        if constexpr (E4M3) {
            a = __nv_cvt_float_to_fp8(x * lo, __NV_SATFINITE, __NV_E4M3);
            b = __nv_cvt_float_to_fp8(x * hi, __NV_SATFINITE, __NV_E4M3);
            va = to_value<true>(a);
            vb = to_value<true>(b);
        } else {
            va = rintf(x * lo);
            vb = rintf(x * hi);
            a = (uint32_t)(int)va & 255u;
            b = (uint32_t)(int)vb & 255u;
        }
        const float d = fmaf(-0.5f * (va + vb), s, x);
        const bool second = d == 0.f ? (a & 1u) != 0u : (d > 0.f) == (vb > va);
        w[e >> 2] |= (a != b && second ? b : a) << (8 * (e & 3));
    }
    return make_uint2(w[0], w[1]);
}
// Eight of any values, one by one.
template <bool E4M3, typename T>
__device__ __noinline__ uint2 quotients_slow(const Eight<T> r, float s) {
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e >> 2] |= (s > 0.f ? quotient_slow<E4M3>((double)value_of(r, e), (double)s) : 0u) << (8 * (e & 3));
    return make_uint2(w[0], w[1]);
}

constexpr int kAppendHold = 8;  // vectors of 8 elements that a thread keeps between the two passes

// One block a (page that gains tokens, head, K or V): the largest magnitude of the new values, the page's scale, and the
// new values rounded to it; where the scale grew the page's earlier values are rounded to it again.  The new values are read once and stay in
// registers.  4 prompts of 8190 tokens, 8 heads of 128, bfloat16 to E4M3: 58 us, 3.5 TB/s read and written (35 % of DRAM, the ALU pipe 70 % busy with
// magnitudes, conversions and packing; values read in two passes 130 us).  32 single tokens: 3.6 us, a launch and three latencies.
template <typename T, bool E4M3, bool WIDE, int kThreads>
__global__ void __launch_bounds__(kThreads) append8(const Cache8 c, const Seqs8 s, const Rows8 kr, const Rows8 vr) {
    const Stamp stamp_guard(s.stamp);
    pdl_trigger();
    pdl_wait();
    Seq8 q;
    if (!find_seq(s, blockIdx.z, q)) return;
    const int tid = threadIdx.x, h = blockIdx.x >> 1, hd = c.hd, page = 1 << c.shift;
    const bool is_v = blockIdx.x & 1;
    int64_t row0 = q.start;
    if (s.row_off) {
        row0 += *s.row_off;
        if (row0 < 0 || row0 + q.n > s.row_total || (s.row_cap && q.n > *s.row_cap)) {  // more than the sequence has there
            if (s.flags && tid == 0) atomicOr(s.flags, FIRST_FLAG_BAD_SEQ_TABLE);
            return;
        }
    }
    const int64_t first = ((int64_t)(q.before >> c.shift) + blockIdx.y) << c.shift;  // the page's first position
    const int64_t end = (int64_t)q.before + q.n;
    if (first >= end) return;
    const int p = find_page(s, c.n_pages, q.seq, first >> c.shift);
    if (p < 0) {  // no room: the tokens are left out
        if (s.flags && tid == 0) atomicOr(s.flags, FIRST_FLAG_KV_FULL);
        return;
    }
    const int lo = (int)max((int64_t)q.before - first, (int64_t)0), hi = (int)min(end - first, (int64_t)page);
    const Rows8& r = is_v ? vr : kr;
    // row `lo` of the page
    const T* src = static_cast<const T*>(r.p) + (row0 + first + lo - q.before) * r.tok + h * r.head;
    uint8_t* dst = (is_v ? c.v : c.k) + ((((int64_t)p * c.H + h) << c.shift)) * hd;
    float* scale = (is_v ? c.vs : c.ks) + (int64_t)p * c.H + h;
    const float held = lo > 0 ? *scale : 0.f;
    const int vs = hd == 128 ? 4 : hd == 64 ? 3 : 2, nv = (hi - lo) << vs;  // vectors of a row: 2^vs
    Eight<T> x[kAppendHold];
    uint32_t m = 0;
    const T* from = src + (tid >> vs) * r.tok + (tid & ((1 << vs) - 1)) * 8;
#pragma unroll
    for (int k = 0; k < kAppendHold; ++k) {
        const int i = tid + k * kThreads;
        if (i < nv) x[k] = load8<T, WIDE>(from);
        from += (kThreads >> vs) * r.tok;
    }
    if constexpr (sizeof(T) == 4) {
        if (s.cs && !is_v) {  // (the step) rotary pairs (d, d + hd/2)
            const float2* cs = s.cs + (int64_t)q.seq * (hd / 2);
#pragma unroll
            for (int k = 0; k < kAppendHold; ++k) {
                const int i = tid + k * kThreads, d = (i & ((1 << vs) - 1)) * 8;
                if (i >= nv) break;
                const bool up = d >= hd / 2;
                const int at = up ? d - hd / 2 : d;
                const Eight<T> y = load8<T, WIDE>(src + (int64_t)(i >> vs) * r.tok + (up ? at : d + hd / 2));
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 t = cs[at + e];
                    const float a = __uint_as_float(x[k].w[e]), b = __uint_as_float(y.w[e]);
                    x[k].w[e] = __float_as_uint(up ? a * t.x + b * t.y : a * t.x - b * t.y);
                }
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kAppendHold; ++k)
        if (tid + k * kThreads < nv) m = larger(m, x[k]);
    m = largest<T>(m);
    __shared__ uint32_t red[kThreads / 32];
    uint32_t amax = __reduce_max_sync(0xffffffffu, m);
    if ((tid & 31) == 0) red[tid >> 5] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) amax = max(amax, red[w]);
    const bool odd = amax >= 0x7f800000u;  // not all are finite: the largest of those that are
    if (odd) {
        m = 0;
        for (int k = 0; k < kAppendHold; ++k)
            if (tid + k * kThreads < nv)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t u = __float_as_uint(value_of(x[k], e)) & 0x7fffffffu;
                    m = max(m, u < 0x7f800000u ? u : 0u);
                }
        amax = __reduce_max_sync(0xffffffffu, m);
        __syncthreads();
        if ((tid & 31) == 0) red[tid >> 5] = amax;
        __syncthreads();
        for (int w = 0; w < kThreads / 32; ++w) amax = max(amax, red[w]);
    }
    const float fresh = __uint_as_float(amax) * (1.f / (E4M3 ? 448.f : 127.f));
    const float now = held >= fresh || held != held ? held : fresh;  // (a NaN stays: what the page holds is none either)
    const float inv = now >= 0x1p-100f ? 1.f / now : 0.f;
#pragma unroll
    for (int k = 0; k < kAppendHold; ++k) {
        const int i = tid + k * kThreads;
        if (i < nv) {
            uint2 o;
            if (odd || !(inv > 0.f)) o = quotients_slow<E4M3>(x[k], now);
            else if (!quotients<E4M3>(x[k], inv, o)) o = quotients_exact<E4M3>(x[k], now, inv);
            *reinterpret_cast<uint2*>(dst + lo * hd + i * 8) = o;
        }
    }
    if (lo > 0 && now > held) {
        const float ratio = (float)((double)held / (double)now);
        for (int i = tid; i < lo * hd / 4; i += kThreads) {
            uint32_t* w = reinterpret_cast<uint32_t*>(dst) + i;
            const uint32_t old = *w;
            uint32_t o = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = to_value<E4M3>(old >> (8 * e) & 255u);
                const float y = x * ratio;
                uint32_t code;
                bool sure;
                if constexpr (E4M3) {
                    code = __nv_cvt_float_to_fp8(y * (1.f - 0x1p-20f), __NV_SATFINITE, __NV_E4M3);
                    sure = code == __nv_cvt_float_to_fp8(y * (1.f + 0x1p-20f), __NV_SATFINITE, __NV_E4M3);
                } else {
                    const float rr = rintf(y);
                    code = (uint32_t)(uint8_t)(int8_t)(int)rr;
                    sure = fabsf(y - rr) < 0.4999f;
                }
                if (!sure) code = quotient_slow<E4M3>((double)x * (double)held, (double)now);
                o |= code << (8 * e);
            }
            *w = o;
        }
    }
    if (tid == 0) *scale = now;
}

// Values of pages as rows: one thread a 16 bytes of K and of V, a block neighbouring tokens of a head (adjacent in their pages).
// 4 x 8190 tokens of 8 heads of 128, E4M3 to bfloat16: 38 us, 5.3 TB/s (half of the writes still in L2 at the end).
template <typename T, bool E4M3, bool WIDE>
__global__ void __launch_bounds__(256) read8(const Cache8 c, const Seqs8 s, const Rows8 kr, const Rows8 vr) {
    Seq8 q;
    if (!find_seq(s, blockIdx.y, q)) return;
    const int vs = c.hd == 128 ? 3 : c.hd == 64 ? 2 : 1;  // 2^vs vectors a row
    const int64_t row = (int64_t)blockIdx.x * (256 >> vs) + (threadIdx.x >> vs);
    if (row >= q.n) return;
    const int h = blockIdx.z, d = (threadIdx.x & ((1 << vs) - 1)) * 16;
    const int64_t pos = (int64_t)q.before + row;
    const int p = find_page(s, c.n_pages, q.seq, pos >> c.shift);
    if (p < 0) {
        if (s.flags) atomicOr(s.flags, FIRST_FLAG_BAD_PAGE);
        return;
    }
    const int64_t at = ((((int64_t)p * c.H + h) << c.shift) + (pos & ((1 << c.shift) - 1))) * c.hd + d;
    const float scale[2] = {c.ks[(int64_t)p * c.H + h], c.vs[(int64_t)p * c.H + h]};
    const uint4 in[2] = {*reinterpret_cast<const uint4*>(c.k + at), *reinterpret_cast<const uint4*>(c.v + at)};
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const Rows8& r = w ? vr : kr;
        T* o = static_cast<T*>(r.p) + (q.start + row) * r.tok + h * r.head + d;
        const uint32_t u[4] = {in[w].x, in[w].y, in[w].z, in[w].w};
        struct alignas(16) Out { T e[16 / sizeof(T)]; };
        Out t[sizeof(T)];
#pragma unroll
        for (int e = 0; e < 16; ++e)
            t[e / (16 / sizeof(T))].e[e % (16 / sizeof(T))] = from_f32<T>(to_value<E4M3>(u[e >> 2] >> (8 * (e & 3)) & 255u) * scale[w]);
#pragma unroll
        for (int e = 0; e < (int)sizeof(T); ++e) {
            if constexpr (WIDE) {
                reinterpret_cast<Out*>(o)[e] = t[e];
            } else {
#pragma unroll
                for (int x = 0; x < (int)(16 / sizeof(T)); ++x) o[e * (16 / sizeof(T)) + x] = t[e].e[x];
            }
        }
    }
}

constexpr int kMaxCopyLayers = 96;  // the layers' addresses travel as kernel parameters
struct CopyArgs {
    uint8_t *k[kMaxCopyLayers], *v[kMaxCopyLayers];
    float *ks[kMaxCopyLayers], *vs[kMaxCopyLayers];
    int n_pages[kMaxCopyLayers];
    int L, H;
    int bytes, chunks;  // of a page's K, and pieces it is cut into
    const int32_t* moves;
    int64_t units;
    uint32_t* flags;
};
constexpr int kCopyChunk = 256 * 16 * 4;

// One block a 16 KB of K or V of a move: a thread has four 16-byte loads out before its first store.  Bound by HBM: 5120 moves of 64 tokens
// of 8 heads of 128, 1342 MB read and written, 196 us, 6.8 TB/s.
__global__ void __launch_bounds__(256) copy_pages(const __grid_constant__ CopyArgs a) {
    const int64_t unit = blockIdx.x;
    const int piece = (int)(unit % (2 * a.chunks)), chunk = piece >> 1;
    const int32_t* m = a.moves + unit / (2 * a.chunks) * 3;
    const int l = m[0], from = m[1], to = m[2];
    if (l < 0 || l >= a.L || from < 0 || to < 0 || from >= a.n_pages[l] || to >= a.n_pages[l]) {
        if (a.flags && threadIdx.x == 0) atomicOr(a.flags, FIRST_FLAG_BAD_PAGE);
        return;
    }
    if (from == to) return;
    uint8_t* base = piece & 1 ? a.v[l] : a.k[l];
    float* sc = piece & 1 ? a.vs[l] : a.ks[l];
    const int64_t at = (int64_t)chunk * kCopyChunk;
    const uint4* src = reinterpret_cast<const uint4*>(base + (int64_t)from * a.bytes + at);
    uint4* dst = reinterpret_cast<uint4*>(base + (int64_t)to * a.bytes + at);
    const int n = (int)min((int64_t)kCopyChunk, a.bytes - at) / 16;
    uint4 r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if ((int)threadIdx.x + i * 256 < n) r[i] = src[threadIdx.x + i * 256];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if ((int)threadIdx.x + i * 256 < n) dst[threadIdx.x + i * 256] = r[i];
    if (chunk == 0)
        for (int h = threadIdx.x; h < a.H; h += 256) sc[(int64_t)to * a.H + h] = sc[(int64_t)from * a.H + h];
}

bool aligned16(const Rows8& r) {
    const int es = r.f32 ? 4 : 2;
    return reinterpret_cast<uintptr_t>(r.p) % 16 == 0 && r.tok * es % 16 == 0 && r.head * es % 16 == 0;
}

}  // namespace

namespace first {

cudaError_t append8_launch(const Cache8& c, const Seqs8& s, const Rows8& k, const Rows8& v, cudaStream_t st, bool pdl) {
    const int pages = (int)(((int64_t)s.max_new + (1 << c.shift) - 2) / (1 << c.shift) + 1);  // that a sequence's tokens touch at most
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(2 * c.H, s.max_new == 1 ? 1 : pages, s.B);  // (neighbouring heads of a token run together)
    const bool large = (c.hd << c.shift) > 128 * 8 * kAppendHold;    // a page's head in 128 threads' registers, or 256's
    cfg.blockDim = dim3(large ? 256 : 128);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl ? 1 : 0;
    const bool wide = aligned16(k) && aligned16(v);
#define FIRST_APPEND(T, E, W) return large ? cudaLaunchKernelEx(&cfg, append8<T, E, W, 256>, c, s, k, v) : cudaLaunchKernelEx(&cfg, append8<T, E, W, 128>, c, s, k, v)
    if (k.f32) {
        if (c.e4m3) { if (wide) FIRST_APPEND(float, true, true); else FIRST_APPEND(float, true, false); }
        else { if (wide) FIRST_APPEND(float, false, true); else FIRST_APPEND(float, false, false); }
    }
    if (c.e4m3) { if (wide) FIRST_APPEND(__nv_bfloat16, true, true); else FIRST_APPEND(__nv_bfloat16, true, false); }
    if (wide) FIRST_APPEND(__nv_bfloat16, false, true); else FIRST_APPEND(__nv_bfloat16, false, false);
#undef FIRST_APPEND
}

}  // namespace first

extern "C" {

int first_append8(const first_cache8* cache, const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v,
                  int64_t v_token_stride, int64_t v_head_stride, int32_t dtype, const int32_t* cu_new, int32_t total,
                  const int32_t* pages, int32_t max_pages, const int32_t* len, int32_t B, int32_t max_new, uint32_t* flags,
                  void* stream) {
    int rc = check_cache8(cache);
    if (rc || (rc = check_seqs8(pages, max_pages, len, cu_new, B, total, max_new, flags)) ||
        (rc = check_rows8(k, k_token_stride, k_head_stride, cache->n_kv_heads, cache->head_dim, dtype, total, false)) ||
        (rc = check_rows8(v, v_token_stride, v_head_stride, cache->n_kv_heads, cache->head_dim, dtype, total, false)))
        return rc;
    if (B == 0 || total == 0 || max_new == 0) return FIRST_OK;
    const Cache8 c = cache8_of(*cache);
    if (B > 65535 || (int64_t)max_pages * cache->page > (1 << 30) || (max_new >> c.shift) > 65000) return FIRST_E_CAPACITY;
    Seqs8 s;
    s.pages = pages; s.width = max_pages; s.len = len; s.cu = cu_new;
    s.B = B; s.total = total; s.max_new = std::min(max_new, total); s.flags = flags;
    const bool f32 = dtype == FIRST_DTYPE_F32;
    const Rows8 kr{const_cast<void*>(k), k_token_stride, k_head_stride, f32}, vr{const_cast<void*>(v), v_token_stride, v_head_stride, f32};
    return append8_launch(c, s, kr, vr, static_cast<cudaStream_t>(stream), false) == cudaSuccess ? FIRST_OK : FIRST_E_CUDA;
}

int first_read8(const first_cache8* cache, const int32_t* pages, int32_t max_pages, const int32_t* start, const int32_t* cu,
                int32_t B, int32_t total, int32_t max_rows, void* k, int64_t k_token_stride, int64_t k_head_stride, void* v,
                int64_t v_token_stride, int64_t v_head_stride, int32_t dtype, uint32_t* flags, void* stream) {
    int rc = check_cache8(cache);
    if (rc || (rc = check_seqs8(pages, max_pages, start, cu, B, total, max_rows, flags)) ||
        (rc = check_rows8(k, k_token_stride, k_head_stride, cache->n_kv_heads, cache->head_dim, dtype, total, true)) ||
        (rc = check_rows8(v, v_token_stride, v_head_stride, cache->n_kv_heads, cache->head_dim, dtype, total, true)))
        return rc;
    if (B == 0 || total == 0 || max_rows == 0) return FIRST_OK;
    if (B > 65535 || (int64_t)max_pages * cache->page > (1 << 30)) return FIRST_E_CAPACITY;
    const Cache8 c = cache8_of(*cache);
    Seqs8 s;
    s.pages = pages; s.width = max_pages; s.len = start; s.cu = cu;
    s.B = B; s.total = total; s.max_new = std::min(max_rows, total); s.flags = flags;
    const bool f32 = dtype == FIRST_DTYPE_F32;
    const Rows8 kr{k, k_token_stride, k_head_stride, f32}, vr{v, v_token_stride, v_head_stride, f32};
    const int per = 256 / (c.hd / 16);
    const dim3 grid((unsigned)((s.max_new - 1) / per + 1), B, c.H);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool wide = aligned16(kr) && aligned16(vr);
#define FIRST_READ(T, E, W) read8<T, E, W><<<grid, 256, 0, st>>>(c, s, kr, vr)
    if (f32) {
        if (c.e4m3) { if (wide) FIRST_READ(float, true, true); else FIRST_READ(float, true, false); }
        else { if (wide) FIRST_READ(float, false, true); else FIRST_READ(float, false, false); }
    } else {
        if (c.e4m3) { if (wide) FIRST_READ(__nv_bfloat16, true, true); else FIRST_READ(__nv_bfloat16, true, false); }
        else { if (wide) FIRST_READ(__nv_bfloat16, false, true); else FIRST_READ(__nv_bfloat16, false, false); }
    }
#undef FIRST_READ
    return cudaGetLastError() == cudaSuccess ? FIRST_OK : FIRST_E_CUDA;
}

int first_copy_pages(const first_cache8* layers, int32_t n_layers, const int32_t* moves, int64_t n_moves, uint32_t* flags,
                     void* stream) {
    if (!layers || n_layers <= 0 || n_moves < 0 || (n_moves > 0 && !moves)) return FIRST_E_ARG;
    if (n_layers > kMaxCopyLayers || !words_ok({moves, flags})) return FIRST_E_UNSUPPORTED;
    CopyArgs a{};
    for (int l = 0; l < n_layers; ++l) {
        int rc = check_cache8(layers + l);
        if (rc) return rc;
        const first_cache8 &c = layers[l], &d = layers[0];
        if (c.format != d.format || c.n_kv_heads != d.n_kv_heads || c.page != d.page || c.head_dim != d.head_dim) return FIRST_E_SHAPE;
        a.k[l] = static_cast<uint8_t*>(c.k);
        a.v[l] = static_cast<uint8_t*>(c.v);
        a.ks[l] = c.k_scale;
        a.vs[l] = c.v_scale;
        a.n_pages[l] = c.n_pages;
    }
    if (n_moves == 0) return FIRST_OK;
    a.L = n_layers;
    a.H = layers[0].n_kv_heads;
    a.bytes = a.H * layers[0].page * layers[0].head_dim;
    a.chunks = (a.bytes + kCopyChunk - 1) / kCopyChunk;
    a.moves = moves;
    if (n_moves > (0x7fffffff / 2) / a.chunks) return FIRST_E_CAPACITY;  // (grid size)
    a.units = n_moves * 2 * a.chunks;
    a.flags = flags;
    copy_pages<<<(unsigned)a.units, 256, 0, static_cast<cudaStream_t>(stream)>>>(a);
    return cudaGetLastError() == cudaSuccess ? FIRST_OK : FIRST_E_CUDA;
}

}  // extern "C"
