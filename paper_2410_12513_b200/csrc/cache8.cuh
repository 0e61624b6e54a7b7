// Device helpers of the paged 8-bit cache: 8-bit values to halves for the tensor cores, sequences and their pages.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"
#include "first.h"
#include "ops.h"

namespace first {

// Four 8-bit values -> two pairs of halves, exactly.  Integers: 0x64 above a byte is 1024 + byte.
template <bool E4M3>
__device__ __forceinline__ void to_halves(uint32_t w, uint32_t& a, uint32_t& b) {
    if constexpr (E4M3) {
        asm("{.reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}"
            : "=r"(a), "=r"(b) : "r"(w));
    } else {
        const uint32_t u = w ^ 0x80808080u;
        const __half2 bias = __half2half2(__ushort_as_half(0x6480));  // 1152
        uint32_t x = __byte_perm(u, 0x64646464u, 0x4140), y = __byte_perm(u, 0x64646464u, 0x4342);
        const __half2 p = __hsub2(*reinterpret_cast<__half2*>(&x), bias), q = __hsub2(*reinterpret_cast<__half2*>(&y), bias);
        a = *reinterpret_cast<const uint32_t*>(&p);
        b = *reinterpret_cast<const uint32_t*>(&q);
    }
}

// One 8-bit value as float32.
template <bool E4M3>
__device__ __forceinline__ float to_value(uint32_t byte) {
    if constexpr (E4M3) {
        __nv_fp8_e4m3 x;
        x.__x = (__nv_fp8_storage_t)byte;
        return (float)x;
    } else {
        return (float)(int8_t)byte;
    }
}

// Sequence of grid row b: its new tokens' rows [start, start + n), the tokens before them.  false: nothing to do (or a
// table entry that cannot be, which raises FIRST_FLAG_BAD_SEQ_TABLE).
struct Seq8 {
    int seq, start, n, before;
};
__device__ __forceinline__ bool find_seq(const Seqs8& s, int b, Seq8& q) {
    if (s.m_dev && b >= __ldg(s.m_dev)) return false;
    q.seq = s.idx ? s.idx[b] : b;
    q.start = s.cu ? s.cu[b] : b * s.each;
    const int64_t n = s.cu ? (int64_t)s.cu[b + 1] - q.start : s.each;
    q.before = s.len[q.seq];
    if (n == 0 && q.start >= 0 && q.start <= s.total) return false;
    if (q.start < 0 || n < 0 || q.start + n > s.total || n > s.max_new || q.before < 0 || q.before > 0x7fffffff - n) {
        if (s.flags && threadIdx.x == 0) atomicOr(s.flags, FIRST_FLAG_BAD_SEQ_TABLE);
        return false;
    }
    q.n = (int)n;
    return true;
}

// Page i of a sequence, -1 where it has none; ids outside the cache raise FIRST_FLAG_BAD_PAGE.
__device__ __forceinline__ int raw_page(const Seqs8& s, int seq, int64_t i) {
    return i < s.width ? s.pages[(int64_t)seq * s.width + i] : -1;
}
__device__ __forceinline__ int check_page(const Seqs8& s, int n_pages, int p) {
    if (p < -1 || p >= n_pages) {
        if (s.flags) atomicOr(s.flags, FIRST_FLAG_BAD_PAGE);
        return -1;
    }
    return p;
}
__device__ __forceinline__ int find_page(const Seqs8& s, int n_pages, int seq, int64_t i) {
    return check_page(s, n_pages, raw_page(s, seq, i));
}

}  // namespace first
