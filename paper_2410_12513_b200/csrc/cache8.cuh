// Device helpers of the paged 8-bit cache: its values, sequences and their pages.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"
#include "first.h"
#include "ops.h"

namespace first {

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
