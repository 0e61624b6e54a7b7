// Host-side launch interfaces of the operators that serve both a standalone entry point and the step: low-rank
// adapters (lora.cu), per-request sampling (sample.cu) and the paged 8-bit cache (append8.cu, attn8.cu).  Arguments are checked by the callers.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <initializer_list>

#include "first.h"

namespace first {

constexpr int kSMs = 148;  // of a B200; for rules on grid sizes in calls without a context
constexpr int kLoraMaxSegments = 4, kLoraMaxRank = 128;

enum LoraX { kLoraXF32 = 0, kLoraXBf16 = 1, kLoraXPair = 2 };  // kLoraXPair: bfloat16 hi + lo halves (x = hi + lo)

// y[row(i)][f] += scale[a] * sum_j B[a][f][j] * (sum_k A[a][seg(f)*R + j][k] * x[i][k]),  a = adapter[seq(i)],
// i < m; seq(i) = idx ? idx[i] : i; row(i) = scatter ? seq(i) : i.  Rows whose adapter is outside [0, n) are left alone.
struct LoraArgs {
    const void *x = nullptr, *x_lo = nullptr;
    int x_kind = kLoraXF32;
    int64_t ldx = 0;
    const void *a = nullptr, *b = nullptr;  // [n][S*R][K], [n][N][R]
    bool w_f32 = false;
    const float* scales = nullptr;          // [n] or NULL (= 1)
    const int32_t* adapter = nullptr;
    int n = 0, S = 1, R = 0, K = 0, N = 0;
    int seg[kLoraMaxSegments + 1] = {};     // borders of the output segments, seg[0] = 0, seg[S] = N
    void* y = nullptr;
    bool y_f32 = true;
    int64_t ldy = 0;
    const int32_t* idx = nullptr;
    bool scatter = false;
    int m = 0;
    const int32_t* m_dev = nullptr;
    int row0 = 0;                           // (set by lora_launch: rows before this piece, for m_dev)
    uint64_t* stamp = nullptr;
};
cudaError_t lora_launch(const LoraArgs& a, cudaStream_t st, bool pdl, int n_sm);

struct SampleArgs {
    const float* logits = nullptr;
    int64_t ld = 0;
    int B = 0, V = 0;
    const float *temperature = nullptr, *top_p = nullptr, *min_p = nullptr, *u = nullptr;  // [B], any but u NULL
    const int32_t* top_k = nullptr;
    int32_t* tokens = nullptr;
    int32_t* pos = nullptr;  // += 1 per row, or NULL
    int move_max = 0;        // (set by sample_launch) so many candidates are left to one CTA
    uint64_t* stamp = nullptr;
};
constexpr int kSampleMaxVocab = 1 << 19;
cudaError_t sample_launch(const SampleArgs& a, cudaStream_t st, bool pdl);

// A kernel's limits are a device's: sets its dynamic shared memory (and clusters of more than 8 CTAs) on the current device, once each.  `done`:
// a bit a device, static beside the kernel.
template <typename K>
cudaError_t allow_launch(K kern, int smem, bool large_clusters, std::atomic<uint64_t>& done) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load(std::memory_order_acquire) & bit)) return cudaSuccess;
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess && large_clusters) e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
    return e;
}

// One layer of a paged 8-bit cache: pages of 2^shift tokens, [n_pages][H][2^shift][hd] bytes, one scale a (page, head).
struct Cache8 {
    uint8_t *k = nullptr, *v = nullptr;
    float *ks = nullptr, *vs = nullptr;
    int n_pages = 0, H = 0, shift = 0, hd = 0;
    bool e4m3 = false;
};
// Sequences over it.  New token i of sequence b is row cu[b] + i of the caller's tensors (cu NULL: row r is the one new
// token of sequence idx ? idx[r] : r) and has position len[b] + i.  m_dev: live rows, as in the step's kernels.
struct Seqs8 {
    const int32_t* pages = nullptr;  // [.][width], -1 = no page
    int64_t width = 0;
    const int32_t *len = nullptr, *cu = nullptr;
    int B = 0, total = 0, max_new = 1;
    int each = 1;                    // without cu: new tokens of every sequence
    const int64_t* row_off = nullptr;  // dev, or NULL: the sequence's rows start that much later (one sequence alone)
    int64_t row_total = 0;           // with it: rows that there are,
    const int32_t* row_cap = nullptr;  // dev, or NULL: of them the sequence's own
    const int32_t *idx = nullptr, *m_dev = nullptr;
    uint32_t* flags = nullptr;       // or NULL
    const float2* cs = nullptr;      // [.][hd/2] by sequence: rotate q and k on the way (the step), or NULL
    uint64_t* stamp = nullptr;
};
struct Rows8 {                       // a tensor [tokens][heads][hd], strides in elements
    void* p = nullptr;
    int64_t tok = 0, head = 0;
    bool f32 = true;
};
cudaError_t append8_launch(const Cache8& c, const Seqs8& s, const Rows8& k, const Rows8& v, cudaStream_t st, bool pdl);

struct Attn8Args {
    Cache8 c;
    Seqs8 s;
    Rows8 q, out;                    // out.p NULL: out_hi / out_lo instead (the step's bfloat16 pair), out's strides
    __nv_bfloat16 *out_hi = nullptr, *out_lo = nullptr;
    int G = 1;
    float scale = 1.f;
    float *part_o = nullptr, *part_ml = nullptr;  // room for attn8_part_floats: unfinished results, [rows][splits][hd] and [..][2]; or NULL
};
// Floats that a call of these sizes has a use for (0: none); rows: query rows of a KV head.
int64_t attn8_part_floats(int64_t B, int64_t H, int64_t rows, int hd, int64_t longest, bool f32, int n_sm);
cudaError_t attn8_launch(const Attn8Args& a, cudaStream_t st, bool pdl, int n_sm);

// Checks of arguments: FIRST_OK or an error.
inline bool words_ok(std::initializer_list<const void*> arrays) {  // arrays of 32-bit values (NULL is fine) begin at a multiple of their size
    for (const void* p : arrays)
        if (reinterpret_cast<uintptr_t>(p) % 4) return false;
    return true;
}
int check_cache8(const first_cache8* c);
int check_seqs8(const int32_t* pages, int32_t max_pages, const int32_t* len, const int32_t* cu, int32_t B, int32_t total, int32_t max_new,
                const uint32_t* flags);
int check_rows8(const void* p, int64_t tok, int64_t head, int32_t heads, int32_t hd, int32_t dtype, int64_t total, bool written);
Cache8 cache8_of(const first_cache8& c);

}  // namespace first
