// Host-side launch interfaces of the operators that serve both a standalone entry point and the step: low-rank
// adapters (lora.cu) and per-request sampling (sample.cu).  Arguments are checked by the callers.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

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

}  // namespace first
