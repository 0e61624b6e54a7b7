// Low-rank adapters of many requests beside a shared projection (the paper's "LoRA Compensation Module" keeps one
// adapter merged into the weights; here every row of a batch may have its own):
//   y[r] += scale[a] * B_a (A_a x[r]),  a = adapter of row r.
#include "common.cuh"
#include "first.h"
#include "ops.h"

namespace first {
namespace {

template <typename T>
__device__ __forceinline__ float at(const void* p, int64_t i) { return to_f32(static_cast<const T*>(p)[i]); }

// One block per row: A x into shared memory (one warp per row of A), then one thread per output feature.
template <typename WT, typename YT>
__global__ void __launch_bounds__(256) lora_rows(const LoraArgs p) {
    const Stamp stamp_guard(p.stamp);
    extern __shared__ float h[];  // [S*R]
    pdl_trigger();
    pdl_wait();
    const int i = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (p.m_dev && i >= *p.m_dev) return;
    const int s = p.idx ? p.idx[i] : i, ad = p.adapter[s];
    if (ad < 0 || ad >= p.n) return;
    const int M = p.S * p.R;
    const WT* A = static_cast<const WT*>(p.a) + (int64_t)ad * M * p.K;
    const WT* B = static_cast<const WT*>(p.b) + (int64_t)ad * p.N * p.R;
    for (int j = warp; j < M; j += 8) {
        float acc = 0.f;
        for (int k = lane; k < p.K; k += 32) {
            const int64_t e = (int64_t)i * p.ldx + k;
            float x = p.x_kind == kLoraXF32 ? at<float>(p.x, e) : at<__nv_bfloat16>(p.x, e);
            if (p.x_kind == kLoraXPair) x += at<__nv_bfloat16>(p.x_lo, e);
            acc += x * to_f32(A[(int64_t)j * p.K + k]);
        }
        acc = warp_sum(acc);
        if (lane == 0) h[j] = acc;
    }
    __syncthreads();
    const float sc = p.scales ? p.scales[ad] : 1.f;
    YT* y = static_cast<YT*>(p.y) + (int64_t)(p.scatter ? s : i) * p.ldy;
    for (int f = threadIdx.x; f < p.N; f += 256) {
        int sg = 0;
        while (sg + 1 < p.S && f >= p.seg[sg + 1]) ++sg;
        float acc = 0.f;
        for (int j = 0; j < p.R; ++j) acc += to_f32(B[(int64_t)f * p.R + j]) * h[sg * p.R + j];
        y[f] = from_f32<YT>(to_f32(y[f]) + sc * acc);
    }
}

}  // namespace

cudaError_t lora_launch(const LoraArgs& a, cudaStream_t st, bool pdl, int) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(a.m);
    cfg.blockDim = dim3(256);
    cfg.dynamicSmemBytes = sizeof(float) * a.S * a.R;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl ? 1 : 0;
    auto kern = a.w_f32 ? (a.y_f32 ? lora_rows<float, float> : lora_rows<float, __nv_bfloat16>)
                        : (a.y_f32 ? lora_rows<__nv_bfloat16, float> : lora_rows<__nv_bfloat16, __nv_bfloat16>);
    return cudaLaunchKernelEx(&cfg, kern, a);
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
    return lora_launch(p, static_cast<cudaStream_t>(stream), false, 148) == cudaSuccess ? FIRST_OK : FIRST_E_CUDA;
}
