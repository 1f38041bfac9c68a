// Layer norm forward and backward.
#include "lm_rows.cuh"

namespace dct {
namespace {

constexpr uint32_t kNormMaxWidth = 65536u;
constexpr uint32_t kNormThreads = 256u;
constexpr uint32_t kNormMaxParts = 592u;

template <typename T, typename P>
__global__ void __launch_bounds__(kNormThreads)
norm_fwd_kernel(const T* __restrict__ x, uint32_t rows, uint32_t d, uint32_t ld, const P* __restrict__ weight,
                const P* __restrict__ bias, float eps, T* y, uint32_t ld_y, float* __restrict__ mean_out,
                float* __restrict__ rstd_out) {
    __shared__ float scratch[32];
    for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T* xr = x + static_cast<size_t>(row) * ld;
        float sum = 0.0f;
        for (uint32_t j = threadIdx.x; j < d; j += kNormThreads) sum += to_f32(xr[j]);
        const float mean = cta_join<SumOp>(sum, scratch) / static_cast<float>(d);
        float sq = 0.0f;
        for (uint32_t j = threadIdx.x; j < d; j += kNormThreads) {
            const float c = to_f32(xr[j]) - mean;
            sq = fmaf(c, c, sq);
        }
        const float rstd = 1.0f / sqrtf(cta_join<SumOp>(sq, scratch) / static_cast<float>(d) + eps);
        T* yr = y + static_cast<size_t>(row) * ld_y;
        for (uint32_t j = threadIdx.x; j < d; j += kNormThreads) {
            const float w = weight ? to_f32(weight[j]) : 1.0f, b = bias ? to_f32(bias[j]) : 0.0f;
            yr[j] = from_f32<T>(fmaf((to_f32(xr[j]) - mean) * rstd, w, b));
        }
        if (threadIdx.x == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
}

// partial sums of the parameter gradients: CTA (c, part) adds the rows part, part + parts, ... of 256 columns
template <typename T>
__global__ void __launch_bounds__(kNormThreads)
norm_param_parts_kernel(const T* __restrict__ dy, uint32_t ld_dy, const T* __restrict__ x, uint32_t rows, uint32_t d,
                        uint32_t ld, const float* __restrict__ mean, const float* __restrict__ rstd,
                        float* __restrict__ parts) {
    const uint32_t j = blockIdx.x * kNormThreads + threadIdx.x;
    if (j >= d) return;
    float dw = 0.0f, db = 0.0f;
    for (uint32_t row = blockIdx.y; row < rows; row += gridDim.y) {
        const float g = to_f32(dy[static_cast<size_t>(row) * ld_dy + j]);
        const float h = (to_f32(x[static_cast<size_t>(row) * ld + j]) - mean[row]) * rstd[row];
        dw = fmaf(g, h, dw);
        db += g;
    }
    float* p = parts + static_cast<size_t>(blockIdx.y) * 2 * d;
    p[j] = dw;
    p[d + j] = db;
}

__global__ void __launch_bounds__(kNormThreads)
norm_param_sum_kernel(const float* __restrict__ parts, uint32_t num, uint32_t d, float* __restrict__ dweight,
                      float* __restrict__ dbias) {
    const uint32_t j = blockIdx.x * kNormThreads + threadIdx.x;
    if (j >= d) return;
    float dw = 0.0f, db = 0.0f;
    for (uint32_t i = 0; i < num; ++i) {
        dw += parts[static_cast<size_t>(i) * 2 * d + j];
        db += parts[static_cast<size_t>(i) * 2 * d + d + j];
    }
    if (dweight) dweight[j] = dw;
    if (dbias) dbias[j] = db;
}

template <typename T, typename P>
__global__ void __launch_bounds__(kNormThreads)
norm_bwd_kernel(const T* dy, uint32_t ld_dy, const T* x, uint32_t rows, uint32_t d, uint32_t ld,
                const P* __restrict__ weight, const float* __restrict__ mean, const float* __restrict__ rstd, T* dx,
                uint32_t ld_dx) {
    __shared__ float scratch[32];
    for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T* xr = x + static_cast<size_t>(row) * ld;
        const T* gr = dy + static_cast<size_t>(row) * ld_dy;
        T* out = dx + static_cast<size_t>(row) * ld_dx;
        const float mu = mean[row], r = rstd[row];
        float s1 = 0.0f, s2 = 0.0f;
        for (uint32_t j = threadIdx.x; j < d; j += kNormThreads) {
            const float g = to_f32(gr[j]) * (weight ? to_f32(weight[j]) : 1.0f);
            s1 += g;
            s2 = fmaf(g, (to_f32(xr[j]) - mu) * r, s2);
        }
        const float m1 = cta_join<SumOp>(s1, scratch) / static_cast<float>(d);
        const float m2 = cta_join<SumOp>(s2, scratch) / static_cast<float>(d);
        for (uint32_t j = threadIdx.x; j < d; j += kNormThreads) {
            const float g = to_f32(gr[j]) * (weight ? to_f32(weight[j]) : 1.0f);
            out[j] = from_f32<T>(r * (g - m1 - (to_f32(xr[j]) - mu) * r * m2));
        }
    }
}

uint32_t norm_parts(uint32_t rows) { return rows < kNormMaxParts ? (rows ? rows : 1) : kNormMaxParts; }

template <typename T, typename P>
dct_status_t launch_norm_fwd(const void* x, uint32_t rows, uint32_t d, uint32_t ld, const void* weight, const void* bias,
                             float eps, void* y, uint32_t ld_y, float* mean_out, float* rstd_out, cudaStream_t stream) {
    const uint32_t grid = rows < 4096u ? rows : 4096u;
    norm_fwd_kernel<T, P><<<grid, kNormThreads, 0, stream>>>(static_cast<const T*>(x), rows, d, ld,
                                                             static_cast<const P*>(weight), static_cast<const P*>(bias),
                                                             eps, static_cast<T*>(y), ld_y, mean_out, rstd_out);
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}

template <typename T, typename P>
dct_status_t launch_norm_bwd(const void* dy, uint32_t ld_dy, const void* x, uint32_t rows, uint32_t d, uint32_t ld,
                             const void* weight, const float* mean, const float* rstd, void* dx, uint32_t ld_dx,
                             float* dweight, float* dbias, float* parts, cudaStream_t stream) {
    if (dweight || dbias) {        // before dx, which may take the place of dy or x
        const uint32_t cols = (d + kNormThreads - 1) / kNormThreads, num = norm_parts(rows);
        norm_param_parts_kernel<T><<<dim3(cols, num), kNormThreads, 0, stream>>>(
            static_cast<const T*>(dy), ld_dy, static_cast<const T*>(x), rows, d, ld, mean, rstd, parts);
        DCT_CUDA_TRY(cudaGetLastError());
        norm_param_sum_kernel<<<cols, kNormThreads, 0, stream>>>(parts, num, d, dweight, dbias);
        DCT_CUDA_TRY(cudaGetLastError());
    }
    const uint32_t grid = rows < 4096u ? rows : 4096u;
    norm_bwd_kernel<T, P><<<grid, kNormThreads, 0, stream>>>(static_cast<const T*>(dy), ld_dy, static_cast<const T*>(x),
                                                             rows, d, ld, static_cast<const P*>(weight), mean, rstd,
                                                             static_cast<T*>(dx), ld_dx);
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}

bool refused_parameter(const void* p, dct_dtype_t t, uint32_t d, const void* out, size_t out_bytes) {
    return p && (!aligned_to(p, element_size(t)) || spans_overlap(p, d * element_size(t), out, out_bytes));
}

}  // namespace
}  // namespace dct

using namespace dct;

extern "C" dct_status_t dct_layer_norm_fwd(const void* x, dct_dtype_t dtype, uint32_t rows, uint32_t d, uint32_t ld,
                                           const void* weight, const void* bias, dct_dtype_t param_dtype, float eps,
                                           void* y, uint32_t ld_y, float* mean_out, float* rstd_out,
                                           dct_stream_t stream_) {
    if (!known_dtype(dtype) || !known_dtype(param_dtype)) return DCT_ERR_UNSUPPORTED;
    if (d == 0 || d > kNormMaxWidth || ld < d || ld_y < d || !std::isfinite(eps) || eps < 0.0f) return DCT_ERR_INVALID_ARG;
    if (rows == 0) return DCT_OK;
    if (!x || !y) return DCT_ERR_INVALID_ARG;
    const size_t es = element_size(dtype), out_bytes = span_bytes(rows, d, ld_y, es);
    if (!aligned_to(x, es) || !aligned_to(y, es) || !aligned_to(mean_out, 4) || !aligned_to(rstd_out, 4) ||
        !in_place_or_apart(x, ld, y, ld_y, rows, d, es) || refused_parameter(weight, param_dtype, d, y, out_bytes) ||
        refused_parameter(bias, param_dtype, d, y, out_bytes))
        return DCT_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    auto launch = dtype == DCT_F32
        ? (param_dtype == DCT_F32 ? launch_norm_fwd<float, float> : launch_norm_fwd<float, __nv_bfloat16>)
        : (param_dtype == DCT_F32 ? launch_norm_fwd<__nv_bfloat16, float> : launch_norm_fwd<__nv_bfloat16, __nv_bfloat16>);
    return launch(x, rows, d, ld, weight, bias, eps, y, ld_y, mean_out, rstd_out, stream);
}

extern "C" size_t dct_layer_norm_bwd_workspace_bytes(uint32_t rows, uint32_t d) {
    if (d == 0 || d > kNormMaxWidth) return 0;
    return (static_cast<size_t>(norm_parts(rows)) * 2 * d * sizeof(float) + 255) & ~static_cast<size_t>(255);
}

extern "C" dct_status_t dct_layer_norm_bwd(const void* dy, uint32_t ld_dy, const void* x, dct_dtype_t dtype,
                                           uint32_t rows, uint32_t d, uint32_t ld, const void* weight,
                                           dct_dtype_t param_dtype, const float* mean, const float* rstd, void* dx,
                                           uint32_t ld_dx, float* dweight, float* dbias, void* workspace,
                                           size_t workspace_bytes, dct_stream_t stream_) {
    if (!known_dtype(dtype) || !known_dtype(param_dtype)) return DCT_ERR_UNSUPPORTED;
    if (d == 0 || d > kNormMaxWidth || ld < d || ld_dy < d || ld_dx < d) return DCT_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (!aligned_to(dweight, 4) || !aligned_to(dbias, 4)) return DCT_ERR_INVALID_ARG;
    if (rows == 0) {
        if (dweight) DCT_CUDA_TRY(cudaMemsetAsync(dweight, 0, d * sizeof(float), stream));
        if (dbias) DCT_CUDA_TRY(cudaMemsetAsync(dbias, 0, d * sizeof(float), stream));
        return DCT_OK;
    }
    if (!dy || !x || !mean || !rstd || !dx) return DCT_ERR_INVALID_ARG;
    const size_t es = element_size(dtype);
    if (!aligned_to(dy, es) || !aligned_to(x, es) || !aligned_to(dx, es) || !aligned_to(mean, 4) || !aligned_to(rstd, 4) ||
        !in_place_or_apart(dy, ld_dy, dx, ld_dx, rows, d, es) || !in_place_or_apart(x, ld, dx, ld_dx, rows, d, es) ||
        refused_parameter(weight, param_dtype, d, dx, span_bytes(rows, d, ld_dx, es)))
        return DCT_ERR_INVALID_ARG;
    if ((dweight || dbias) && (!workspace || !aligned_to(workspace, 256) ||
                               workspace_bytes < dct_layer_norm_bwd_workspace_bytes(rows, d)))
        return DCT_ERR_WORKSPACE;
    float* parts = static_cast<float*>(workspace);
    auto launch = dtype == DCT_F32
        ? (param_dtype == DCT_F32 ? launch_norm_bwd<float, float> : launch_norm_bwd<float, __nv_bfloat16>)
        : (param_dtype == DCT_F32 ? launch_norm_bwd<__nv_bfloat16, float> : launch_norm_bwd<__nv_bfloat16, __nv_bfloat16>);
    return launch(dy, ld_dy, x, rows, d, ld, weight, mean, rstd, dx, ld_dx, dweight, dbias, parts, stream);
}
