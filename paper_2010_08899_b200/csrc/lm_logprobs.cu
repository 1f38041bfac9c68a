// Log-probabilities of given tokens, entropy and the most likely columns of rows of logits; and their gradient.
#include "lm_rows.cuh"

namespace dct {
namespace {

constexpr uint32_t kLpThreads = 256u;

// The k best columns of a row as (order key << 32 | ~column): larger is better, and all are distinct.
template <typename T>
__device__ void row_top_exact(const T* xr, uint32_t vocab, uint32_t k, uint64_t* keys, uint32_t* scratch,
                              uint32_t* counter) {
    // the largest key that at least k columns reach
    uint32_t lo = 0, hi = 0xFFFFFFFFu;
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2 + 1;
        uint32_t n = 0;
        for (uint32_t j = threadIdx.x; j < vocab; j += kLpThreads) n += order_key(to_f32(xr[j])) >= mid;
        if (cta_count(n, scratch) >= k) lo = mid;
        else hi = mid - 1;
    }
    // fewer than k columns are above it ...
    if (threadIdx.x == 0) *counter = 0;
    __syncthreads();
    for (uint32_t j = threadIdx.x; j < vocab; j += kLpThreads) {
        const uint32_t key = order_key(to_f32(xr[j]));
        if (key > lo) keys[atomicAdd(counter, 1u)] = static_cast<uint64_t>(key) << 32 | (0xFFFFFFFFu - j);
    }
    __syncthreads();
    // ... and the lowest columns that equal it fill up
    uint32_t have = *counter;
    for (uint32_t j0 = 0; j0 < vocab && have < k; j0 += kLpThreads) {
        const uint32_t j = j0 + threadIdx.x;
        const bool hit = j < vocab && order_key(to_f32(xr[j])) == lo;
        const uint32_t ballot = __ballot_sync(0xFFFFFFFFu, hit);
        __syncthreads();
        if (lane_id() == 0) scratch[threadIdx.x >> 5] = __popc(ballot);
        __syncthreads();
        uint32_t before = 0, all = 0;
        for (uint32_t w = 0; w < kLpThreads / 32; ++w) {
            if (w < (threadIdx.x >> 5)) before += scratch[w];
            all += scratch[w];
        }
        const uint32_t at = have + before + __popc(ballot & lanemask_lt());
        if (hit && at < k) keys[at] = static_cast<uint64_t>(lo) << 32 | (0xFFFFFFFFu - j);
        have += all;
    }
    __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(kLpThreads)
lm_logprobs_kernel(const T* __restrict__ logits, uint32_t rows, uint32_t vocab, uint32_t ld, float inv_t,
                   const int32_t* __restrict__ tokens, uint32_t top, float* __restrict__ logprob_out,
                   float* __restrict__ entropy_out, float* __restrict__ stats_out, int32_t* __restrict__ top_ids,
                   float* __restrict__ top_logprobs, dct_result_t* __restrict__ result) {
    __shared__ float scratch[32];
    __shared__ uint32_t counts[32], counter;
    __shared__ uint64_t keys[DCT_LM_MAX_TOP];
    for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T* xr = logits + static_cast<size_t>(row) * ld;
        float best = minus_inf();
        for (uint32_t j = threadIdx.x; j < vocab; j += kLpThreads) best = fmaxf(best, to_f32(xr[j]));
        const float m = cta_join<MaxOp>(best, scratch) * inv_t;
        const float ref = m == minus_inf() ? 0.0f : m;
        float s = 0.0f, st = 0.0f;
        for (uint32_t j = threadIdx.x; j < vocab; j += kLpThreads) {
            const float t = fmaf(to_f32(xr[j]), inv_t, -ref);
            const float e = expf(t);
            s += e;
            if (e != 0.0f) st = fmaf(e, t, st);
        }
        s = cta_join<SumOp>(s, scratch);
        st = cta_join<SumOp>(st, scratch);
        const bool empty = m == minus_inf() && s == 0.0f;
        const float logsum = empty ? 0.0f : logf(s);
        if (threadIdx.x == 0) {
            if (tokens) {
                const int32_t tok = tokens[row];
                float lp = 0.0f;
                if (tok >= 0 && static_cast<uint32_t>(tok) < vocab) lp = fmaf(to_f32(xr[tok]), inv_t, -ref) - logsum;
                else if (tok >= 0 && result) atomicMax(&result->status, static_cast<uint32_t>(DCT_ERR_BAD_MASK));
                logprob_out[row] = lp;
            }
            if (entropy_out) entropy_out[row] = empty ? 0.0f : logsum - st / s;
            if (stats_out) {
                stats_out[2 * static_cast<size_t>(row)] = m;
                stats_out[2 * static_cast<size_t>(row) + 1] = logsum;
            }
        }
        if (top == 0) continue;
        row_top_exact(xr, vocab, top, keys, counts, &counter);
        for (uint32_t i = threadIdx.x; i < top; i += kLpThreads) {
            const uint64_t key = keys[i];
            uint32_t rank = 0;
            for (uint32_t q = 0; q < top; ++q) rank += keys[q] > key;
            const uint32_t col = 0xFFFFFFFFu - static_cast<uint32_t>(key);
            const size_t at = static_cast<size_t>(row) * top + rank;
            top_ids[at] = static_cast<int32_t>(col);
            top_logprobs[at] = fmaf(to_f32(xr[col]), inv_t, -ref) - logsum;
        }
        __syncthreads();
    }
}

template <typename T>
__global__ void __launch_bounds__(kLpThreads)
lm_logprobs_bwd_kernel(const T* logits, uint32_t rows, uint32_t vocab, uint32_t ld, float inv_t,
                       const int32_t* __restrict__ tokens, const float* __restrict__ stats,
                       const float* __restrict__ entropy, const float* __restrict__ grad_logprob,
                       const float* __restrict__ grad_entropy, T* grad, uint32_t ld_grad) {
    for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T* xr = logits + static_cast<size_t>(row) * ld;
        T* out = grad + static_cast<size_t>(row) * ld_grad;
        const float m = stats[2 * static_cast<size_t>(row)], logsum = stats[2 * static_cast<size_t>(row) + 1];
        const bool empty = m == minus_inf();
        const float ref = empty ? 0.0f : m;
        const int32_t tok = grad_logprob ? tokens[row] : -1;
        const bool asked = tok >= 0 && static_cast<uint32_t>(tok) < vocab && !empty;
        const float a = asked ? grad_logprob[row] : 0.0f;
        const float c = grad_entropy ? grad_entropy[row] : 0.0f, h = grad_entropy ? entropy[row] : 0.0f;
        for (uint32_t j = threadIdx.x; j < vocab; j += kLpThreads) {
            const float lp = fmaf(to_f32(xr[j]), inv_t, -ref) - logsum;
            const float p = expf(lp);
            float g = -a * p;
            if (p != 0.0f) g = fmaf(-c * p, lp + h, g);
            if (asked && j == static_cast<uint32_t>(tok)) g += a;
            out[j] = from_f32<T>(g * inv_t);
        }
    }
}

bool refused_logits(const void* logits, dct_dtype_t dtype, uint32_t vocab, uint32_t ld, float inv_t) {
    return vocab == 0 || vocab > DCT_LM_MAX_VOCAB || ld < vocab || !usable_temperature(inv_t) ||
           !aligned_to(logits, element_size(dtype));
}

}  // namespace
}  // namespace dct

using namespace dct;

extern "C" dct_status_t dct_lm_logprobs_fwd(const void* logits, dct_dtype_t dtype, uint32_t rows, uint32_t vocab,
                                            uint32_t ld, float inv_temperature, const int32_t* tokens, uint32_t top,
                                            float* logprob_out, float* entropy_out, float* stats_out, int32_t* top_ids,
                                            float* top_logprobs, dct_result_t* result, dct_stream_t stream_) {
    if (!known_dtype(dtype)) return DCT_ERR_UNSUPPORTED;
    if (refused_logits(logits, dtype, vocab, ld, inv_temperature) || top > vocab || top > DCT_LM_MAX_TOP ||
        !aligned_to(result, 8))
        return DCT_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (rows != 0) {
        if (!logits || (tokens != nullptr) != (logprob_out != nullptr) || (top && (!top_ids || !top_logprobs)) ||
            !aligned_to(tokens, 4) || !aligned_to(logprob_out, 4) || !aligned_to(entropy_out, 4) ||
            !aligned_to(stats_out, 4) || (top && (!aligned_to(top_ids, 4) || !aligned_to(top_logprobs, 4))))
            return DCT_ERR_INVALID_ARG;
    }
    if (result) DCT_CUDA_TRY(cudaMemsetAsync(result, 0, sizeof(dct_result_t), stream));
    if (rows == 0) return DCT_OK;
    const uint32_t grid = rows < 4096u ? rows : 4096u;
    if (dtype == DCT_F32)
        lm_logprobs_kernel<float><<<grid, kLpThreads, 0, stream>>>(
            static_cast<const float*>(logits), rows, vocab, ld, inv_temperature, tokens, top, logprob_out, entropy_out,
            stats_out, top_ids, top_logprobs, result);
    else
        lm_logprobs_kernel<__nv_bfloat16><<<grid, kLpThreads, 0, stream>>>(
            static_cast<const __nv_bfloat16*>(logits), rows, vocab, ld, inv_temperature, tokens, top, logprob_out,
            entropy_out, stats_out, top_ids, top_logprobs, result);
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}

extern "C" dct_status_t dct_lm_logprobs_bwd(const void* logits, dct_dtype_t dtype, uint32_t rows, uint32_t vocab,
                                            uint32_t ld, float inv_temperature, const int32_t* tokens,
                                            const float* stats, const float* entropy, const float* grad_logprob,
                                            const float* grad_entropy, void* grad_logits, uint32_t ld_grad,
                                            dct_stream_t stream_) {
    if (!known_dtype(dtype)) return DCT_ERR_UNSUPPORTED;
    if (refused_logits(logits, dtype, vocab, ld, inv_temperature) || ld_grad < vocab) return DCT_ERR_INVALID_ARG;
    if (rows == 0) return DCT_OK;
    const size_t es = element_size(dtype);
    if (!logits || !stats || !grad_logits || (grad_logprob && !tokens) || (grad_entropy && !entropy) ||
        !aligned_to(grad_logits, es) || !aligned_to(tokens, 4) || !aligned_to(stats, 4) || !aligned_to(entropy, 4) ||
        !aligned_to(grad_logprob, 4) || !aligned_to(grad_entropy, 4) ||
        !in_place_or_apart(logits, ld, grad_logits, ld_grad, rows, vocab, es))
        return DCT_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const uint32_t grid = rows < 4096u ? rows : 4096u;
    if (dtype == DCT_F32)
        lm_logprobs_bwd_kernel<float><<<grid, kLpThreads, 0, stream>>>(
            static_cast<const float*>(logits), rows, vocab, ld, inv_temperature, tokens, stats, entropy, grad_logprob,
            grad_entropy, static_cast<float*>(grad_logits), ld_grad);
    else
        lm_logprobs_bwd_kernel<__nv_bfloat16><<<grid, kLpThreads, 0, stream>>>(
            static_cast<const __nv_bfloat16*>(logits), rows, vocab, ld, inv_temperature, tokens, stats, entropy,
            grad_logprob, grad_entropy, static_cast<__nv_bfloat16*>(grad_logits), ld_grad);
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}
