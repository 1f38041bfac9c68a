// Distillation from a teacher's top log-probabilities: loss and gradient of rows of logits.
#include "lm_rows.cuh"

namespace dct {
namespace {

constexpr uint32_t kDsThreads = 256u;

template <typename T, bool kTail>
__global__ void __launch_bounds__(kDsThreads)
lm_distill_kernel(const T* logits, uint32_t rows, uint32_t vocab, uint32_t ld, float inv_t,
                  const int32_t* __restrict__ teacher_ids, const float* __restrict__ teacher_lp, uint32_t top,
                  const float* __restrict__ grad_loss, float* __restrict__ loss_out, T* grad, uint32_t ld_grad,
                  dct_result_t* __restrict__ result) {
    extern __shared__ uint32_t named[];                    // one bit per column: some slot names it
    __shared__ float scratch[32];
    __shared__ int32_t ids[DCT_LM_MAX_TEACHER_TOP];
    __shared__ float q[DCT_LM_MAX_TEACHER_TOP], t_s[DCT_LM_MAX_TEACHER_TOP], z_s[DCT_LM_MAX_TEACHER_TOP];
    const uint32_t words = (vocab + 31) / 32;
    for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T* xr = logits + static_cast<size_t>(row) * ld;
        __syncthreads();
        for (uint32_t w = threadIdx.x; w < words; w += kDsThreads) named[w] = 0;
        __syncthreads();
        float best_t = minus_inf();
        bool bad = false, broken = false;
        for (uint32_t i = threadIdx.x; i < top; i += kDsThreads) {
            int32_t id = teacher_ids[static_cast<size_t>(row) * top + i];
            float t = teacher_lp[static_cast<size_t>(row) * top + i];
            bad |= id >= 0 && static_cast<uint32_t>(id) >= vocab;
            if (id < 0 || static_cast<uint32_t>(id) >= vocab) {
                id = -1;
                t = minus_inf();
            } else {
                atomicOr(&named[id >> 5], 1u << (id & 31));
                z_s[i] = to_f32(xr[id]);
            }
            broken |= t != t;
            ids[i] = id;
            t_s[i] = t;
            best_t = fmaxf(best_t, t);
        }
        if (bad && result) atomicMax(&result->status, static_cast<uint32_t>(DCT_ERR_BAD_MASK));
        best_t = cta_join<MaxOp>(best_t, scratch);
        broken = __syncthreads_or(broken);
        const bool no_teacher = best_t == minus_inf() && !broken;
        // the teacher's side: log q = t - log_norm
        float log_norm = 0.0f;
        if (!kTail && !no_teacher) {
            float s = 0.0f;
            for (uint32_t i = threadIdx.x; i < top; i += kDsThreads) s += expf(t_s[i] - best_t);
            log_norm = best_t + logf(cta_join<SumOp>(s, scratch));
        }
        float q_sum = 0.0f;
        for (uint32_t i = threadIdx.x; i < top; i += kDsThreads) {
            q[i] = expf(t_s[i] - log_norm);
            q_sum += q[i];
        }
        q_sum = cta_join<SumOp>(q_sum, scratch);
        const float q_r = kTail ? (q_sum > 1.0f ? 0.0f : 1.0f - q_sum) : 0.0f;

        // the student's side
        float best = minus_inf();
        for (uint32_t j = threadIdx.x; j < vocab; j += kDsThreads) best = fmaxf(best, to_f32(xr[j]));
        best = cta_join<MaxOp>(best, scratch) * inv_t;
        const float ref = best == minus_inf() ? 0.0f : best;
        float s = 0.0f, s_rest = 0.0f;
        for (uint32_t j = threadIdx.x; j < vocab; j += kDsThreads) {
            const float e = expf(fmaf(to_f32(xr[j]), inv_t, -ref));
            s += e;
            if (kTail && !(named[j >> 5] >> (j & 31) & 1u)) s_rest += e;
        }
        s = cta_join<SumOp>(s, scratch);
        if (kTail) s_rest = cta_join<SumOp>(s_rest, scratch);
        const bool nothing = (best == minus_inf() && s == 0.0f) || (!kTail && no_teacher);
        broken |= s != s;
        const float nan = __uint_as_float(0x7FFFFFFFu);
        const float logsum = logf(s), log_rest = logf(s_rest);
        float loss = 0.0f;
        for (uint32_t i = threadIdx.x; i < top; i += kDsThreads)
            if (q[i] != 0.0f && ids[i] >= 0)
                loss += q[i] * (t_s[i] - log_norm - (fmaf(z_s[i], inv_t, -ref) - logsum));
        loss = cta_join<SumOp>(loss, scratch);
        if (kTail && q_r != 0.0f && s_rest != 0.0f) loss += q_r * (logf(q_r) - (log_rest - logsum));
        if (broken) loss = nan;
        if (nothing) loss = 0.0f;
        if (loss_out && threadIdx.x == 0) loss_out[row] = loss;
        if (!grad) continue;

        T* out = grad + static_cast<size_t>(row) * ld_grad;
        const float scale = broken ? nan : (grad_loss ? grad_loss[row] : 1.0f) * inv_t;
        const float p_r = kTail ? s_rest / s : 0.0f;
        __syncthreads();                                   // (in place: every z_s is taken)
        for (uint32_t j = threadIdx.x; j < vocab; j += kDsThreads) {
            const float t = fmaf(to_f32(xr[j]), inv_t, -ref);
            float g;
            if (kTail) g = s_rest == 0.0f ? 0.0f : expf(t - log_rest) * (p_r - q_r);
            else g = expf(t - logsum);
            out[j] = from_f32<T>(nothing ? 0.0f : g * scale);
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < top; i += kDsThreads) {
            const int32_t id = ids[i];
            if (id < 0 || nothing) continue;
            float mass = 0.0f;
            bool first = true;
            for (uint32_t k = 0; k < top; ++k)
                if (ids[k] == id) {
                    first &= k >= i;
                    mass += q[k];
                }
            if (first) out[id] = from_f32<T>((expf(fmaf(z_s[i], inv_t, -ref) - logsum) - mass) * scale);
        }
    }
}

template <typename T, bool kTail>
dct_status_t launch_distill(const void* logits, uint32_t rows, uint32_t vocab, uint32_t ld, float inv_t,
                            const int32_t* ids, const float* lps, uint32_t top, const float* grad_loss, float* loss_out,
                            void* grad, uint32_t ld_grad, dct_result_t* result, cudaStream_t stream) {
    auto kernel = lm_distill_kernel<T, kTail>;
    const size_t smem = (vocab + 31) / 32 * 4;
    if (smem > 16 * 1024)
        DCT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
    const uint32_t grid = rows < 4096u ? rows : 4096u;
    kernel<<<grid, kDsThreads, smem, stream>>>(static_cast<const T*>(logits), rows, vocab, ld, inv_t, ids, lps, top,
                                               grad_loss, loss_out, static_cast<T*>(grad), ld_grad, result);
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}

}  // namespace
}  // namespace dct

using namespace dct;

extern "C" dct_status_t dct_lm_distill(const void* logits, dct_dtype_t dtype, uint32_t rows, uint32_t vocab, uint32_t ld,
                                       float inv_temperature, const int32_t* teacher_ids, const float* teacher_logprobs,
                                       uint32_t top, dct_distill_mode_t mode, const float* grad_loss, float* loss_out,
                                       void* grad_logits, uint32_t ld_grad, dct_result_t* result,
                                       dct_stream_t stream_) {
    if (!known_dtype(dtype) || (mode != DCT_DISTILL_RENORM && mode != DCT_DISTILL_TAIL)) return DCT_ERR_UNSUPPORTED;
    const size_t es = element_size(dtype);
    if (vocab == 0 || vocab > DCT_LM_MAX_VOCAB || ld < vocab || !usable_temperature(inv_temperature) || top == 0 ||
        top > DCT_LM_MAX_TEACHER_TOP || !aligned_to(logits, es) || !aligned_to(result, 8))
        return DCT_ERR_INVALID_ARG;
    if (rows != 0) {
        if (!logits || !teacher_ids || !teacher_logprobs || (!loss_out && !grad_logits) || !aligned_to(teacher_ids, 4) ||
            !aligned_to(teacher_logprobs, 4) || !aligned_to(grad_loss, 4) || !aligned_to(loss_out, 4))
            return DCT_ERR_INVALID_ARG;
        if (grad_logits && (ld_grad < vocab || !aligned_to(grad_logits, es) ||
                            !in_place_or_apart(logits, ld, grad_logits, ld_grad, rows, vocab, es)))
            return DCT_ERR_INVALID_ARG;
    }
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (result) DCT_CUDA_TRY(cudaMemsetAsync(result, 0, sizeof(dct_result_t), stream));
    if (rows == 0) return DCT_OK;
    auto launch = dtype == DCT_F32
        ? (mode == DCT_DISTILL_TAIL ? launch_distill<float, true> : launch_distill<float, false>)
        : (mode == DCT_DISTILL_TAIL ? launch_distill<__nv_bfloat16, true> : launch_distill<__nv_bfloat16, false>);
    return launch(logits, rows, vocab, ld, inv_temperature, teacher_ids, teacher_logprobs, top, grad_loss, loss_out,
                  grad_logits, ld_grad, result, stream);
}
