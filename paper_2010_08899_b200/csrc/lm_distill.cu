// Distillation from a teacher's top log-probabilities: loss and gradient of rows of logits.
#include "lm_rows.cuh"

namespace dct {
namespace {

constexpr uint32_t kMaxCluster = 8u;

struct DistillArgs {
    uint32_t rows, vocab, ld;
    float inv_t, c;                 // 1 / T and log2 e / T
    const int32_t* ids;
    const float* lps;
    uint32_t top;
    const float* grad_loss;
    float* loss_out;
    uint32_t ld_grad, mark_words;
    dct_result_t* result;
};

// xmax, s: the largest of some values and sum exp(value - xmax) over them, to the accuracy of expf
__device__ __forceinline__ void add_value(RowPart& p, float v) {
    if (v > p.xmax) {
        p.s = p.xmax == minus_inf() ? p.s + 1.0f : fmaf(p.s, expf(p.xmax - v), 1.0f);
        p.xmax = v;
    } else if (v != minus_inf()) {            // NaN comes here
        p.s += expf(v - p.xmax);
    }
}

// A row's cluster of CTAs reads its logits twice: for the sums, and, when those are joined, for the gradient; the second time
// they come from L2, as few enough rows are under way.  The teacher's slots of the next row, and the logits that this row's
// slots name, are fetched while the row streams by.  `marks` has a bit for every element of the slice's units that a
// slot names.  kTail: those are left out of the sums, so that the remainder is summed and not a difference.  The gradient is
// first written as if no column were named, and the named ones once more afterwards.
// Slot i belongs to thread i mod kThreads throughout.
template <typename T, uint32_t kThreads, bool kTail, bool kCluster>
__global__ void __launch_bounds__(kThreads, 768 / kThreads)
lm_distill_kernel(const T* logits, T* grad, const DistillArgs a) {
    constexpr uint32_t E = Unit<T>::kElems, kWarps = kThreads / 32;
    extern __shared__ __align__(16) uint32_t dynamic[];
    __shared__ RowPart student_parts[kWarps], teacher_parts[kWarps], named_parts[kWarps], slice_part, slice_named;
    __shared__ float loss_parts[kWarps];
    __shared__ uint32_t repeated_flag;
    uint32_t* const marks = dynamic;
    int32_t* const ids_by_turn = reinterpret_cast<int32_t*>(marks + a.mark_words);       // two rows
    float* const t_by_turn = reinterpret_cast<float*>(ids_by_turn + 2 * a.top);           // two rows
    uint32_t* const z_words = reinterpret_cast<uint32_t*>(t_by_turn + 2 * a.top);
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = lane_id();
    const uint32_t rank = kCluster ? cluster_rank() : 0u, ctas = kCluster ? cluster_size() : 1u;
    const uint32_t clusters = gridDim.x / ctas;

    auto fetch_slots = [&](uint32_t of_row, uint32_t turn) {
        const size_t at = static_cast<size_t>(of_row) * a.top;
        for (uint32_t i = tid; i < a.top; i += kThreads) {
            copy_word_async(ids_by_turn + turn * a.top + i, a.ids + at + i);
            copy_word_async(t_by_turn + turn * a.top + i, a.lps + at + i);
        }
    };
    uint32_t row_id = blockIdx.x / ctas;
    fetch_slots(row_id, 0);
    copy_commit();
    for (uint32_t w = tid; w < a.mark_words; w += kThreads) marks[w] = 0;
    if (tid == 0) repeated_flag = 0;
    for (uint32_t turn = 0;; turn ^= 1) {
        const T* xr = logits + static_cast<size_t>(row_id) * a.ld;
        const RowView<T> row(xr, a.vocab);
        const Slice slice(row.units, rank, ctas);
        const uint32_t u0 = slice.u0, u1 = slice.u1;
        const int32_t* ids = ids_by_turn + turn * a.top;
        const float* t_s = t_by_turn + turn * a.top;
        copy_wait<0>();
        __syncthreads();                                   // the last row's marks are gone, its numbers are read

        auto in_slice = [&](uint32_t i) {
            const uint32_t p = static_cast<uint32_t>(ids[i]) + row.lead;
            return p >= u0 * E && p < u1 * E;
        };
        auto inside = [&](uint32_t i) { return ids[i] >= 0 && static_cast<uint32_t>(ids[i]) < a.vocab; };
        bool bad = false;
        for (uint32_t i = tid; i < a.top; i += kThreads) {
            if (!inside(i)) {
                bad |= ids[i] >= 0;
                continue;
            }
            const uintptr_t x = reinterpret_cast<uintptr_t>(xr + ids[i]);
            copy_word_async(z_words + i, reinterpret_cast<const void*>(x & ~static_cast<uintptr_t>(3)));
            if (in_slice(i)) {
                const uint32_t at = static_cast<uint32_t>(ids[i]) + row.lead - u0 * E, bit = 1u << (at & 31);
                if (atomicOr(&marks[at >> 5], bit) & bit) repeated_flag = 1;
            }
        }
        copy_commit();
        const bool more = a.rows - row_id > clusters;
        if (more) fetch_slots(row_id + clusters, turn ^ 1);
        copy_commit();
        if (bad && a.result && rank == 0) atomicMax(&a.result->status, static_cast<uint32_t>(DCT_ERR_BAD_MASK));
        if (kTail) __syncthreads();                        // all marks are set

        // first reading: the student's sums
        auto marked = [&](uint32_t u) {
            const uint32_t at = (u - u0) * E;
            return marks[at >> 5] >> (at & 31) & ((1u << E) - 1);
        };
        RowSums sums;
        float x_best = minus_inf();
        stream_units<T, kThreads>(row, u0, u1, [&](uint4 (&v)[4], uint32_t first) {
            if (kTail) {
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {
                    const uint32_t u = first + i * kThreads, bits = u < u1 ? marked(u) : 0u;
                    if (bits) {
#pragma unroll
                        for (uint32_t e = 0; e < E; ++e)
                            if (bits >> e & 1u) Unit<T>::set(v[i], e, minus_inf());
                    }
                }
            }
            const float best = fmaxf(Unit<T>::best(v[0], v[2]), Unit<T>::best(v[1], v[3]));
            x_best = fmaxf(x_best, best);
            sums.add<T, false>(v, best, a.c);
        });
        const RowPart mine = sums.part(warp_max(x_best), a.c);

        // the slots: the teacher's values, and (kTail) the student's at the slice's named columns, each column once
        copy_wait<1>();
        auto logit = [&](uint32_t i) {
            const uint32_t w = z_words[i];
            if (sizeof(T) == 4) return __uint_as_float(w);
            return __uint_as_float(reinterpret_cast<uintptr_t>(xr + ids[i]) & 2u ? w & 0xFFFF0000u : w << 16);
        };
        auto first_of_its_column = [&](uint32_t i) {
            for (uint32_t k = 0; k < i; ++k)
                if (ids[k] == ids[i]) return false;
            return true;
        };
        RowPart teacher{minus_inf(), 0.0f, 0.0f}, named{minus_inf(), 0.0f, 0.0f};
        float q_sum = 0.0f;
        {
            const bool repeated = kTail && repeated_flag != 0;
            for (uint32_t i = tid; i < a.top; i += kThreads) {
                if (!inside(i)) continue;
                if (kTail) {
                    q_sum += expf(t_s[i]);
                    if (in_slice(i) && (!repeated || first_of_its_column(i))) add_value(named, __fmul_rn(logit(i), a.inv_t));
                } else {
                    add_value(teacher, t_s[i]);
                }
            }
        }
        if (kTail) {
            q_sum = warp_join<SumOp>(q_sum);
            named.join_lanes(kLog2E, 32);
        } else {
            teacher.join_lanes(kLog2E, 32);
        }
        if (lane == 0) {
            student_parts[warp] = mine;
            teacher_parts[warp] = kTail ? RowPart{0.0f, q_sum, 0.0f} : teacher;
            if (kTail) named_parts[warp] = named;
        }
        __syncthreads();

        // every warp joins the parts of all
        RowPart student = student_parts[lane & (kWarps - 1)];
        student.join_lanes(a.c, kWarps);
        if (student.s == 0.0f && student.xmax > minus_inf())
            student = low_part(row, u0, u1, student.xmax, a.c, [=](uint32_t u, uint32_t i) {
                const uint32_t at = (u - u0) * E + i;
                return !kTail || !(marks[at >> 5] >> (at & 31) & 1u);
            });
        if (kTail) {
            named = named_parts[lane & (kWarps - 1)];
            named.join_lanes(kLog2E, kWarps);
        }
        if (kCluster) {
            if (tid == 0) {
                slice_part = student;
                slice_named = named;
            }
            cluster_barrier();
            const uint32_t c = lane & (kMaxCluster - 1);
            student = named = RowPart{minus_inf(), 0.0f, 0.0f};
            if (c < ctas) {
                student.xmax = ld_remote_f32(remote_smem(&slice_part.xmax, c));
                student.s = ld_remote_f32(remote_smem(&slice_part.s, c));
                if (kTail) {
                    named.xmax = ld_remote_f32(remote_smem(&slice_named.xmax, c));
                    named.s = ld_remote_f32(remote_smem(&slice_named.s, c));
                }
            }
            student.join_lanes(a.c, kMaxCluster);
            if (kTail) named.join_lanes(kLog2E, kMaxCluster);
            cluster_arrive();                              // (waited for at the end of the row)
        }
        teacher = teacher_parts[lane & (kWarps - 1)];
        teacher.join_lanes(kLog2E, kWarps);                // (kTail: all xmax are 0, s becomes the sum of q)
        const bool repeated = repeated_flag != 0;

        // log Z = z_max + log_total; the streamed columns' share p_streamed of the student's distribution (1 unless kTail)
        const float z_streamed = __fmul_rn(student.xmax, a.inv_t), exact_rest = fmaf(student.xmax, a.inv_t, -z_streamed);
        float z_max = z_streamed, log_total = logf(student.s) + (student.xmax > minus_inf() ? exact_rest : 0.0f);
        float log_streamed = 0.0f, q_rest = 0.0f, log_norm = 0.0f;
        if (kTail) {
            const float log_s = log_total;
            z_max = fmaxf(z_streamed, named.xmax);
            float total = named.s == 0.0f ? 0.0f : named.s * expf(named.xmax - z_max);
            if (student.s != 0.0f) total += expf((z_streamed - z_max) + log_s);
            log_total = logf(total);
            log_streamed = (z_streamed - z_max) + (log_s - log_total);
            q_rest = teacher.s > 1.0f ? 0.0f : 1.0f - teacher.s;
        } else {
            log_norm = teacher.xmax + logf(teacher.s);
        }
        const bool broken = log_total != log_total || teacher.s != teacher.s;
        const bool nothing = (!broken && z_max == minus_inf()) || (!kTail && teacher.s == 0.0f);
        const bool remainder = kTail && student.s != 0.0f;
        auto log_p = [&](uint32_t i) { return fmaf(logit(i), a.inv_t, -z_max) - log_total; };
        auto log_q = [&](uint32_t i) { return t_s[i] - log_norm; };

        if (a.loss_out && rank == 0) {
            float loss = 0.0f;
            for (uint32_t i = tid; i < a.top; i += kThreads)
                if (inside(i)) {
                    const float lq = log_q(i), q = expf(lq);
                    if (q != 0.0f) loss = fmaf(q, lq - log_p(i), loss);
                }
            if (remainder && tid == 0 && q_rest != 0.0f) loss = fmaf(q_rest, logf(q_rest) - log_streamed, loss);
            loss = warp_join<SumOp>(loss);
            if (lane == 0) loss_parts[warp] = loss;
        }
        T* out = grad + static_cast<size_t>(row_id) * a.ld_grad;
        const float scale = __fmul_rn(a.grad_loss ? a.grad_loss[row_id] : 1.0f, a.inv_t);
        if (grad) {
            // second reading: 2^((x - xmax) c) times one factor
            const bool aligned = same_boundary(xr, out);
            float factor = scale / student.s;
            if (kTail) factor = remainder ? factor * (expf(log_streamed) - q_rest) : 0.0f;
            if (broken) factor = __uint_as_float(0x7FFFFFFFu);
            if (nothing) factor = 0.0f;
            const float x_ref = student.xmax == minus_inf() ? 0.0f : -student.xmax;
            const uint64_t shift = pack2(x_ref, x_ref), by_c = pack2(a.c, a.c), by_factor = pack2(factor, factor);
            for (uint32_t batch = u0; batch < u1; batch += 4 * kThreads) {
                const uint32_t first = batch + tid;
                uint4 v[4];
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i)
                    if (first + i * kThreads < u1) v[i] = ld_unit(row.base + first + i * kThreads);
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {
                    const uint32_t u = first + i * kThreads;
                    if (u >= u1) break;
                    float g[E];
#pragma unroll
                    for (uint32_t e = 0; e < E; e += 2) {
                        float y0, y1;
                        unpack2(mul2(add2(pack2(Unit<T>::get(v[i], e), Unit<T>::get(v[i], e + 1)), shift), by_c), y0, y1);
                        // (a named column may be far above the others that the factor belongs to: written again below)
                        if (kTail) {
                            y0 = fminf(y0, 64.0f);
                            y1 = fminf(y1, 64.0f);
                        }
                        unpack2(mul2(pack2(exp2_fast(y0), exp2_fast(y1)), by_factor), g[e], g[e + 1]);
                        if (nothing) g[e] = g[e + 1] = 0.0f;            // whatever the logits are
                    }
                    store_unit(row, out, u, g, aligned);
                }
            }
        }
        __syncthreads();                                   // the gradient is written, the loss' parts are there

        if (a.loss_out && rank == 0 && warp == 0) {
            float loss = lane < kWarps ? loss_parts[lane] : 0.0f;
            loss = warp_join<SumOp>(loss);
            if (lane == 0) a.loss_out[row_id] = nothing ? 0.0f : broken ? __uint_as_float(0x7FFFFFFFu) : loss;
        }
        for (uint32_t i = tid; i < a.top; i += kThreads) {
            if (!inside(i)) continue;
            if (!in_slice(i)) continue;
            marks[(static_cast<uint32_t>(ids[i]) + row.lead - u0 * E) >> 5] = 0;
            if (!grad || nothing || (repeated && !first_of_its_column(i))) continue;
            float q = expf(log_q(i));
            if (repeated)
                for (uint32_t k = i + 1; k < a.top; ++k)
                    if (ids[k] == ids[i]) q += expf(log_q(k));
            out[ids[i]] = from_f32<T>(broken ? __uint_as_float(0x7FFFFFFFu) : (expf(log_p(i)) - q) * scale);
        }
        if (tid == 0) repeated_flag = 0;
        if (kCluster) cluster_wait();
        if (!more) break;
        row_id += clusters;
    }
}

template <typename T, uint32_t kThreads, bool kTail>
dct_status_t launch_distill_threads(const void* logits, void* grad, DistillArgs a, uint32_t cluster, cudaStream_t stream) {
    const int sms = sm_count();
    if (sms <= 0) return DCT_ERR_CUDA;
    const uint32_t units = a.vocab / Unit<T>::kElems + 2, share = (units + cluster - 1) / cluster;
    a.mark_words = ((share * Unit<T>::kElems + 31) / 32 + 3) & ~3u;
    const size_t smem = 4 * static_cast<size_t>(a.mark_words) + 20 * static_cast<size_t>(a.top);
    const T* x = static_cast<const T*>(logits);
    T* g = static_cast<T*>(grad);
    const uint64_t wanted = static_cast<uint64_t>(a.rows) * cluster;
    const uint32_t room = static_cast<uint32_t>(sms) * (768 / kThreads) / cluster * cluster;
    const uint32_t grid = static_cast<uint32_t>(wanted < room ? wanted : room);
    if (cluster > 1) {
        auto kernel = lm_distill_kernel<T, kThreads, kTail, true>;
        if (smem > 32 * 1024)
            DCT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
        DCT_CUDA_TRY(launch_clusters(kernel, grid, kThreads, cluster, smem, stream, x, g, a));
        return DCT_OK;
    }
    auto kernel = lm_distill_kernel<T, kThreads, kTail, false>;
    if (smem > 32 * 1024)
        DCT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
    kernel<<<grid, kThreads, smem, stream>>>(x, g, a);
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}

template <typename T, bool kTail>
dct_status_t launch_distill(const void* logits, void* grad, const DistillArgs& a, cudaStream_t stream) {
    const int sms = sm_count();
    if (sms <= 0) return DCT_ERR_CUDA;
    const uint32_t units = a.vocab / Unit<T>::kElems + 2;
    uint32_t cluster = 1;
    while (cluster < kMaxCluster && static_cast<uint64_t>(a.rows) * cluster * 2 <= 3ull * sms && units / (cluster * 2) >= 512) cluster *= 2;
    while (cluster < kMaxCluster && units / cluster > 16384) cluster *= 2;
    return launch_distill_threads<T, 256, kTail>(logits, grad, a, cluster, stream);
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
    const DistillArgs args{rows, vocab, ld, inv_temperature, log2_scale(inv_temperature), teacher_ids, teacher_logprobs, top,
                           grad_loss, loss_out, ld_grad, 0, result};
    auto launch = dtype == DCT_F32
        ? (mode == DCT_DISTILL_TAIL ? launch_distill<float, true> : launch_distill<float, false>)
        : (mode == DCT_DISTILL_TAIL ? launch_distill<__nv_bfloat16, true> : launch_distill<__nv_bfloat16, false>);
    return launch(logits, grad_logits, args, stream);
}
