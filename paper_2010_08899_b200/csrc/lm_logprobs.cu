// Log-probabilities of given tokens, entropy and the most likely columns of rows of logits; and their gradient.
#include "lm_rows.cuh"

namespace dct {
namespace {

constexpr uint32_t kMaxCluster = 8u;
constexpr uint32_t kMaxima = 4096u;           // noted maxima of a CTA (16 for each of 256 threads)
constexpr uint32_t kCandidates = 2048u;       // columns the selection holds at a time
constexpr uint32_t kRankable = 512u;          // ... and the most it puts in order by counting

struct LogProbArgs {
    uint32_t rows, vocab, ld;
    float inv_t;
    const int32_t* tokens;
    uint32_t top;
    float *logprob_out, *entropy_out, *stats_out;
    int32_t* top_ids;
    float* top_logprobs;
    dct_result_t* result;
};

// What one CTA knows of its slice of the row, read by the others of its cluster.
struct SlicePart {
    float m, s, st;
    uint32_t kept;
};

template <uint32_t kThreads> struct LogProbShared {
    static constexpr uint32_t kGroups = kMaxima / kThreads;
    float group_max[kMaxima];
    uint64_t candidates[kCandidates];
    uint64_t best[DCT_LM_MAX_TOP];
    uint16_t hits[kMaxima];
    float slots[96];
    uint32_t counts[32];
    uint32_t counter, hit_count;
    SlicePart part;
};

__device__ __forceinline__ float value_of_key(uint32_t key) {       // the inverse of order_key
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// The selection of a slice's best columns.  A column is (order key << 32 | ~column): larger is better, all distinct.
// While the row streams by, every thread notes the largest element of each batch of units it reads.  The kk-th
// largest of the threads' own maxima is a bound that at least kk columns reach and, for kk well below the number of
// threads, not many more do (T ln(T / (T - kk)) for columns in no particular order); only batches whose noted maximum reaches it
// are read again, and of them the elements that reach it are put in order by counting.
template <typename T, uint32_t kThreads> struct Selector {
    static constexpr uint32_t E = Unit<T>::kElems;
    const RowView<T>& row;
    uint32_t u0, u1;                // the slice's units
    uint32_t per_group;             // batches per noted maximum
    LogProbShared<kThreads>& sh;

    template <typename F> __device__ __forceinline__ void each_element(uint32_t u, F&& f) const {
        const uint4 v = ld_unit(row.base + u);
#pragma unroll
        for (uint32_t i = 0; i < E; ++i) {
            const uint32_t col = row.column(u, i);
            if (col < row.width) f(order_key(Unit<T>::get(v, i)), col);
        }
    }
    __device__ __forceinline__ static uint64_t entry(uint32_t key, uint32_t col) {
        return static_cast<uint64_t>(key) << 32 | (0xFFFFFFFFu - col);
    }
    // candidates := the slice's columns with key >= bound (> bound if strict); returns how many there are, of which the
    // first kCandidates found are stored.  The groups whose maximum reaches the bound are listed first and their units
    // then dealt out over all threads: every load is independent of the others.
    __device__ uint32_t collect(uint32_t bound, bool strict) {
        __syncthreads();
        if (threadIdx.x == 0) sh.counter = sh.hit_count = 0;
        __syncthreads();
        const uint32_t low = strict ? bound + 1 : bound;          // (bound = 0xFFFFFFFF is no element's key)
        const uint32_t span = per_group * 4 * kThreads, groups = (u1 - u0 + span - 1) / span;
        for (uint32_t g = 0; g < groups; ++g)
            if (order_key(sh.group_max[g * kThreads + threadIdx.x]) >= low)
                sh.hits[atomicAdd(&sh.hit_count, 1u)] = static_cast<uint16_t>(g * kThreads + threadIdx.x);
        __syncthreads();
        const uint32_t in_group = per_group * 4, items = sh.hit_count * in_group;
        for (uint32_t item = threadIdx.x; item < items; item += kThreads) {
            const uint32_t hit = sh.hits[item / in_group];
            const uint32_t u = u0 + (hit / kThreads * in_group + item % in_group) * kThreads + hit % kThreads;
            if (u >= u1) continue;
            const uint4 v = ld_unit(row.base + u);
            if (low > 1 && order_key(Unit<T>::best(v, v, v, v)) < low) continue;
#pragma unroll
            for (uint32_t i = 0; i < E; ++i) {
                const uint32_t col = row.column(u, i), key = order_key(Unit<T>::get(v, i));
                if (key >= low && col < row.width) {
                    const uint32_t at = atomicAdd(&sh.counter, 1u);
                    if (at < kCandidates) sh.candidates[at] = entry(key, col);
                }
            }
        }
        __syncthreads();
        return sh.counter;
    }
    // the kk-th largest key of the slice, by halving the range of keys: 32 passes
    __device__ uint32_t kth_key(uint32_t kk) {
        uint32_t lo = 0, hi = 0xFFFFFFFFu;
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2 + 1;
            uint32_t n = 0;
            for (uint32_t u = u0 + threadIdx.x; u < u1; u += kThreads)
                each_element(u, [&](uint32_t key, uint32_t) { n += key >= mid; });
            if (cta_count(n, sh.counts) >= kk) lo = mid;
            else hi = mid - 1;
        }
        return lo;
    }
    // appends the lowest columns whose key is `key` until there are kk candidates
    __device__ void fill_with_equals(uint32_t key, uint32_t have, uint32_t kk) {
        for (uint32_t first = u0; first < u1 && have < kk; first += kThreads) {
            const uint32_t u = first + threadIdx.x;
            uint32_t mine = 0;
            if (u < u1) each_element(u, [&](uint32_t k, uint32_t) { mine += k == key; });
            uint32_t before = mine;                         // inclusive sum over the lanes
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t t = __shfl_up_sync(0xFFFFFFFFu, before, o);
                if (lane_id() >= static_cast<uint32_t>(o)) before += t;
            }
            __syncthreads();
            if (lane_id() == 31) sh.counts[threadIdx.x >> 5] = before;
            __syncthreads();
            uint32_t at = have + before - mine, all = 0;
            for (uint32_t w = 0; w < kThreads / 32; ++w) {
                if (w < (threadIdx.x >> 5)) at += sh.counts[w];
                all += sh.counts[w];
            }
            if (u < u1 && mine)
                each_element(u, [&](uint32_t k, uint32_t col) {
                    if (k == key) {
                        if (at < kk) sh.candidates[at] = entry(key, col);
                        ++at;
                    }
                });
            have += all;
        }
        __syncthreads();
    }
    // keeps the kk best of n candidates, kk < n, in no order
    __device__ void cut(uint32_t n, uint32_t kk) {
        uint64_t lo = 0, hi = ~0ull;
        while (lo < hi) {
            const uint64_t mid = lo + (hi - lo) / 2 + 1;
            uint32_t c = 0;
            for (uint32_t i = threadIdx.x; i < n; i += kThreads) c += sh.candidates[i] >= mid;
            c = cta_count(c, sh.counts);
            if (c >= kk) lo = mid;
            else hi = mid - 1;
            if (c == kk) break;
        }
        if (threadIdx.x == 0) sh.counter = 0;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < n; i += kThreads)
            if (sh.candidates[i] >= lo) sh.best[atomicAdd(&sh.counter, 1u)] = sh.candidates[i];
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < kk; i += kThreads) sh.candidates[i] = sh.best[i];
        __syncthreads();
    }
    // best[0 .. kk) := the slice's kk best columns in order.  thread_max: the largest element of this thread's batches.
    __device__ void run(float thread_max, uint32_t kk) {
        const uint32_t units = u1 - u0;
        uint32_t bound = 0;
        if (min(units, kThreads) >= kk) {
            const uint32_t key = threadIdx.x < units ? order_key(thread_max) : 0u;
            uint32_t lo = __reduce_min_sync(0xFFFFFFFFu, key), hi = __reduce_max_sync(0xFFFFFFFFu, key);
            __syncthreads();
            if (lane_id() == 0) {
                sh.counts[threadIdx.x >> 5] = hi;
                sh.slots[threadIdx.x >> 5] = __uint_as_float(lo);
            }
            __syncthreads();
            for (uint32_t w = 0; w < kThreads / 32; ++w) {
                hi = max(hi, sh.counts[w]);
                lo = min(lo, __float_as_uint(sh.slots[w]));
            }
            // at least kk threads reach lo, fewer reach hi + 1; a few more than kk are as good as kk
            while (lo < hi) {
                const uint32_t mid = lo + (hi - lo) / 2 + 1;
                const uint32_t c = __syncthreads_count(key >= mid);
                if (c >= kk) lo = mid;
                else hi = mid - 1;
                if (c >= kk && c <= kk + kk / 4 + 2) break;
            }
            bound = lo;
        }
        uint32_t n = collect(bound, false);
        if (n < kk) {                          // threads whose only elements lie outside the row or are NaN
            bound = 0;
            n = collect(bound, false);
        }
        if (n > kCandidates) {                 // many equal to the bound, or sorted columns
            n = collect(bound, true);
            if (n > kCandidates) {
                bound = kth_key(kk);
                n = collect(bound, true);
            }
            if (n < kk) {
                fill_with_equals(bound, n, kk);
                n = kk;
            }
        }
        if (n > kRankable) {
            cut(n, kk);
            n = kk;
        }
        for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
            const uint64_t key = sh.candidates[i];
            uint32_t rank = 0;
            for (uint32_t q = 0; q < n; ++q) rank += sh.candidates[q] > key;
            if (rank < kk) sh.best[rank] = key;
        }
        __syncthreads();
    }
};

// A cluster of CTAs takes a row, each CTA a slice of its units; the CTAs join their sums and their ordered best columns
// through each other's shared memory.
template <typename T, uint32_t kThreads, bool kCluster>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads)
lm_logprobs_kernel(const T* __restrict__ logits, const LogProbArgs a) {
    __shared__ LogProbShared<kThreads> sh;
    const uint32_t tid = threadIdx.x;
    const uint32_t rank = kCluster ? cluster_rank() : 0u, ctas = kCluster ? cluster_size() : 1u;
    const uint32_t clusters = gridDim.x / ctas;
    for (uint32_t row_id = blockIdx.x / ctas; row_id < a.rows; row_id += clusters) {
        const T* xr = logits + static_cast<size_t>(row_id) * a.ld;
        const RowView<T> row(xr, a.vocab);
        const uint32_t share = (row.units + ctas - 1) / ctas;
        const uint32_t u0 = min(row.units, rank * share), u1 = min(row.units, u0 + share);
        int32_t tok = -1;
        float x_tok = 0.0f;
        if (tid == 0 && rank == 0 && a.tokens) {
            tok = a.tokens[row_id];
            if (tok >= 0 && static_cast<uint32_t>(tok) < a.vocab) x_tok = to_f32(xr[tok]);
        }

        // one pass: sums, and the largest element of every batch of four units
        RowSums sums;
        const uint32_t batches = (u1 - u0 + 4 * kThreads - 1) / (4 * kThreads);
        const uint32_t per_group = max(1u, (batches + sh.kGroups - 1) / sh.kGroups);
        float thread_max = minus_inf(), group_max = minus_inf();
        uint32_t in_group = 0, group = 0;
        for (uint32_t b = 0; b < batches; ++b) {
            const uint32_t first = u0 + b * 4 * kThreads + tid;
            uint4 v[4];
            load_batch<T, kThreads>(v, row, first, u1);
            mask_batch<T, kThreads>(v, row, first, u1);
            const float best = Unit<T>::best(v[0], v[1], v[2], v[3]);
            sums.add<T, true>(v, best, a.inv_t);
            group_max = fmaxf(group_max, best);
            if (++in_group == per_group || b + 1 == batches) {
                sh.group_max[group * kThreads + tid] = group_max;
                thread_max = fmaxf(thread_max, group_max);
                group_max = minus_inf();
                in_group = 0;
                ++group;
            }
        }
        // the slice's sums, relative to its largest z
        sums.join_cta(__fmul_rn(thread_max, a.inv_t), sh.slots);
        float m = sums.ref, s = sums.s, st = sums.st;

        uint32_t kept = 0;
        if (a.top) {
            const uint32_t columns = u1 == u0 ? 0u
                : min(a.vocab, u1 * Unit<T>::kElems - row.lead) - (u0 == 0 ? 0u : u0 * Unit<T>::kElems - row.lead);
            kept = min(a.top, columns);
            if (kept) Selector<T, kThreads>{row, u0, u1, per_group, sh}.run(thread_max, kept);
        }

        if (kCluster) {
            if (tid == 0) sh.part = SlicePart{m, s, st, kept};
            cluster_barrier();
            float all_m = minus_inf();
            for (uint32_t c = 0; c < ctas; ++c) all_m = fmaxf(all_m, ld_remote_f32(remote_smem(&sh.part.m, c)));
            s = st = 0.0f;
            for (uint32_t c = 0; c < ctas; ++c) {
                RowSums other;
                other.ref = ld_remote_f32(remote_smem(&sh.part.m, c));
                other.s = ld_remote_f32(remote_smem(&sh.part.s, c));
                other.st = ld_remote_f32(remote_smem(&sh.part.st, c));
                other.finish(all_m);
                s = __fadd_rn(s, other.s);
                st = __fadd_rn(st, other.st);
            }
            m = all_m;
        }
        const bool empty = m == minus_inf() && s == 0.0f;
        const float ref = m == minus_inf() ? 0.0f : m;
        const float logsum = empty ? 0.0f : logf(s);
        if (tid == 0 && rank == 0) {
            if (a.tokens) {
                const bool inside = tok >= 0 && static_cast<uint32_t>(tok) < a.vocab;
                a.logprob_out[row_id] = inside ? fmaf(x_tok, a.inv_t, -ref) - logsum : 0.0f;
                if (tok >= 0 && !inside && a.result) atomicMax(&a.result->status, static_cast<uint32_t>(DCT_ERR_BAD_MASK));
            }
            if (a.entropy_out) a.entropy_out[row_id] = empty ? 0.0f : logsum - st / s;
            if (a.stats_out) {
                a.stats_out[2 * static_cast<size_t>(row_id)] = m;
                a.stats_out[2 * static_cast<size_t>(row_id) + 1] = logsum;
            }
        }
        if (a.top) {
            // a column's place: its place in its own slice's list, and how many of each other list are better
            uint32_t starts = 0;
            if (kCluster) {
                for (uint32_t c = 0; c < ctas; ++c) {
                    const uint32_t n = ld_remote_u32(remote_smem(&sh.part.kept, c));
                    for (uint32_t i = tid; i < n; i += kThreads)
                        sh.candidates[c * DCT_LM_MAX_TOP + i] = ld_remote_u64(remote_smem(&sh.best[i], c));
                    if (tid == 0) sh.counts[c] = n;
                    starts += n;
                }
                __syncthreads();
            }
            for (uint32_t i = tid; i < kept; i += kThreads) {
                const uint64_t key = sh.best[i];
                uint32_t place = i;
                if (kCluster) {
                    for (uint32_t c = 0; c < ctas; ++c) {
                        if (c == rank) continue;
                        const uint64_t* list = sh.candidates + c * DCT_LM_MAX_TOP;
                        uint32_t lo = 0, hi = sh.counts[c];         // list[0 .. lo) are better
                        while (lo < hi) {
                            const uint32_t mid = (lo + hi) / 2;
                            if (list[mid] > key) lo = mid + 1;
                            else hi = mid;
                        }
                        place += lo;
                    }
                }
                if (place < a.top) {
                    const size_t at = static_cast<size_t>(row_id) * a.top + place;
                    a.top_ids[at] = static_cast<int32_t>(0xFFFFFFFFu - static_cast<uint32_t>(key));
                    a.top_logprobs[at] = fmaf(value_of_key(static_cast<uint32_t>(key >> 32)), a.inv_t, -ref) - logsum;
                }
            }
        }
        if (kCluster) cluster_barrier();          // nobody reads this CTA's shared memory any more
        else __syncthreads();
    }
}

// Elementwise: a CTA takes four units per thread of one row.
constexpr uint32_t kBwdThreads = 256u, kBwdUnits = 4u;

struct LogProbBwdArgs {
    uint32_t rows, vocab, ld;
    float inv_t;
    const int32_t* tokens;
    const float *stats, *entropy, *grad_logprob, *grad_entropy;
    uint32_t ld_grad, chunks;
};

template <typename T>
__global__ void __launch_bounds__(kBwdThreads)
lm_logprobs_bwd_kernel(const T* logits, T* grad, const LogProbBwdArgs q) {
    constexpr uint32_t E = Unit<T>::kElems;
    const uint64_t tiles = static_cast<uint64_t>(q.rows) * q.chunks;
    for (uint64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const uint32_t row_id = static_cast<uint32_t>(tile / q.chunks);
        const uint32_t first = static_cast<uint32_t>(tile % q.chunks) * (kBwdUnits * kBwdThreads) + threadIdx.x;
        const T* xr = logits + static_cast<size_t>(row_id) * q.ld;
        T* out = grad + static_cast<size_t>(row_id) * q.ld_grad;
        const RowView<T> row(xr, q.vocab);
        const bool aligned = same_boundary(xr, out);
        uint4 v[kBwdUnits];
#pragma unroll
        for (uint32_t i = 0; i < kBwdUnits; ++i) {
            const uint32_t u = first + i * kBwdThreads;
            if (u < row.units) v[i] = ld_unit(row.base + u);
        }
        const float m = q.stats[2 * static_cast<size_t>(row_id)], logsum = q.stats[2 * static_cast<size_t>(row_id) + 1];
        const bool empty = m == minus_inf();
        const float ref = empty ? 0.0f : m;
        const int32_t tok = q.grad_logprob ? q.tokens[row_id] : -1;
        const bool asked = tok >= 0 && static_cast<uint32_t>(tok) < q.vocab && !empty;
        const float a = asked ? q.grad_logprob[row_id] : 0.0f;
        const float c = q.grad_entropy ? q.grad_entropy[row_id] : 0.0f, h = q.grad_entropy ? q.entropy[row_id] : 0.0f;
        const uint32_t tok_at = asked ? static_cast<uint32_t>(tok) + row.lead : 0xFFFFFFFFu;
        const uint64_t scale = pack2(q.inv_t, q.inv_t), shift = pack2(-ref, -ref), less = pack2(-logsum, -logsum);
        const uint64_t to_log2 = pack2(kLog2E, kLog2E), plus = pack2(h, h), minus_c = pack2(-c, -c), minus_a = pack2(-a, -a);
#pragma unroll
        for (uint32_t i = 0; i < kBwdUnits; ++i) {
            const uint32_t u = first + i * kBwdThreads;
            if (u >= row.units) break;
            float g[E];
#pragma unroll
            for (uint32_t e = 0; e < E; e += 2) {
                float l0, l1, y0, y1;
                unpack2(add2(fma2(pack2(Unit<T>::get(v[i], e), Unit<T>::get(v[i], e + 1)), scale, shift), less), l0, l1);
                // (a column without weight: its log p may be -inf, and 0 * -inf is not 0)
                const uint64_t lp = pack2(max_nan(l0, -1.0e4f), max_nan(l1, -1.0e4f));
                unpack2(mul2(lp, to_log2), y0, y1);
                const uint64_t p = pack2(exp2_fast(y0), exp2_fast(y1));
                unpack2(mul2(mul2(p, fma2(minus_c, add2(lp, plus), minus_a)), scale), g[e], g[e + 1]);
            }
            if (tok_at / E == u) {
#pragma unroll
                for (uint32_t e = 0; e < E; ++e)
                    g[e] = fmaf(tok_at % E == e ? a : 0.0f, q.inv_t, g[e]);
            }
            store_unit(row, out, u, g, aligned);
        }
    }
}

template <typename T, uint32_t kThreads>
dct_status_t launch_logprobs_threads(const void* logits, const LogProbArgs& a, uint32_t cluster, cudaStream_t stream) {
    const T* x = static_cast<const T*>(logits);
    const uint32_t clusters = a.rows < (1u << 20) ? a.rows : 1u << 20;
    if (cluster == 1)
        lm_logprobs_kernel<T, kThreads, false><<<clusters, kThreads, 0, stream>>>(x, a);
    else
        DCT_CUDA_TRY(launch_clusters(lm_logprobs_kernel<T, kThreads, true>, clusters * cluster, kThreads, cluster, 0, stream, x, a));
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}

template <typename T> dct_status_t launch_logprobs(const void* logits, const LogProbArgs& a, cudaStream_t stream) {
    const int sms = sm_count();
    if (sms <= 0) return DCT_ERR_CUDA;
    const uint32_t units = (a.vocab + Unit<T>::kElems - 1) / Unit<T>::kElems;
    // a row goes to as many CTAs as it takes to give every SM two, while each still has a batch of four units per thread
    uint32_t cluster = 1;
    while (cluster < kMaxCluster && static_cast<uint64_t>(a.rows) * cluster * 2 <= static_cast<uint64_t>(sms) * 2 &&
           units / (cluster * 2) >= 1024)
        cluster *= 2;
    if (a.top > 128) return launch_logprobs_threads<T, 512>(logits, a, cluster, stream);
    return launch_logprobs_threads<T, 256>(logits, a, cluster, stream);
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
    const LogProbArgs args{rows, vocab, ld, inv_temperature, tokens, top, logprob_out, entropy_out, stats_out, top_ids, top_logprobs, result};
    return dtype == DCT_F32 ? launch_logprobs<float>(logits, args, stream) : launch_logprobs<__nv_bfloat16>(logits, args, stream);
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
    // (a row that starts inside a unit spans one unit more)
    const uint32_t units = vocab / static_cast<uint32_t>(16 / es) + 2, tile = kBwdUnits * kBwdThreads;
    const LogProbBwdArgs args{rows, vocab, ld, inv_temperature, tokens, stats, entropy, grad_logprob, grad_entropy, ld_grad,
                              (units + tile - 1) / tile};
    const uint64_t tiles = static_cast<uint64_t>(rows) * args.chunks;
    const uint32_t grid = static_cast<uint32_t>(tiles < (1u << 30) ? tiles : 1u << 30);
    if (dtype == DCT_F32)
        lm_logprobs_bwd_kernel<float><<<grid, kBwdThreads, 0, stream>>>(static_cast<const float*>(logits),
                                                                        static_cast<float*>(grad_logits), args);
    else
        lm_logprobs_bwd_kernel<__nv_bfloat16><<<grid, kBwdThreads, 0, stream>>>(
            static_cast<const __nv_bfloat16*>(logits), static_cast<__nv_bfloat16*>(grad_logits), args);
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}
