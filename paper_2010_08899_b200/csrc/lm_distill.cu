// Distillation from a teacher's top log-probabilities: loss and gradient of rows of logits.
#include "lm_rows.cuh"

namespace dct {
namespace {

constexpr uint32_t kMaxCluster = 8u;

struct DistillArgs {
    uint32_t rows, vocab, ld;
    Scale by;
    const int32_t* ids;
    const float* lps;
    uint32_t top;
    const float* grad_loss;
    float* loss_out;
    uint32_t ld_grad, chunks, mark_words, spin_limit;      // of a CTA's slice at most; polls a wait may take
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

// A row belongs to a cluster of CTAs, a slice of it to each, and a slice's chunks of 128 units (2 KiB) in turn to the CTA's
// warps.  The logits are needed twice, for the sums and, when those are joined, for the gradient.  kStaged: a warp fetches
// its chunks by bulk copies into shared memory, works on them twice and, as it lets go of each, asks for the next row's, so
// that they cross the memory bus once and are under way while other work is done; otherwise (slices that would leave an SM one CTA)
// they are loaded twice, the second time from L2.  The teacher's slots of the next row, and the logits that this row's slots name, are fetched while the
// row streams by.  `marks` has a bit for every element of the slice's units that a slot names.  kTail: those are left out of
// the sums, so that the remainder is summed and not a difference.  The gradient is first written as if no column were named,
// and the named ones once more afterwards.
// Slot i belongs to thread i mod kThreads throughout.
// With y_j = (x_j - xmax) c and S = sum 2^y over the streamed columns:
//   RENORM: gradient of a column 2^y (scale / S), a named one's less its q scale;
//   TAIL:   of a column that is not named 2^y (p_r - q_r) scale / S, with p_r the streamed columns' share of the whole: the
//           factor p_j (1 - q_r / p_r) without the quotient, which overflows where the remainder is tiny.
// What bounds it: instructions and the latencies between them, 2.2 a cycle of 4 at the 24 warps to an SM that the rows' shared memory and 80
// registers leave.  An element takes two powers of two (the special function unit is at 57 %) and 15.7 instructions of its thread in all, of which 12.6 are
// the two readings and the rest is the row's joins, logarithms and slots; with the remainder 19.5.  Reading and writing 2^27 bf16 logits alone would
// take 82 us.  4096 rows of 32768 bf16, 64 slots: 111 us (4.8 TB/s; every logit is read from DRAM once), fp32 182 us (5.9); 1024 rows of 131072 bf16,
// 128 slots and the remainder: 140 us (3.8 TB/s).
constexpr uint32_t kChunkUnits = 128u, kChunkBytes = 16u * kChunkUnits;
constexpr uint32_t kMaxChunksPerWarp = 16u;
// shared memory of a CTA that a staged slice may take: three CTAs to an SM.  (With one, loading twice is faster: 256 rows of 262144
// fp32, 8 CTAs to a row, 195 us staged and 138 loaded twice; rows of 32768 bf16 154 us loaded twice and 111 staged.)
constexpr uint32_t kStagedLimit = 90u * 1024u;

template <typename T, uint32_t kThreads, bool kTail, bool kCluster, bool kStaged>
__global__ void __launch_bounds__(kThreads, 768 / kThreads)
lm_distill_kernel(const T* logits, T* grad, const DistillArgs a) {
    constexpr uint32_t E = Unit<T>::kElems, kWarps = kThreads / 32;
    extern __shared__ __align__(128) uint32_t dynamic[];
    __shared__ RowPart student_parts[kWarps], named_parts[kWarps];
    // the sums of the cluster's slices: every CTA pushes its own to all, two rows in turn.  (A row's numbers arrive only after every CTA
    // has had the last row's, so two places are enough, and no barrier has to wait for the gradient's stores.)
    __shared__ __align__(16) float4 pushed[kCluster ? 2 : 1][kMaxCluster];
    __shared__ uint64_t joined[2];
    __shared__ float loss_parts[kWarps];
    __shared__ uint32_t repeated_flag, weight_flag, nan_flag, gave_up;      // of the row's slots; a wait ran out
    __shared__ uint64_t arrived[kStaged ? kWarps * kMaxChunksPerWarp : 1];
    uint4* const stage = reinterpret_cast<uint4*>(dynamic);
    uint32_t* const marks = dynamic + (kStaged ? a.chunks * (kChunkBytes / 4) : 0);
    int32_t* const ids_by_turn = reinterpret_cast<int32_t*>(marks + a.mark_words);       // two rows
    float* const t_by_turn = reinterpret_cast<float*>(ids_by_turn + 2 * a.top);           // two rows
    uint32_t* const z_words = reinterpret_cast<uint32_t*>(t_by_turn + 2 * a.top);
    const uint32_t tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = lane_id();
    const uint32_t rank = kCluster ? cluster_rank() : 0u, ctas = kCluster ? cluster_size() : 1u;
    const uint32_t clusters = gridDim.x / ctas;
    uint32_t phases = 0, join_phases = 0;       // the parity each of this warp's barriers is waited for with
    bool stuck = false, join_stuck = false;     // a copy, the cluster's sums did not come at all: no more are waited for

    // (staged) asks for chunk k of a row's slice
    auto fetch_chunk = [&](const RowView<T>& of_row, const Slice& of_slice, uint32_t k) {
        const uint32_t first = of_slice.u0 + k * kChunkUnits;
        if (lane == 0 && first < of_slice.u1 && !stuck) {
            const uint32_t bytes = 16u * min(kChunkUnits, of_slice.u1 - first);
            uint64_t* bar = &arrived[warp * kMaxChunksPerWarp + k / kWarps];
            mbar_arrive_expect_tx(bar, bytes);
            bulk_load(stage + k * kChunkUnits, of_row.base + first, bytes, bar);
        }
    };
    auto fetch_slots = [&](uint32_t of_row, uint32_t turn) {
        const size_t at = static_cast<size_t>(of_row) * a.top;
        for (uint32_t i = tid; i < a.top; i += kThreads) {
            copy_word_async(ids_by_turn + turn * a.top + i, a.ids + at + i);
            copy_word_async(t_by_turn + turn * a.top + i, a.lps + at + i);
        }
    };
    uint32_t row_id = blockIdx.x / ctas;
    if (tid == 0) repeated_flag = weight_flag = nan_flag = gave_up = 0;
    __syncthreads();
    if (kStaged) {
        if (lane == 0) {
            for (uint32_t j = 0; j < kMaxChunksPerWarp; ++j) mbar_init(&arrived[warp * kMaxChunksPerWarp + j], 1);
            mbar_init_fence();
            fence_proxy_async_smem();
        }
        __syncwarp();
        const RowView<T> row(logits + static_cast<size_t>(row_id) * a.ld, a.vocab);
        for (uint32_t k = warp; k < a.chunks; k += kWarps) fetch_chunk(row, Slice(row.units, rank, ctas), k);
    }
    if (kCluster) {
        if (tid == 0) {
            mbar_init(&joined[0], 1);
            mbar_init(&joined[1], 1);
            mbar_init_fence();
        }
        cluster_arrive();                                  // (waited for before the first push)
    }
    fetch_slots(row_id, 0);
    copy_commit();
    for (uint32_t w = tid; w < a.mark_words; w += kThreads) marks[w] = 0;
    for (uint32_t turn = 0;; turn ^= 1) {
        const T* xr = logits + static_cast<size_t>(row_id) * a.ld;
        const RowView<T> row(xr, a.vocab);
        const Slice slice(row.units, rank, ctas);
        const uint32_t u0 = slice.u0, u1 = slice.u1;
        const int32_t* ids = ids_by_turn + turn * a.top;
        const float* t_s = t_by_turn + turn * a.top;
        const float scale = __fmul_rn(a.grad_loss ? __ldg(a.grad_loss + row_id) : 1.0f, a.by.inv_t);
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
            if (t_s[i] > minus_inf()) weight_flag = 1;
            if (t_s[i] != t_s[i]) nan_flag = 1;
            const uintptr_t x = reinterpret_cast<uintptr_t>(xr + ids[i]);
            copy_word_async(z_words + i, reinterpret_cast<const void*>(x & ~static_cast<uintptr_t>(3)));
            if (in_slice(i)) {
                const uint32_t at = static_cast<uint32_t>(ids[i]) + row.lead - u0 * E, bit = 1u << (at & 31);
                if (atomicOr(&marks[at >> 5], bit) & bit) repeated_flag = 1;
            }
        }
        copy_commit();
        const bool more = a.rows - row_id > clusters;
        const RowView<T> next_row(logits + static_cast<size_t>(more ? row_id + clusters : row_id) * a.ld, a.vocab);
        const Slice next_slice(next_row.units, rank, ctas);
        if (more) fetch_slots(row_id + clusters, turn ^ 1);
        copy_commit();
        if (bad && a.result && rank == 0) atomicMax(&a.result->status, static_cast<uint32_t>(DCT_ERR_BAD_MASK));
        if (kTail) __syncthreads();                        // all marks are set

        // first reading: the student's sums
        // (a unit's marks: a byte of bf16, half a byte of fp32)
        auto marked = [&](uint32_t u) -> uint32_t {
            const uint8_t* bytes = reinterpret_cast<const uint8_t*>(marks);
            if (sizeof(T) == 2) return bytes[u - u0];
            return bytes[(u - u0) >> 1] >> ((u - u0) & 1u) * 4 & 15u;
        };
        RowSums sums;
        float x_best = minus_inf();
        for (uint32_t k = warp; u0 + k * kChunkUnits < u1; k += kWarps) {
            const uint32_t first = u0 + k * kChunkUnits + lane;
            uint4 v[4];
            if (kStaged) {
                const uint32_t j = k / kWarps;
                uint64_t* const bar = &arrived[warp * kMaxChunksPerWarp + j];
                if (stuck || !__all_sync(0xFFFFFFFFu, mbar_wait_bounded(bar, phases >> j & 1u, a.spin_limit, &gave_up))) {
                    *const_cast<volatile uint32_t*>(&gave_up) = 1;       // this row and the rest become NaN
                    if (!stuck) stuck = !__all_sync(0xFFFFFFFFu, mbar_drain(bar, phases >> j & 1u));
                }
                phases ^= 1u << j;
            }
            if (kTail && kStaged) {                        // -inf at the named columns, for both readings; a word of marks to a lane
                const uint32_t w = k * (4 * E) + lane;
                uint32_t bits = lane < 4 * E && w < a.mark_words ? marks[w] : 0u;
                if (__any_sync(0xFFFFFFFFu, bits)) {
                    for (; bits; bits &= bits - 1) reinterpret_cast<T*>(stage)[32 * w + __ffs(bits) - 1] = from_f32<T>(minus_inf());
                    if (!grad) fence_proxy_async_smem();   // the next row's copy comes after this
                    __syncwarp();
                }
            }
            const uint4* from = kStaged ? stage + k * kChunkUnits + lane : row.base + first;
            if (first - lane + kChunkUnits <= u1) {        // a whole chunk
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) v[i] = kStaged ? from[32 * i] : ld_unit(from + 32 * i);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {
                    v[i] = make_uint4(Unit<T>::kMinusInf, Unit<T>::kMinusInf, Unit<T>::kMinusInf, Unit<T>::kMinusInf);
                    if (first + 32 * i < u1) v[i] = kStaged ? from[32 * i] : ld_unit(from + 32 * i);
                }
            }
            if (row.ragged && (first < kChunkUnits || first - lane + kChunkUnits >= row.units)) {      // can hold an end of the row
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i)
                    if (first + 32 * i < u1) row.mask(v[i], first + 32 * i);
            }
            if (kTail && !kStaged) {
                uint32_t bits[4];
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) bits[i] = marked(min(first + 32 * i, u1 - 1));
                if (bits[0] | bits[1] | bits[2] | bits[3]) {
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
                        for (uint32_t e = 0; e < E; ++e)
                            if (bits[i] >> e & 1u) Unit<T>::set(v[i], e, minus_inf());
                }
            }
            if (kStaged && !grad) {
                __syncwarp();                              // every lane has its units
                if (more) fetch_chunk(next_row, next_slice, k);
            }
            const float best = fmaxf(Unit<T>::best(v[0], v[2]), Unit<T>::best(v[1], v[3]));
            x_best = fmaxf(x_best, best);
            sums.add<T, false>(v, best, a.by.c);
        }
        if (kTail && kStaged && grad) fence_proxy_async_smem();      // the next row's copies come after what was written to `stage`
        const RowPart mine = sums.part<false>(warp_max(x_best), a.by.c);

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
        RowPart named{minus_inf(), 0.0f, 0.0f};
        float q_sum = 0.0f;
        if (kTail) {
            const bool repeated = repeated_flag != 0;
            for (uint32_t i = tid; i < a.top; i += kThreads) {
                if (!inside(i)) continue;
                q_sum += expf(t_s[i]);
                if (in_slice(i) && (!repeated || first_of_its_column(i))) add_value(named, __fmul_rn(logit(i), a.by.inv_t));
            }
            q_sum = warp_join<SumOp>(q_sum);
            named.join_lanes<32, false>(kLog2E);
        }
        if (lane == 0) {
            student_parts[warp] = mine;
            if (kTail) {
                named.st = q_sum;
                named_parts[warp] = named;
            }
        }
        __syncthreads();

        // every warp joins the parts of all
        RowPart student = student_parts[lane & (kWarps - 1)];
        student.join_lanes<kWarps, false>(a.by.c);
        // (the same for the whole CTA.  The warps read the slice again, a share each, and no warp goes on to write a gradient, which may
        // take the logits' place, before all have read theirs)
        if (student.xmax > minus_inf() && far_off(__fmul_rn(student.xmax, a.by.inv_t))) {
            const RowPart share = far_part(row, u0 + warp * 32, kThreads, u1, student.xmax, a.by, [=](uint32_t u, uint32_t i) {
                const uint32_t at = (u - u0) * E + i;
                return !kTail || !(marks[at >> 5] >> (at & 31) & 1u);
            });
            __syncthreads();                               // the parts of the first reading have been read
            if (lane == 0) student_parts[warp] = share;
            __syncthreads();
            student = student_parts[lane & (kWarps - 1)];
            student.join_lanes<kWarps, false>(a.by.c);
        }
        if (kTail) {
            named = named_parts[lane & (kWarps - 1)];
            q_sum = named.st;
#pragma unroll
            for (uint32_t o = kWarps / 2; o > 0; o >>= 1) q_sum = __fadd_rn(q_sum, __shfl_xor_sync(0xFFFFFFFFu, q_sum, o));
            named.st = 0.0f;
            named.join_lanes<kWarps, false>(kLog2E);
        }
        if (kCluster) {
            if (row_id == blockIdx.x / ctas) cluster_wait();         // (the first row) every CTA's mbarriers are there
            if (warp == 0) {
                if (lane == 0 && !join_stuck) mbar_arrive_expect_tx(&joined[turn], 16 * ctas);
                __syncwarp();
                if (lane < ctas)
                    push_remote(remote_smem(&pushed[turn][rank], lane), student.xmax, gave_up ? __uint_as_float(0x7FFFFFFFu) : student.s,
                                named.xmax, named.s, remote_smem(&joined[turn], lane));
            }
            if (join_stuck || !__all_sync(0xFFFFFFFFu, mbar_wait_bounded(&joined[turn], join_phases >> turn & 1u, a.spin_limit, &gave_up))) {
                *const_cast<volatile uint32_t*>(&gave_up) = 1;
                if (!join_stuck) join_stuck = !__all_sync(0xFFFFFFFFu, mbar_drain(&joined[turn], join_phases >> turn & 1u));
            }
            join_phases ^= 1u << turn;
            const uint32_t c = lane & (kMaxCluster - 1);
            student = named = RowPart{minus_inf(), 0.0f, 0.0f};
            if (c < ctas) {
                const float4 of = pushed[turn][c];
                student.xmax = of.x;
                student.s = of.y;
                named.xmax = of.z;
                named.s = of.w;
            }
            student.join_slices<kMaxCluster, false>(a.by);
            if (kTail) named.join_lanes<kMaxCluster, false>(kLog2E);
        }
        // the norm of the teacher's values: the warps that have slots find it for themselves
        RowPart teacher{minus_inf(), 0.0f, 0.0f};
        if (!kTail && warp * 32 < a.top) {
            for (uint32_t i = lane; i < a.top; i += 32)
                if (inside(i)) add_value(teacher, t_s[i]);
            __syncwarp();
            teacher.join_lanes<32, false>(kLog2E);
        }
        const bool repeated = repeated_flag != 0;
        const bool no_teacher = !kTail && !weight_flag && !nan_flag;

        // log Z = z_max + log_total; the streamed columns' share p_streamed of the student's distribution (1 unless kTail)
        const float z_streamed = __fmul_rn(student.xmax, a.by.inv_t);
        float z_max = z_streamed, log_total = logf(student.s) + beyond_max(student.xmax, a.by.inv_t, z_streamed);
        float log_streamed = 0.0f, q_rest = 0.0f, t_max = 0.0f, log_norm = 0.0f;
        if (kTail) {
            const float log_s = log_total;
            z_max = fmaxf(z_streamed, named.xmax);
            float total = named.s == 0.0f ? 0.0f : named.s * expf(named.xmax - z_max);
            if (student.s != 0.0f) total += expf((z_streamed - z_max) + log_s);
            log_total = logf(total);
            log_streamed = (z_streamed - z_max) + (log_s - log_total);
            q_rest = q_sum > 1.0f ? 0.0f : 1.0f - q_sum;
        } else {
            t_max = teacher.xmax;                          // (apart from the sum's logarithm, which a common offset would round away)
            log_norm = logf(teacher.s);
        }
        const bool broken = log_total != log_total || nan_flag || gave_up;
        const bool nothing = (!broken && z_max == minus_inf()) || no_teacher;
        const bool remainder = kTail && student.s != 0.0f;
        const bool far = far_off(z_max);
        auto log_p = [&](uint32_t i) {                     // (as less_max: a row without a number is not asked for its log p)
            return (far ? __fadd_rn(__fmul_rn(logit(i), a.by.inv_t), -z_max) : fmaf(logit(i), a.by.inv_t, -z_max)) - log_total;
        };
        auto log_q = [&](uint32_t i) { return (t_s[i] - t_max) - log_norm; };

        if (a.loss_out && rank == 0) {
            float loss = 0.0f;
            for (uint32_t i = tid; i < a.top; i += kThreads)
                if (inside(i)) {
                    const float lq = log_q(i), q = expf(lq);
                    if (q != 0.0f) loss = fmaf(q, lq - log_p(i), loss);
                }
            if (remainder && tid == 0 && q_rest != 0.0f) loss = fmaf(q_rest, logf(q_rest) - log_streamed, loss);
            loss = warp_join<SumOp>(loss);
            if (lane == 0) loss_parts[warp] = broken ? __uint_as_float(0x7FFFFFFFu) : loss;
        }
        T* out = grad + static_cast<size_t>(row_id) * a.ld_grad;
        if (grad) {
            // second reading: 2^((x - xmax) c) times one factor
            const bool aligned = same_boundary(xr, out);
            float factor = scale / student.s;
            if (kTail) factor = remainder ? factor * (expf(log_streamed) - q_rest) : 0.0f;
            if (broken) factor = __uint_as_float(0x7FFFFFFFu);
            auto write_chunks = [&](auto&& two) {
                auto gradient = [&](const uint4& unit, float (&g)[E]) {
#pragma unroll
                    for (uint32_t e = 0; e < E; e += 2)
                        unpack2(two(pack2(Unit<T>::get(unit, e), Unit<T>::get(unit, e + 1))), g[e], g[e + 1]);
                };
                for (uint32_t k = warp; u0 + k * kChunkUnits < u1; k += kWarps) {
                    const uint32_t start = u0 + k * kChunkUnits, first = start + lane;
                    uint4 v[4];
                    const uint4* from = kStaged ? stage + k * kChunkUnits + lane : row.base + first;
                    if (aligned && start + kChunkUnits <= u1 && (!row.ragged || (start >= kChunkUnits && start + kChunkUnits < row.units))) {
                        // a whole chunk inside the row, laid out alike: no unit needs a look
#pragma unroll
                        for (uint32_t i = 0; i < 4; ++i) v[i] = kStaged ? from[32 * i] : ld_unit(from + 32 * i);
                        if (kStaged) {
                            __syncwarp();                  // every lane has its units
                            if (more) fetch_chunk(next_row, next_slice, k);
                        }
                        T* const to = out + row.column(first, 0);
#pragma unroll
                        for (uint32_t i = 0; i < 4; ++i) {
                            float g[E];
                            gradient(v[i], g);
                            // (rows that are loaded twice had better keep L2: 146 and 138 us for 256 rows of 262144 fp32)
                            if (kStaged) st_unit(to + 32 * i * E, Unit<T>::pack(g));
                            else st_unit_stream(to + 32 * i * E, Unit<T>::pack(g));
                        }
                        continue;
                    }
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i)
                        if (first + 32 * i < u1) v[i] = kStaged ? from[32 * i] : ld_unit(from + 32 * i);
                    if (kStaged) {
                        __syncwarp();
                        if (more) fetch_chunk(next_row, next_slice, k);
                    }
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        float g[E];
                        gradient(v[i], g);
                        if (first + 32 * i < u1) store_unit(row, out, first + 32 * i, g, aligned);
                    }
                }
            };
            const float ref = __fmul_rn(student.xmax, a.by.c);
            // (a named column may be far above the others, whose factor this is: it is written again below; staged, it is -inf by now)
            auto powers = [&](uint64_t y) {
                float y0, y1;
                unpack2(y, y0, y1);
                return kTail && !kStaged ? pack2(exp2_fast(fminf(y0, 64.0f)), exp2_fast(fminf(y1, 64.0f))) : pack2(exp2_fast(y0), exp2_fast(y1));
            };
            if (nothing) {                                 // whatever the logits are
                write_chunks([](uint64_t) { return 0ull; });
            } else if (!far_off(z_streamed)) {
                // x c - ref instead of (x - xmax) c, what xmax c is off ref by goes into the factor
                factor *= exp2_fast(-fmaf(student.xmax, a.by.c, -ref));
                const uint64_t by_c = pack2(a.by.c, a.by.c), shift = pack2(-ref, -ref), by_factor = pack2(factor, factor);
                write_chunks([&](uint64_t x) { return mul2(powers(fma2(x, by_c, shift)), by_factor); });
            } else {                                       // (or none but -inf)
                // (rare: one unit after the other, which leaves the other rows' registers alone: 4096 rows of 32768 fp32 182 us, with a third loop
                // like the others 194)
                const float less = z_streamed == minus_inf() ? 0.0f : -z_streamed;
                for (uint32_t k = warp; u0 + k * kChunkUnits < u1; k += kWarps) {
#pragma unroll 1
                    for (uint32_t i = lane; i < kChunkUnits && u0 + k * kChunkUnits + i < u1; i += 32) {
                        const uint32_t u = u0 + k * kChunkUnits + i;
                        const uint4 unit = kStaged ? stage[k * kChunkUnits + i] : ld_unit(row.base + u);
                        float g[E];
#pragma unroll
                        for (uint32_t e = 0; e < E; ++e) {
                            const float y = __fmul_rn(__fadd_rn(__fmul_rn(Unit<T>::get(unit, e), a.by.inv_t), less), kLog2E);
                            g[e] = __fmul_rn(exp2_fast(kTail && !kStaged ? fminf(y, 64.0f) : y), factor);
                        }
                        store_unit(row, out, u, g, aligned);
                    }
                    if (kStaged) {
                        __syncwarp();
                        if (more) fetch_chunk(next_row, next_slice, k);
                    }
                }
            }
        }
        // (a row may have a chunk more than the one before it)
        if (kStaged && more)
            for (uint32_t k = warp; k < a.chunks; k += kWarps)
                if (u0 + k * kChunkUnits >= u1) fetch_chunk(next_row, next_slice, k);
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
        if (tid == 0) {
            repeated_flag = weight_flag = nan_flag = 0;
            if (gave_up && a.result) atomicMax(&a.result->status, static_cast<uint32_t>(DCT_ERR_TIMEOUT));
        }
        if (!more) break;
        row_id += clusters;
    }
    if (kStaged && stuck && lane == 0) copies_settle();
    if (kCluster) {                                        // nobody pushes to a CTA that is gone
        cluster_barrier();
        if (join_stuck) copies_settle();
    }
}

template <typename T, uint32_t kThreads, bool kTail, bool kCluster, bool kStaged>
dct_status_t launch_distill_shape(const void* logits, void* grad, const DistillArgs& a, uint32_t cluster, cudaStream_t stream) {
    const int sms = sm_count();
    if (sms <= 0) return DCT_ERR_CUDA;
    const size_t smem = (kStaged ? static_cast<size_t>(a.chunks) * kChunkBytes : 0) + 4 * static_cast<size_t>(a.mark_words) +
                        20 * static_cast<size_t>(a.top);
    auto kernel = lm_distill_kernel<T, kThreads, kTail, kCluster, kStaged>;
    static SharedLimit allowed;
    const dct_status_t allowed_st = allow_shared(kernel, smem, allowed);
    if (allowed_st != DCT_OK) return allowed_st;
    uint32_t per_sm = static_cast<uint32_t>((227 * 1024) / (smem + 3 * 1024));
    per_sm = per_sm < 1 ? 1 : per_sm < 768 / kThreads ? per_sm : 768 / kThreads;
    const T* x = static_cast<const T*>(logits);
    T* g = static_cast<T*>(grad);
    uint32_t at_once = static_cast<uint32_t>(sms) * per_sm;
    if (kCluster && cluster > 1) {
        static ClusterCounts kept[768 / kThreads + 1];
        const dct_status_t st = clusters_at_once(kernel, kThreads, cluster, smem, kept[per_sm], &at_once);
        if (st != DCT_OK) return st;
    }
    const uint32_t grid = (a.rows < at_once ? a.rows : at_once) * cluster;
    if (kCluster) {
        DCT_CUDA_TRY(launch_clusters(kernel, grid, kThreads, cluster, smem, stream, x, g, a));
    } else {
        kernel<<<grid, kThreads, smem, stream>>>(x, g, a);
        DCT_CUDA_TRY(cudaGetLastError());
    }
    return DCT_OK;
}

template <typename T, bool kTail>
dct_status_t launch_distill(const void* logits, void* grad, DistillArgs a, cudaStream_t stream) {
    const int sms = sm_count();
    if (sms <= 0) return DCT_ERR_CUDA;
    const uint32_t units = a.vocab / Unit<T>::kElems + 2, chunks = (units + kChunkUnits - 1) / kChunkUnits;
    // Slices of at most about 66 KiB leave room for three CTAs of eight warps on an SM; few rows are split further, while each
    // CTA still has a chunk per warp.
    uint32_t cluster = 1;
    while (cluster < kMaxCluster && (chunks > 34 * cluster || (static_cast<uint64_t>(a.rows) * cluster * 2 <= 3ull * sms && chunks >= 16 * cluster)))
        cluster *= 2;
    const uint32_t share = (units + cluster - 1) / cluster;
    a.chunks = (share + kChunkUnits - 1) / kChunkUnits;
    a.mark_words = ((share * Unit<T>::kElems + 31) / 32 + 3) & ~3u;
    a.spin_limit = debug_config().spin_limit;
    const bool staged = static_cast<size_t>(a.chunks) * kChunkBytes + 4 * a.mark_words + 20 * a.top <= kStagedLimit &&
                        a.chunks <= 8 * kMaxChunksPerWarp;
    if (!staged) return launch_distill_shape<T, 256, kTail, true, false>(logits, grad, a, cluster, stream);
    if (cluster > 1) return launch_distill_shape<T, 256, kTail, true, true>(logits, grad, a, cluster, stream);
    // about four chunks to a warp
    if (a.chunks <= 5) return launch_distill_shape<T, 32, kTail, false, true>(logits, grad, a, 1, stream);
    if (a.chunks <= 10) return launch_distill_shape<T, 64, kTail, false, true>(logits, grad, a, 1, stream);
    if (a.chunks <= 20) return launch_distill_shape<T, 128, kTail, false, true>(logits, grad, a, 1, stream);
    return launch_distill_shape<T, 256, kTail, false, true>(logits, grad, a, 1, stream);
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
    const DistillArgs args{rows, vocab, ld, Scale{inv_temperature, log2_scale(inv_temperature)}, teacher_ids, teacher_logprobs, top,
                           grad_loss, loss_out, ld_grad, 0, 0, 0, result};
    auto launch = dtype == DCT_F32
        ? (mode == DCT_DISTILL_TAIL ? launch_distill<float, true> : launch_distill<float, false>)
        : (mode == DCT_DISTILL_TAIL ? launch_distill<__nv_bfloat16, true> : launch_distill<__nv_bfloat16, false>);
    return launch(logits, grad_logits, args, stream);
}
