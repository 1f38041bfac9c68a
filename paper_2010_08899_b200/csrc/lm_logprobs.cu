// Log-probabilities of given tokens, entropy and the most likely columns of rows of logits; and their gradient.
#include "lm_rows.cuh"

namespace dct {
namespace {

constexpr uint32_t kMaxCluster = 8u;
constexpr uint32_t kRankable = 512u;          // the most columns the selection puts in order

struct LogProbArgs {
    uint32_t rows, vocab, ld;
    Scale by;
    const int32_t* tokens;
    uint32_t top;
    float *logprob_out, *entropy_out, *stats_out;
    int32_t* top_ids;
    float* top_logprobs;
    dct_result_t* result;
    uint32_t spin_limit;            // polls a wait for the cluster's other CTAs may take
};

template <uint32_t kThreads> struct LogProbShared {
    static constexpr uint32_t kWarps = kThreads / 32;
    static constexpr uint32_t kGroups = 16;                                        // maxima a thread notes
    static constexpr uint32_t kMaxTop = kThreads;                                  // (half the classes the bound comes from)
    static constexpr uint32_t kCandidates = 8 * kThreads;                          // columns the selection holds
    float group_max[kGroups * kThreads];
    uint64_t candidates[kCandidates];
    uint64_t best[kMaxTop];
    float class_max[2 * kThreads];
    alignas(4) uint16_t hits[kGroups * kThreads];
    RowPart warp_part[2][kWarps];      // by turns, row by row
    float m, logsum;                   // of the whole row
    uint32_t counts[32];
    uint32_t counter, hit_count, bound, tied, gave_up;
};

__device__ __forceinline__ float value_of_key(uint32_t key) {       // the inverse of order_key
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// The selection of a slice's best columns.  A column is (order key << 32 | ~column): larger is better, all distinct.
// While the row streams by, every thread notes the largest element of each pair of units it reads, and that of its even and of
// its odd units.  The kk-th largest of these N = 2 kThreads class maxima is a bound that at least kk columns
// reach and, for kk well below N, not many more do (N ln(N / (N - kk)) for columns in no particular order: 74 for 64 of
// 256); only pairs of units whose noted maximum reaches it are read again, and of them the elements that reach it are put
// in order.
template <typename T, uint32_t kThreads> struct Selector {
    static constexpr uint32_t E = Unit<T>::kElems;
    static constexpr uint32_t kCandidates = LogProbShared<kThreads>::kCandidates;
    RowView<T> row;
    uint32_t u0, u1;                // the slice's units
    uint32_t group_shift;           // log2 of the pairs of units per noted maximum
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
    // By one warp, from the class maxima: a key that at least kk of them reach, and not many more if that can be had
    // (0 if fewer than kk classes have a unit).  tied: many more of them equal it.
    __device__ __forceinline__ uint32_t find_bound(uint32_t kk, bool& tied) const {
        constexpr uint32_t N = 2 * kThreads / 32;
        const uint32_t units = u1 - u0;
        tied = false;
        if (min(units, 2 * kThreads) < kk) return 0;
        uint32_t key[N], lo = 0xFFFFFFFFu, hi = 0;
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) {
            const uint32_t t = i * 32 + lane_id();           // (the class's first unit)
            key[i] = t < units ? order_key(sh.class_max[t]) : 0u;
            lo = min(lo, key[i]);
            hi = max(hi, key[i]);
        }
        lo = __reduce_min_sync(0xFFFFFFFFu, lo);
        hi = __reduce_max_sync(0xFFFFFFFFu, hi);
        // A mask (-inf, the type's lowest value, classes that have no unit) leaves many classes at the least key: the rest is the range, or,
        // if it is fewer than kk, that key is the bound.  (37 rows of 50021 fp32 with twenty columns left: 12.9 us without this, 11.7 with)
        for (uint32_t turn = 0; turn < 2 && lo < order_key(-1.0e30f) && lo < hi; ++turn) {
            uint32_t n = 0, next = 0xFFFFFFFFu;
#pragma unroll
            for (uint32_t i = 0; i < N; ++i) {
                n += key[i] > lo;
                if (key[i] > lo) next = min(next, key[i]);
            }
            n = __reduce_add_sync(0xFFFFFFFFu, n);
            next = __reduce_min_sync(0xFFFFFFFFu, next);
            if (n < kk) hi = lo;
            else lo = next;
        }
        // at least kk classes reach lo, fewer reach hi + 1; a few more than kk are as good as kk.  (Counting the range into 256 parts
        // instead of halving it: no difference for many rows, 0.3 us more for one row, whose code is not in the caches yet.)
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2 + 1;
            uint32_t n = 0;
#pragma unroll
            for (uint32_t i = 0; i < N; ++i) n += key[i] >= mid;
            n = __reduce_add_sync(0xFFFFFFFFu, n);
            if (n >= kk) lo = mid;
            else hi = mid - 1;
            if (n >= kk && n <= kk + kk / 8 + 1) return lo;
        }
        uint32_t n = 0;
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) n += key[i] >= lo;
        tied = __reduce_add_sync(0xFFFFFFFFu, n) > 2 * kk + 8;
        return lo;
    }
    // candidates := the slice's columns with key >= low; returns how many there are, of which the first kCandidates
    // found are stored.  The groups whose maximum reaches the bound are listed first; their units are then dealt out over all
    // threads.
    __device__ __forceinline__ uint32_t collect(uint32_t low) const {
        if (threadIdx.x == 0) sh.counter = sh.hit_count = 0;
        __syncthreads();
        const uint32_t group_units = 2u << group_shift, span = group_units * kThreads;
        // (the order of floats and of keys is the same from -inf up; below that, everything is a candidate)
        const bool all = low <= 0x007FFFFFu;
        const float low_value = value_of_key(low);
        const uint32_t groups = group_shift ? (u1 - u0 + span - 1) / span : (u1 - u0 + 2 * span - 1) / (2 * span) * 2;
        uint32_t mine = 0;
#pragma unroll
        for (uint32_t g = 0; g < sh.kGroups; ++g)
            mine |= static_cast<uint32_t>(g < groups && (all || sh.group_max[g * kThreads + threadIdx.x] >= low_value)) << g;
        if (mine) {
            uint32_t at = atomicAdd(&sh.hit_count, static_cast<uint32_t>(__popc(mine)));
            for (; mine; mine &= mine - 1) sh.hits[at++] = static_cast<uint16_t>((__ffs(mine) - 1) * kThreads + threadIdx.x);
        }
        __syncthreads();
        const uint32_t unit_shift = group_shift + 1, items = sh.hit_count << unit_shift;
        for (uint32_t item0 = threadIdx.x; item0 < items; item0 += 2 * kThreads) {
            uint4 v[2];
            uint32_t us[2];
#pragma unroll
            for (uint32_t q = 0; q < 2; ++q) {
                const uint32_t item = item0 + q * kThreads;
                us[q] = 0xFFFFFFFFu;
                if (item < items) {
                    const uint32_t slot = sh.hits[item >> unit_shift];
                    const uint32_t g = slot / kThreads, j = item & (group_units - 1);
                    // (a pair is the first and third or the second and fourth unit of a batch, a larger group whole batches)
                    const uint32_t at = group_shift ? g * group_units + j : (g >> 1) * 4 + (g & 1) + 2 * j;
                    const uint32_t u = u0 + at * kThreads + slot % kThreads;
                    if (u < u1) {
                        us[q] = u;
                        v[q] = ld_unit(row.base + u);
                    }
                }
            }
#pragma unroll
            for (uint32_t q = 0; q < 2; ++q) {
                if (us[q] == 0xFFFFFFFFu) continue;
                uint32_t found = 0;
#pragma unroll
                for (uint32_t i = 0; i < E; ++i)
                    found |= static_cast<uint32_t>(all ? order_key(Unit<T>::get(v[q], i)) >= low : Unit<T>::get(v[q], i) >= low_value) << i;
                if (row.ragged && row.at_an_end(us[q])) {
#pragma unroll
                    for (uint32_t i = 0; i < E; ++i)
                        if (row.column(us[q], i) >= row.width) found &= ~(1u << i);
                }
                if (!found) continue;
                uint32_t at = atomicAdd(&sh.counter, static_cast<uint32_t>(__popc(found)));
#pragma unroll
                for (uint32_t i = 0; i < E; ++i)
                    if (found >> i & 1u) {
                        if (at < kCandidates) sh.candidates[at] = entry(order_key(Unit<T>::get(v[q], i)), row.column(us[q], i));
                        ++at;
                    }
            }
        }
        __syncthreads();
        const uint32_t n = sh.counter;
        __syncthreads();                       // (the counters may be set anew)
        return n;
    }
    // the kk-th largest key of the slice, by halving the range of keys: 32 passes
    __device__ __noinline__ static uint32_t kth_key(const Selector s, uint32_t kk) {
        uint32_t lo = 0, hi = 0xFFFFFFFFu;
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2 + 1;
            uint32_t n = 0;
            for (uint32_t u = s.u0 + threadIdx.x; u < s.u1; u += kThreads)
                s.each_element(u, [&](uint32_t key, uint32_t) { n += key >= mid; });
            if (cta_count(n, s.sh.counts) >= kk) lo = mid;
            else hi = mid - 1;
        }
        return lo;
    }
    // appends the lowest columns whose key is `key` until there are kk candidates; returns how many there are then
    __device__ __noinline__ static uint32_t fill_with_equals(const Selector s, uint32_t key, uint32_t have, uint32_t kk) {
        for (uint32_t first = s.u0; first < s.u1 && have < kk; first += kThreads) {
            const uint32_t u = first + threadIdx.x;
            uint32_t mine = 0;
            if (u < s.u1) s.each_element(u, [&](uint32_t k, uint32_t) { mine += k == key; });
            uint32_t before = mine;                         // inclusive sum over the lanes
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t t = __shfl_up_sync(0xFFFFFFFFu, before, o);
                if (lane_id() >= static_cast<uint32_t>(o)) before += t;
            }
            __syncthreads();
            if (lane_id() == 31) s.sh.counts[threadIdx.x >> 5] = before;
            __syncthreads();
            uint32_t at = have + before - mine, all = 0;
            for (uint32_t w = 0; w < kThreads / 32; ++w) {
                if (w < (threadIdx.x >> 5)) at += s.sh.counts[w];
                all += s.sh.counts[w];
            }
            if (u < s.u1 && mine)
                s.each_element(u, [&](uint32_t k, uint32_t col) {
                    if (k == key) {
                        if (at < kk) s.sh.candidates[at] = entry(key, col);
                        ++at;
                    }
                });
            have += all;
        }
        __syncthreads();
        return min(have, kk);
    }
    // keeps the kk best of n candidates, kk < n, in no order
    __device__ __noinline__ static void cut(LogProbShared<kThreads>& sh, uint32_t n, uint32_t kk) {
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
    // best[0 .. kk) := the kk best of n <= kRankable candidates in order.  Every warp sorts runs of 32 in its registers;
    // an entry's place is how many entries of each run are better, by bisection.
    __device__ __forceinline__ void in_order(uint32_t n, uint32_t kk) const {
        const uint32_t runs = (n + 31) / 32, lane = lane_id();
        for (uint32_t run = threadIdx.x >> 5; run < runs; run += kThreads / 32) {
            uint64_t key = run * 32 + lane < n ? sh.candidates[run * 32 + lane] : 0ull;
#pragma unroll
            for (uint32_t size = 2; size <= 32; size *= 2)
#pragma unroll
                for (uint32_t step = size / 2; step > 0; step /= 2) {
                    const uint64_t other = __shfl_xor_sync(0xFFFFFFFFu, key, step);
                    const bool keep_larger = ((lane & step) == 0) == ((lane & size) == 0 || size == 32);
                    key = (key > other) == keep_larger ? key : other;
                }
            sh.candidates[run * 32 + lane] = key;                 // (kCandidates is a multiple of 32)
        }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
            const uint64_t key = sh.candidates[i];
            uint32_t place = 0;
#pragma unroll 4
            for (uint32_t run = 0; run < runs; ++run) {
                const uint64_t* list = sh.candidates + run * 32;
                uint32_t better = 0;
#pragma unroll
                for (uint32_t step = 16; step > 0; step /= 2)
                    if (list[better + step - 1] > key) better += step;
                place += better + (list[better] > key);
            }
            if (place < kk) sh.best[place] = key;
        }
        __syncthreads();
    }
    // best[0 .. kk) := the slice's kk best columns in order.  The class maxima are in class_max.
    __device__ __forceinline__ void run(uint32_t kk) const {
        if (threadIdx.x < 32) {
            bool tied;
            const uint32_t b = find_bound(kk, tied);
            if (threadIdx.x == 0) {
                sh.bound = b;
                sh.tied = tied;
            }
        }
        __syncthreads();
        // (rows that a mask leaves little of: the columns that equal the bound are too many to look at, their lowest few will do)
        bool above = sh.tied;                  // the candidates are the columns above the bound
        uint32_t bound = sh.bound, low = bound + above, n;
        for (;;) {
            n = collect(low);
            if (n < kk && !above && bound != 0) {        // classes whose only elements lie outside the row or are NaN
                bound = low = 0;
            } else if (n > kCandidates) {                // many equal to the bound, or sorted columns
                if (above) bound = kth_key(*this, kk);
                above = true;
                low = bound + 1;                         // (0xFFFFFFFF is no element's key)
            } else {
                break;
            }
        }
        if (n < kk) {
            n = fill_with_equals(*this, bound, n, kk);
            if (n < kk) fill_with_equals(*this, 0, n, kk);       // NaN: some class of the bound had nothing else
            n = kk;
        }
        if (n > kRankable) {
            cut(sh, n, kk);
            n = kk;
        }
        in_order(n, kk);
    }
};

// One thread: the row's m and log sum, and the results that are numbers per row.  x: the logit of the token (any number if that is
// none of the row's).
__device__ __forceinline__ void write_row(const LogProbArgs& a, uint32_t row_id, float x, int32_t tok, const RowPart& all,
                                          float& m_out, float& logsum_out) {
    const float m = __fmul_rn(all.xmax, a.by.inv_t);
    const bool empty = m == minus_inf() && all.s == all.s;
    // (s belongs to the exact product xmax / T: the rounding of m goes into the logarithm)
    const float log_s = logf(all.s), logsum = empty ? 0.0f : log_s + beyond_max(all.xmax, a.by.inv_t, m);
    m_out = m;
    logsum_out = logsum;
    if (a.tokens) {
        float lp = 0.0f;
        if (tok >= 0 && static_cast<uint32_t>(tok) < a.vocab) {
            lp = less_max(x, a.by.inv_t, m) - logsum;
        } else if (tok >= 0 && a.result) {
            atomicMax(&a.result->status, static_cast<uint32_t>(DCT_ERR_BAD_MASK));
        }
        a.logprob_out[row_id] = lp;
    }
    if (a.entropy_out) a.entropy_out[row_id] = empty ? 0.0f : fmaf(-kLn2, all.st / all.s, log_s);
    if (a.stats_out) {
        a.stats_out[2 * static_cast<size_t>(row_id)] = m;
        a.stats_out[2 * static_cast<size_t>(row_id) + 1] = logsum;
    }
}

// log p_j = z_j - m - s, entropy = s - mean of (z - m), and the `top` best columns, from one reading of the logits.
// A cluster of CTAs takes a row, each CTA a slice of its units; the CTAs join their sums and their ordered best columns
// through each other's shared memory.
// What bounds it: without alternatives reading, 4096 rows of 32768 bf16 in 50 us (5.4 TB/s), fp32 in 88 us (6.1 TB/s).  With 64
// alternatives bf16 takes 71 us: 10 instructions per element and thread in all, and after the reading the selection's short phases
// one after the other (bound, list, some 80 pairs read again, order), which only other CTAs on the SM fill.  So it is the
// number of warps that counts: 32 to an SM 71 us, 28 73 us, 20 with a batch loaded ahead into registers 88 us; bringing the next row
// into L2 during the selection made it 77, as the selection's own random reads waited longer.
template <typename T, uint32_t kThreads, bool kCluster>
__global__ void __launch_bounds__(kThreads, kThreads <= 128 ? 1024 / kThreads : 4)
lm_logprobs_kernel(const T* __restrict__ logits, const LogProbArgs a) {
    constexpr uint32_t kWarps = kThreads / 32;
    __shared__ LogProbShared<kThreads> sh;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = lane_id();
    const uint32_t rank = kCluster ? cluster_rank() : 0u, ctas = kCluster ? cluster_size() : 1u;
    const uint32_t clusters = gridDim.x / ctas;
    // kCluster: every CTA pushes the sums of its slice, and its best columns in order, to all.  (Nobody pushes a row's before all
    // have read the last row's: that is what the cluster's barrier is for.  It is met long before it is waited for.)
    extern __shared__ __align__(16) uint64_t lists[];                  // [ctas][top]
    __shared__ __align__(16) float4 pushed[kMaxCluster];
    __shared__ uint64_t joined;
    if (kCluster) {
        if (tid == 0) {
            sh.gave_up = 0;
            mbar_init(&joined, 1);
            mbar_init_fence();
        }
        cluster_arrive();
    }
    uint32_t turn = 0;
    bool stuck = false;                   // the others' numbers did not come at all
    for (uint32_t row_id = blockIdx.x / ctas;; turn ^= 1) {
        const T* xr = logits + static_cast<size_t>(row_id) * a.ld;
        const RowView<T> row(xr, a.vocab);
        const Slice slice(row.units, rank, ctas);
        const uint32_t u0 = slice.u0, u1 = slice.u1;
        // what the row's token is like, for the thread that will write its log-probability
        int32_t tok = -1;
        if (a.tokens && tid == kThreads - 32) tok = a.tokens[row_id];

        // one pass: sums, and the largest element of every batch of four units
        RowSums sums;
        uint32_t group_shift = 0;
        while ((u1 - u0 + (2 * kThreads << group_shift) - 1) / (2 * kThreads << group_shift) > sh.kGroups) ++group_shift;
        float max0 = minus_inf(), max1 = minus_inf(), group_max = minus_inf();
        uint32_t in_group = 1u << group_shift, slot = tid;
        stream_units<T, kThreads>(row, u0, u1, [&](const uint4 (&v)[4], uint32_t) {
            const float best0 = Unit<T>::best(v[0], v[2]), best1 = Unit<T>::best(v[1], v[3]), best = fmaxf(best0, best1);
            sums.add<T, true>(v, best, a.by.c);
            max0 = fmaxf(max0, best0);
            max1 = fmaxf(max1, best1);
            if (group_shift == 0) {                                  // the same for the whole CTA
                sh.group_max[slot] = best0;
                if (slot + kThreads < sh.kGroups * kThreads) sh.group_max[slot + kThreads] = best1;
                slot += 2 * kThreads;
            } else {
                group_max = fmaxf(group_max, best);
                sh.group_max[slot] = group_max;                      // (written again until the group is complete)
                if ((in_group -= 2) == 0) {
                    group_max = minus_inf();
                    in_group = 1u << group_shift;
                    slot += kThreads;
                }
            }
        });
        if (a.top) {
            sh.class_max[tid] = max0;
            sh.class_max[kThreads + tid] = max1;
        }
        const RowPart mine = sums.part<true>(warp_max(fmaxf(max0, max1)), a.by.c);
        if (lane == 0) sh.warp_part[turn][warp] = mine;
        __syncthreads();
        // a row that is far off (the same for the whole CTA) is summed again, by all warps
        const float x_slice = warp_max(sh.warp_part[turn][lane & (kWarps - 1)].xmax);
        if (x_slice > minus_inf() && far_off(__fmul_rn(x_slice, a.by.inv_t))) {
            const RowPart share = far_part(row, u0 + warp * 32, kThreads, u1, x_slice, a.by, [](uint32_t, uint32_t) { return true; });
            __syncthreads();                                         // (the parts' largest have been read)
            if (lane == 0) sh.warp_part[turn][warp] = share;
            __syncthreads();
        }

        float x_tok = 0.0f;
        if (tid == kThreads - 32 && tok >= 0 && static_cast<uint32_t>(tok) < a.vocab) x_tok = to_f32(xr[tok]);
        if (kCluster) {
            cluster_wait();
            if (tid == 0 && !stuck) {
                uint32_t listed = 0;
                for (uint32_t c = 0; c < ctas; ++c)
                    if (c != rank) listed += min(a.top, Slice(row.units, c, ctas).columns(row));
                mbar_arrive_expect_tx(&joined, 16 * ctas + 8 * listed);
            }
        }
        // the last warp joins the slice's sums (and writes the results of a row that is one slice); the first meanwhile looks
        // for the bound of the selection
        if (warp == kWarps - 1) {
            RowPart all = sh.warp_part[turn][lane & (kWarps - 1)];
            all.join_lanes<kWarps, true>(a.by.c);
            if (kCluster) {
                if (lane < ctas) push_remote(remote_smem(&pushed[rank], lane), all.xmax, all.s, all.st, 0.0f, remote_smem(&joined, lane));
            } else if (lane == 0) {
                write_row(a, row_id, x_tok, tok, all, sh.m, sh.logsum);
            }
        }
        uint32_t kept = 0;
        if (a.top) {
            kept = min(a.top, slice.columns(row));
            if (kept) Selector<T, kThreads>{row, u0, u1, group_shift, sh}.run(kept);
        }

        uint32_t* const places = reinterpret_cast<uint32_t*>(sh.hits);      // no longer in use
        if (kCluster) {
            for (uint32_t item = tid; item < ctas * kept; item += kThreads) {
                const uint32_t c = item / kept, i = item % kept;
                if (c != rank) push_remote(remote_smem(&lists[rank * a.top + i], c), sh.best[i], remote_smem(&joined, c));
            }
            for (uint32_t i = tid; i < kept; i += kThreads) places[i] = i;
            if (stuck || !mbar_wait_bounded(&joined, turn, a.spin_limit, &sh.gave_up)) {
                *const_cast<volatile uint32_t*>(&sh.gave_up) = 1;                // this row and the rest become NaN
                if (!stuck) stuck = !mbar_drain(&joined, turn);
            }
            __syncthreads();
            if (warp == kWarps - 1) {
                RowPart all{minus_inf(), 0.0f, 0.0f};
                const uint32_t c = lane & (kMaxCluster - 1);
                if (c < ctas) {
                    const float4 of = pushed[c];
                    all = RowPart{of.x, sh.gave_up ? __uint_as_float(0x7FFFFFFFu) : of.y, of.z};
                }
                all.join_slices<kMaxCluster, true>(a.by);
                if (lane == 0) {
                    LogProbArgs mine = a;
                    if (rank != 0) {
                        mine.tokens = nullptr;
                        mine.entropy_out = mine.stats_out = nullptr;
                    }
                    if (sh.gave_up && a.result) atomicMax(&a.result->status, static_cast<uint32_t>(DCT_ERR_TIMEOUT));
                    write_row(mine, row_id, x_tok, tok, all, sh.m, sh.logsum);
                }
            }
            // a column's place: its place in its own slice's list, and how many of each other list are better
            for (uint32_t item = tid; item < ctas * kept; item += kThreads) {
                const uint32_t c = item / kept, i = item % kept;
                if (c == rank) continue;
                const uint64_t key = sh.best[i], *list = lists + c * a.top;
                uint32_t lo = 0, hi = min(a.top, Slice(row.units, c, ctas).columns(row));         // list[0 .. lo) are better
                while (lo < hi) {
                    const uint32_t mid = (lo + hi) / 2;
                    if (list[mid] > key) lo = mid + 1;
                    else hi = mid;
                }
                if (lo) atomicAdd(&places[i], lo);
            }
            __syncthreads();
            cluster_arrive();             // what the others pushed has been read
        }
        for (uint32_t i = tid; i < kept; i += kThreads) {
            const uint64_t key = sh.best[i];
            const uint32_t place = kCluster ? places[i] : i;
            if (place < a.top) {
                const size_t at = static_cast<size_t>(row_id) * a.top + place;
                a.top_ids[at] = static_cast<int32_t>(0xFFFFFFFFu - static_cast<uint32_t>(key));
                a.top_logprobs[at] = less_max(value_of_key(static_cast<uint32_t>(key >> 32)), a.by.inv_t, sh.m) - sh.logsum;
            }
        }
        // (No barrier: the warps' parts alternate, and what else the next row writes it writes behind its first barrier.)
        if (a.rows - row_id <= clusters) break;
        row_id += clusters;
    }
    if (kCluster) {                       // nobody pushes to a CTA that is gone
        cluster_wait();
        if (stuck) copies_settle();
    }
}

// grad_j = (1 / T) (a (1[j = token] - p_j) - c p_j (log p_j + entropy)), elementwise: a CTA takes four units per thread of one
// row.  p comes from the saved m and log sum, so no row is summed again; the product with log2 e is a step of its own here (log p
// itself is needed to fp32 accuracy).  Memory bound: 1023 rows of 50021 fp32 at a stride of 50048 in 62 us, 4096 of 32768 bf16 in 80 us (both 6.6 TB/s);
// where the gradient lies off the logits' 16-byte boundaries it is stored element by element (306 us).
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
        // z - m as the forward call forms it: the product with 1 / T by the fma, or (rows far off) rounded before it; the other factor
        // is 1 (and known only here: a product and a sum of pairs would come out as one fma again)
        const float before = far_off(ref) ? q.inv_t : 1.0f, within = far_off(ref) ? 1.0f : q.inv_t;
        const uint64_t first_scale = pack2(before, before), then_scale = pack2(within, within);
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
                const uint64_t x = mul2(pack2(Unit<T>::get(v[i], e), Unit<T>::get(v[i], e + 1)), first_scale);
                unpack2(add2(fma2(x, then_scale, shift), less), l0, l1);
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
dct_status_t launch_logprobs_threads(const void* logits, const LogProbArgs& a, uint32_t cluster, uint32_t ctas, cudaStream_t stream) {
    const T* x = static_cast<const T*>(logits);
    if constexpr (kThreads == 256) {
        if (cluster > 1) {
            static SharedLimit allowed;
            static ClusterCounts kept[2];
            auto kernel = lm_logprobs_kernel<T, kThreads, true>;
            const bool many = a.top > 128;            // room for the lists: 8 CTAs' of 128 columns leave four CTAs to an SM
            const size_t smem = static_cast<size_t>(cluster) * (many ? 256 : 128) * sizeof(uint64_t);
            dct_status_t st = allow_shared(kernel, smem, allowed, 0);
            if (st != DCT_OK) return st;
            uint32_t at_once = 1;
            st = clusters_at_once(kernel, kThreads, cluster, smem, kept[many], &at_once);
            if (st != DCT_OK) return st;
            DCT_CUDA_TRY(launch_clusters(kernel, (a.rows < at_once ? a.rows : at_once) * cluster, kThreads, cluster, smem, stream, x, a));
            return DCT_OK;
        }
    }
    lm_logprobs_kernel<T, kThreads, false><<<a.rows < ctas ? a.rows : ctas, kThreads, 0, stream>>>(x, a);
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}

template <typename T> dct_status_t launch_logprobs(const void* logits, const LogProbArgs& a, cudaStream_t stream) {
    const int sms = sm_count();
    if (sms <= 0) return DCT_ERR_CUDA;
    const uint32_t units = (a.vocab + Unit<T>::kElems - 1) / Unit<T>::kElems;
    // Threads to a row's CTA, and CTAs to a row: the shape with the least estimated time, in tenths of a microsecond.  A round of
    // CTAs takes what the end of a row costs (join, selection, order; more warps to a row make it shorter but fewer rows share
    // it) and 0.9 us for each batch of four units per thread.  Measured at both ends: 16384 rows of 4096 bf16, top 20: 46 / 66 /
    // 89 / 217 us with 32 / 64 / 128 / 256 threads; 1000 rows of 131072: 137 / 82 / 56 / 63; one row of 32768: 23 / 15 / 10 / 7.8.
    // Splitting a row costs the exchange of the lists, and the more CTAs share an SM the longer their ends take: one row of 32768
    // with 1 / 2 / 4 / 8 CTAs 7.8 / 8.2 / 7.3 / 8.6 us, 100 rows 10.0 / 8.9 / 10.5 / 18.4; one row of 131072 16.6 / 12.6 / 9.5 / 8.4, 64 rows
    // 22.0 / 16.8 / 13.5 / 12.4; 8 rows of 131072 with the top 256 23.0 / 17.7 / 16.0 / 17.5.
    // A selection wants twice as many classes as columns; where the row has many batches, more threads to it are better
    // still (4096 rows of 32768, top 64: 79 us with 64 threads, 71 with 128; 8192 of 8192: 61 and 71).
    uint32_t threads = 256, cluster = 1;
    uint64_t best = ~0ull;
    for (uint32_t t = 32; t <= 256; t *= 2) {
        if (t < 256 && (a.top > t || (a.top > t / 2 && units > 32 * t))) continue;
        const uint64_t slots = static_cast<uint64_t>(sms) * (t <= 128 ? 1024 / t : 4);
        for (uint32_t c = 1; c <= kMaxCluster && (c == 1 || (t == 256 && units / c >= 512)); c *= 2) {
            const uint64_t fit = c == 1 ? slots : slots * 7 / 8;              // (a GPC's SMs are no multiple of a cluster)
            const uint64_t rounds = (static_cast<uint64_t>(a.rows) * c + fit - 1) / fit;
            const uint64_t shared = t < 256 ? 0 : 4ull * a.rows * c >= 16ull * sms ? 16 : 4ull * a.rows * c / sms;
            const uint64_t end = a.top ? (t == 32 ? 100 : t == 64 ? 70 : t == 128 ? 55 : 60) + 50 * a.top / t + shared +
                                             (c == 1 ? 0 : (c == 2 ? 13 : c == 4 ? 19 : 27) + a.top * c / 64)
                                       : (t == 32 ? 40 : t == 64 ? 30 : t == 128 ? 20 : 25) + (c > 1 ? 10 : 0);
            const uint64_t cost = rounds * (end + 9 * ((units / c + 4 * t - 1) / (4 * t)));
            if (cost < best) {
                best = cost;
                threads = t;
                cluster = c;
            }
        }
    }
    const uint32_t ctas = static_cast<uint32_t>(sms) * (threads <= 128 ? 1024 / threads : 4);
    if (threads == 32) return launch_logprobs_threads<T, 32>(logits, a, 1, ctas, stream);
    if (threads == 64) return launch_logprobs_threads<T, 64>(logits, a, 1, ctas, stream);
    if (threads == 128) return launch_logprobs_threads<T, 128>(logits, a, 1, ctas, stream);
    return launch_logprobs_threads<T, 256>(logits, a, cluster, ctas, stream);
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
    const LogProbArgs args{rows, vocab, ld, Scale{inv_temperature, log2_scale(inv_temperature)}, tokens, top, logprob_out, entropy_out, stats_out, top_ids, top_logprobs, result,
                           debug_config().spin_limit};
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
