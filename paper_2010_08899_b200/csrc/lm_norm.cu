// Layer norm forward and backward.
//
// Which kernel takes which width (units of 16 bytes, 8 bf16 or 4 fp32, to a row):
//   up to 32     8, 16 or 32 lanes to a row, four sets of rows at a time (norm_*_narrow_kernel)
//   up to 128    a warp to a row (bf16 backward beyond 64: a CTA)      } norm_fwd_ring_kernel, norm_bwd_units_kernel:
//   up to 2048   a CTA to a row (bf16 backward up to 1024)             } rows through a ring of bulk copies
//   beyond       a CTA to a row that is read again for every sum (norm_fwd_kernel, norm_bwd_kernel, norm_param_parts_kernel);
//                bf16 rows of 1025 to 2048 units with fp32 parameters go forward in registers without a ring (norm_fwd_units_kernel)
// Memory bound: 2 and 3 times the matrix cross the bus.  In a replayed graph (a call of its own adds the launch, 5 us), 16384 rows of 4096 bf16:
// forward 45.5 us (5.9 TB/s), backward 67 us with the parameters' gradients (6.0 TB/s) and 62 us without; fp32 forward 90 us (6.0), backward
// 122 us (6.6).  Rows off the 16-byte boundaries are bound by instructions: 16384 rows of 4095 bf16 72 and 99 us.
#include "lm_rows.cuh"

namespace dct {
namespace {

constexpr uint32_t kNormMaxWidth = 65536u;
constexpr uint32_t kNormThreads = 256u;
constexpr uint32_t kMaxParts = 148u * 6u;        // CTAs that leave partial sums of the parameter gradients, at most
constexpr size_t kMostShared = 226 * 1024;       // dynamic shared memory a CTA may ask for: 227 KiB less what it holds statically

// Rows as units of 16 bytes counted from the row's own first element.  Where a row does not start on a 16-byte boundary, a unit is
// put together from the two aligned pieces it lies in; these are inside the row but for the bytes next to its ends, which share
// a 16-byte piece (and so a page) with it.

// the 16 bytes that start `by` bytes into a, b (by = 0, 2, ... 14)
__device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, uint32_t by) {
    uint32_t w0 = a.x, w1 = a.y, w2 = a.z, w3 = a.w, w4 = b.x, w5 = b.y, w6 = b.z;
    const uint32_t w7 = b.w;
    if (by & 8u) { w0 = w2; w1 = w3; w2 = w4; w3 = w5; w4 = w6; w5 = w7; }
    if (by & 4u) { w0 = w1; w1 = w2; w2 = w3; w3 = w4; w4 = w5; }
    const uint32_t bits = (by & 2u) * 8u;
    return make_uint4(__funnelshift_r(w0, w1, bits), __funnelshift_r(w1, w2, bits), __funnelshift_r(w2, w3, bits),
                      __funnelshift_r(w3, w4, bits));
}

template <typename T> struct NormRow {
    const uint4* base;         // the boundary at or before the row's first element
    uint32_t off;              // bytes from there to it
    uint32_t pieces;           // aligned pieces that hold a part of the row
    __device__ __forceinline__ NormRow(const T* row, uint32_t d) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(row);
        off = static_cast<uint32_t>(at & 15u);
        base = reinterpret_cast<const uint4*>(at & ~static_cast<uintptr_t>(15));
        pieces = (off + d * static_cast<uint32_t>(sizeof(T)) + 15) / 16;
    }
};
// A group of threads works on one row: a warp (kGroup = 32), or the CTA (kGroup = 0; as many warps as the row's width wants, up to 16).
template <uint32_t kGroup> __device__ __forceinline__ uint32_t group_size() { return kGroup ? kGroup : blockDim.x; }
template <uint32_t kGroup> __device__ __forceinline__ void group_sync() {
    if (kGroup == 32) __syncwarp();
    else __syncthreads();
}
// units lane, lane + group size, ... of a row whose aligned pieces ld reads (from global or shared memory), all loads before any use;
// elements past the row's end are whatever lies there.  kWhole, here and below: the group's lanes hold exactly the row's units, all
// of them whole, and every row starts on a 16-byte boundary.
template <uint32_t kGroup, uint32_t kUnits, bool kWhole, typename Ld>
__device__ __forceinline__ void load_units(uint4 (&v)[kUnits], uint32_t lane, uint32_t units, uint32_t off, uint32_t pieces, Ld&& ld) {
#pragma unroll
    for (uint32_t i = 0; i < kUnits; ++i) v[i] = ld(kWhole ? lane + i * group_size<kGroup>() : min(lane + i * group_size<kGroup>(), units - 1));
    if constexpr (!kWhole) {
        if (off == 0) return;
        uint4 b[kUnits];
#pragma unroll
        for (uint32_t i = 0; i < kUnits; ++i) b[i] = ld(min(lane + i * group_size<kGroup>() + 1, pieces - 1));     // (a last piece again: not used)
#pragma unroll
        for (uint32_t i = 0; i < kUnits; ++i) v[i] = shifted(v[i], b[i], off);
    }
}
// the unit's elements in pairs; those at and past `left` (elements of the row from the unit's first on) become `fill`
template <typename T>
__device__ __forceinline__ void unit_pairs(const uint4& v, uint32_t left, float fill, uint64_t (&x)[Unit<T>::kElems / 2]) {
    constexpr uint32_t E = Unit<T>::kElems;
#pragma unroll
    for (uint32_t e = 0; e < E; e += 2) x[e / 2] = pack2(Unit<T>::get(v, e), Unit<T>::get(v, e + 1));
    if (left < E) {
#pragma unroll
        for (uint32_t e = 0; e < E; e += 2) {
            float p, q;
            unpack2(x[e / 2], p, q);
            x[e / 2] = pack2(e < left ? p : fill, e + 1 < left ? q : fill);
        }
    }
}
// kE parameters from column `col` on as pairs, `fill` past the end or without an array.  whole: there is an array on a 16-byte
// boundary and every unit of the row is whole; vector: the former alone (both the same for all threads)
template <typename P, uint32_t kE>
__device__ __forceinline__ void param_pairs(const P* params, bool whole, bool vector, uint32_t col, uint32_t d, float fill,
                                            uint64_t (&x)[kE / 2]) {
    if (whole) {
        col = min(col, d - kE);
    } else if (!vector || col + kE > d) {
#pragma unroll
        for (uint32_t e = 0; e < kE; e += 2)
            x[e / 2] = pack2(params && col + e < d ? to_f32(params[col + e]) : fill,
                             params && col + e + 1 < d ? to_f32(params[col + e + 1]) : fill);
        return;
    }
    if constexpr (kE * sizeof(P) >= 16) {
#pragma unroll
        for (uint32_t q = 0; q < kE * sizeof(P) / 16; ++q) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(params + col) + q);
#pragma unroll
            for (uint32_t e = 0; e < Unit<P>::kElems; e += 2)
                x[q * Unit<P>::kElems / 2 + e / 2] = pack2(Unit<P>::get(v, e), Unit<P>::get(v, e + 1));
        }
    } else {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(params + col));           // four bf16
        const uint4 w = make_uint4(v.x, v.y, 0, 0);
#pragma unroll
        for (uint32_t e = 0; e < kE; e += 2) x[e / 2] = pack2(Unit<P>::get(w, e), Unit<P>::get(w, e + 1));
    }
}

template <typename P> __device__ __forceinline__ bool vector_params(const P* params) {
    return params && (reinterpret_cast<uintptr_t>(params) & 15u) == 0;
}

// sums of a and b over the group, the same in every thread.  slots: 2 x 2 x 32 floats of the group, `turn` alternates from call to
// call (so that one barrier is enough).
template <uint32_t kGroup>
__device__ __forceinline__ void group_sums(float& a, float& b, float* slots, uint32_t turn) {
    a = warp_join<SumOp>(a);
    b = warp_join<SumOp>(b);
    if (kGroup == 32) return;
    float* s = slots + (turn & 1u) * 64;
    const uint32_t warps = blockDim.x / 32, lane = lane_id(), w = lane & 15u;
    if (lane == 0) {
        s[threadIdx.x >> 5] = a;
        s[32 + (threadIdx.x >> 5)] = b;
    }
    __syncthreads();
    a = w < warps ? s[w] : 0.0f;
    b = w < warps ? s[32 + w] : 0.0f;
#pragma unroll
    for (uint32_t o = 8; o > 0; o >>= 1) {
        a = __fadd_rn(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
        b = __fadd_rn(b, __shfl_xor_sync(0xFFFFFFFFu, b, o));
    }
}
template <uint32_t kGroup> __device__ __forceinline__ void group_sum(float& a, float* slots, uint32_t turn) {
    a = warp_join<SumOp>(a);
    if (kGroup == 32) return;
    float* s = slots + (turn & 1u) * 64;
    const uint32_t warps = blockDim.x / 32, lane = lane_id(), w = lane & 15u;
    if (lane == 0) s[threadIdx.x >> 5] = a;
    __syncthreads();
    a = w < warps ? s[w] : 0.0f;
#pragma unroll
    for (uint32_t o = 8; o > 0; o >>= 1) a = __fadd_rn(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
}

// A row of d results of a group.  A row on a 16-byte boundary is written unit by unit; another one is laid out in shared memory as it
// lies against the boundaries (`image`) and its whole aligned pieces are stored by one bulk copy.  Two images take turns: a copy
// has read one by the time the row after the next writes it.
template <typename T, uint32_t kGroup, bool kWhole> struct RowWriter {
    static constexpr uint32_t E = Unit<T>::kElems;
    T* row;
    uint32_t d, off;
    uint32_t* image;
    __device__ __forceinline__ RowWriter(T* row_, uint32_t d_, uint4* images, uint32_t image_units, uint32_t turn)
        : row(row_), d(d_), off(kWhole ? 0u : static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row_) & 15u)),
          image(reinterpret_cast<uint32_t*>(images + (turn & 1u) * image_units)) {}
    // by all lanes of a warp, for neighbouring units
    __device__ __forceinline__ void put(uint32_t u, const uint4& v) {
        if (off) {
            uint32_t* to = image + off / 4 + 4 * u;
            const bool mine = u * E < d;
            if (off & 2u) {          // bf16 half a word off: a word holds the end of one pair and the start of the next
                const uint32_t before = __shfl_up_sync(0xFFFFFFFFu, v.w, 1);
                if (mine) {
                    if (lane_id() == 0) reinterpret_cast<uint16_t*>(to)[1] = static_cast<uint16_t>(v.x);
                    else to[0] = __funnelshift_r(before, v.x, 16);
                    to[1] = __funnelshift_r(v.x, v.y, 16);
                    to[2] = __funnelshift_r(v.y, v.z, 16);
                    to[3] = __funnelshift_r(v.z, v.w, 16);
                    if (lane_id() == 31 || (u + 1) * E >= d) reinterpret_cast<uint16_t*>(to + 4)[0] = static_cast<uint16_t>(v.w >> 16);
                }
            } else if (mine) {
                to[0] = v.x;
                to[1] = v.y;
                to[2] = v.z;
                to[3] = v.w;
            }
        } else if (kWhole || u * E + E <= d) {
            st_unit(row + u * E, v);
        } else {
#pragma unroll
            for (uint32_t e = 0; e < E; ++e)
                if (u * E + e < d) row[u * E + e] = from_f32<T>(Unit<T>::get(v, e));           // (exact: it is a T already)
        }
    }
    __device__ __forceinline__ void finish(uint32_t lane) {
        if (kWhole) return;
        if (!off) {                  // nothing to copy, but its turn passes
            if (lane == 0) {
                bulk_commit();
                bulk_wait_read<1>();
            }
            return;
        }
        fence_proxy_async_smem();
        group_sync<kGroup>();
        const uint32_t end = off + d * static_cast<uint32_t>(sizeof(T)), whole_end = end / 16;      // pieces [1, whole_end) are whole
        uint8_t* base = reinterpret_cast<uint8_t*>(row) - off;
        if (lane == 0) {
            if (whole_end > 1) bulk_store(base + 16, image + 4, 16 * (whole_end - 1));
            bulk_commit();
            bulk_wait_read<1>();
        }
        // the first piece's elements, and those past the last whole one
        const T* elements = reinterpret_cast<const T*>(image);
        if (lane < 2 * E) {
            const uint32_t e = lane < E ? lane : max(whole_end, 1u) * E + lane - E, at = e * static_cast<uint32_t>(sizeof(T));
            if (at >= off && at < end) *reinterpret_cast<T*>(base + at) = elements[e];
        }
    }
    // before the shared memory is given up
    __device__ static __forceinline__ void drain(uint32_t lane) {
        if (!kWhole && lane == 0) bulk_wait_read<0>();
    }
};
template <typename T> __device__ __forceinline__ uint4 pack_unit(const uint64_t (&x)[Unit<T>::kElems / 2]) {
    float g[Unit<T>::kElems];
#pragma unroll
    for (uint32_t e = 0; e < Unit<T>::kElems; e += 2) unpack2(x[e / 2], g[e], g[e + 1]);
    return Unit<T>::pack(g);
}

// Forward: y = (x - mu) r w + b.  The row is read once into registers; the variance is the mean square of the deviations from the
// mean, a second sum over registers (a difference of squares would lose it where the mean is large against the deviation).
// Here a CTA to a row, for rows whose ring and parameters would not fit a CTA's shared memory.
constexpr uint32_t kUnitsThreads = 512u;
template <typename T, typename P>
__global__ void __launch_bounds__(kUnitsThreads)
norm_fwd_units_kernel(const T* x, uint32_t rows, uint32_t d, uint32_t ld, const P* __restrict__ weight,
                      const P* __restrict__ bias, float eps, T* y, uint32_t ld_y, float* __restrict__ mean_out,
                      float* __restrict__ rstd_out) {
    constexpr uint32_t E = Unit<T>::kElems, kUnits = 4;
    extern __shared__ __align__(16) uint4 images[];        // two of an unaligned y
    __shared__ float slots[128];
    const uint32_t lane = threadIdx.x, units = (d + E - 1) / E;
    const bool vec_w = vector_params(weight), vec_b = vector_params(bias), whole = d % E == 0;
    uint32_t turn = 0;
    for (uint64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const NormRow<T> in(x + row * ld, d);
        uint4 raw[kUnits];
        load_units<0, kUnits, false>(raw, lane, units, in.off, in.pieces, [&](uint32_t p) { return ld_unit(in.base + p); });
        uint64_t v[kUnits][E / 2];
        uint64_t sum = 0;
#pragma unroll
        for (uint32_t i = 0; i < kUnits; ++i) {
            const uint32_t u = lane + i * group_size<0>();
            unit_pairs<T>(raw[i], u < units ? d - u * E : 0u, 0.0f, v[i]);
#pragma unroll
            for (uint32_t q = 0; q < E / 2; ++q) sum = add2(sum, v[i][q]);
        }
        float s0, s1;
        unpack2(sum, s0, s1);
        float total = __fadd_rn(s0, s1);
        group_sum<0>(total, slots, turn++);
        const float mean = total / static_cast<float>(d);
        const uint64_t minus_mean = pack2(-mean, -mean);
        uint64_t squares = 0;
#pragma unroll
        for (uint32_t i = 0; i < kUnits; ++i) {
            const uint32_t u = lane + i * group_size<0>(), left = u < units ? d - u * E : 0u;
#pragma unroll
            for (uint32_t q = 0; q < E / 2; ++q) v[i][q] = add2(v[i][q], minus_mean);
            if (left < E) {                        // what is past the end does not deviate
#pragma unroll
                for (uint32_t q = 0; q < E / 2; ++q) {
                    float p0, p1;
                    unpack2(v[i][q], p0, p1);
                    v[i][q] = pack2(2 * q < left ? p0 : 0.0f, 2 * q + 1 < left ? p1 : 0.0f);
                }
            }
#pragma unroll
            for (uint32_t q = 0; q < E / 2; ++q) squares = fma2(v[i][q], v[i][q], squares);
        }
        unpack2(squares, s0, s1);
        float deviation = __fadd_rn(s0, s1);
        group_sum<0>(deviation, slots, turn++);
        const float rstd = 1.0f / sqrtf(deviation / static_cast<float>(d) + eps);
        const uint64_t by_rstd = pack2(rstd, rstd);
        RowWriter<T, 0, false> out(y + row * ld_y, d, images, units + 2, turn / 2);
#pragma unroll
        for (uint32_t i = 0; i < kUnits; ++i) {
            const uint32_t col = (lane + i * group_size<0>()) * E;
            uint64_t w[E / 2], b[E / 2];
            param_pairs<P, E>(weight, vec_w && whole, vec_w, col, d, 1.0f, w);
            param_pairs<P, E>(bias, vec_b && whole, vec_b, col, d, 0.0f, b);
#pragma unroll
            for (uint32_t q = 0; q < E / 2; ++q) v[i][q] = fma2(mul2(v[i][q], by_rstd), w[q], b[q]);
            out.put(lane + i * group_size<0>(), pack_unit<T>(v[i]));
        }
        out.finish(lane);
        if (lane == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
    RowWriter<T, 0, false>::drain(lane);
}

// Narrow rows: a unit to a lane and 32 / kLanes rows to a warp, four such sets of rows at a time.  With a warp to a row the work
// that every row costs (its sums, its addresses) would be most of all there is: 65536 rows of 128 bf16 25 us that way.
constexpr uint32_t kSets = 4u;

template <uint32_t kLanes> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (uint32_t o = kLanes / 2; o > 0; o >>= 1) v = __fadd_rn(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}
// unit u of a row that starts `off` bytes into the piece at base
__device__ __forceinline__ uint4 load_narrow(const uint4* base, uint32_t off, uint32_t pieces, uint32_t u) {
    uint4 v = ld_unit(base + min(u, pieces - 1));
    if (off) v = shifted(v, ld_unit(base + min(u + 1, pieces - 1)), off);
    return v;
}
// `left` elements of the row from the unit's first on
template <typename T> __device__ __forceinline__ void store_narrow(T* to, const uint4& v, uint32_t left) {
    constexpr uint32_t E = Unit<T>::kElems;
    const uintptr_t at = reinterpret_cast<uintptr_t>(to);
    if (left >= E && (at & 15u) == 0) {
        st_unit(to, v);
    } else if (left >= E && (at & 3u) == 0) {
        uint32_t* words = reinterpret_cast<uint32_t*>(to);
        words[0] = v.x;
        words[1] = v.y;
        words[2] = v.z;
        words[3] = v.w;
    } else {
#pragma unroll
        for (uint32_t e = 0; e < E; ++e)
            if (e < left) to[e] = from_f32<T>(Unit<T>::get(v, e));         // (exact: it is a T already)
    }
}

template <typename T, typename P, uint32_t kLanes>
__global__ void __launch_bounds__(256)
norm_fwd_narrow_kernel(const T* x, uint32_t rows, uint32_t d, uint32_t ld, const P* __restrict__ weight,
                       const P* __restrict__ bias, float eps, T* y, uint32_t ld_y, float* __restrict__ mean_out,
                       float* __restrict__ rstd_out, float per_column) {
    constexpr uint32_t E = Unit<T>::kElems, kRows = 32 / kLanes;
    const uint32_t sub = lane_id() % kLanes, col = sub * E, left = col < d ? d - col : 0u;
    uint64_t w[E / 2], b[E / 2];
    param_pairs<P, E>(weight, false, vector_params(weight), col, d, 1.0f, w);
    param_pairs<P, E>(bias, false, vector_params(bias), col, d, 0.0f, b);
    const uint64_t warps = static_cast<uint64_t>(gridDim.x) * 8, warp = static_cast<uint64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    for (uint64_t first = warp * kRows * kSets; first < rows; first += warps * kRows * kSets) {
        uint4 raw[kSets];
#pragma unroll
        for (uint32_t s = 0; s < kSets; ++s) {
            const uint64_t row = min(first + s * kRows + lane_id() / kLanes, static_cast<uint64_t>(rows) - 1);
            const NormRow<T> in(x + row * ld, d);
            raw[s] = load_narrow(in.base, in.off, in.pieces, sub);
        }
#pragma unroll
        for (uint32_t s = 0; s < kSets; ++s) {
            const uint64_t row = first + s * kRows + lane_id() / kLanes;
            uint64_t v[E / 2], sum = 0, squares = 0;
            unit_pairs<T>(raw[s], left, 0.0f, v);
#pragma unroll
            for (uint32_t q = 0; q < E / 2; ++q) sum = add2(sum, v[q]);
            float p0, p1;
            unpack2(sum, p0, p1);
            const float mean = __fmul_rn(lanes_sum<kLanes>(__fadd_rn(p0, p1)), per_column);
            const uint64_t minus_mean = pack2(-mean, -mean);
#pragma unroll
            for (uint32_t q = 0; q < E / 2; ++q) {
                v[q] = add2(v[q], minus_mean);
                if (left < E) {                    // what is past the end does not deviate
                    unpack2(v[q], p0, p1);
                    v[q] = pack2(2 * q < left ? p0 : 0.0f, 2 * q + 1 < left ? p1 : 0.0f);
                }
                squares = fma2(v[q], v[q], squares);
            }
            unpack2(squares, p0, p1);
            const float rstd = rsqrtf(fmaf(lanes_sum<kLanes>(__fadd_rn(p0, p1)), per_column, eps));
            const uint64_t by_rstd = pack2(rstd, rstd);
#pragma unroll
            for (uint32_t q = 0; q < E / 2; ++q) v[q] = fma2(mul2(v[q], by_rstd), w[q], b[q]);
            if (row < rows) {
                if (left) store_narrow(y + row * ld_y + col, pack_unit<T>(v), left);
                if (sub == 0) {
                    if (mean_out) mean_out[row] = mean;
                    if (rstd_out) rstd_out[row] = rstd;
                }
            }
        }
    }
}

template <typename T, typename P, uint32_t kLanes>
__global__ void __launch_bounds__(256)
norm_bwd_narrow_kernel(const T* dy, uint32_t ld_dy, const T* x, uint32_t rows, uint32_t d, uint32_t ld,
                       const P* __restrict__ weight, const float* __restrict__ mean, const float* __restrict__ rstd, T* dx,
                       uint32_t ld_dx, float* __restrict__ parts, float per_column) {
    constexpr uint32_t E = Unit<T>::kElems, kRows = 32 / kLanes;
    __shared__ float4 sums[8][2][kLanes * E / 4];
    chain_release_next();                  // the CTAs that join the partial sums may come and wait
    const uint32_t sub = lane_id() % kLanes, col = sub * E, left = col < d ? d - col : 0u;
    uint64_t w[E / 2], dw[E / 2], db[E / 2];
    param_pairs<P, E>(weight, false, vector_params(weight), col, d, 1.0f, w);
#pragma unroll
    for (uint32_t q = 0; q < E / 2; ++q) dw[q] = db[q] = 0;
    const uint64_t warps = static_cast<uint64_t>(gridDim.x) * 8, warp = static_cast<uint64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    for (uint64_t first = warp * kRows * kSets; first < rows; first += warps * kRows * kSets) {
        uint4 raw_x[kSets], raw_y[kSets];
        float mu[kSets], r[kSets];
#pragma unroll
        for (uint32_t s = 0; s < kSets; ++s) {
            const uint64_t row = min(first + s * kRows + lane_id() / kLanes, static_cast<uint64_t>(rows) - 1);
            const NormRow<T> in_x(x + row * ld, d), in_y(dy + row * ld_dy, d);
            raw_x[s] = load_narrow(in_x.base, in_x.off, in_x.pieces, sub);
            raw_y[s] = load_narrow(in_y.base, in_y.off, in_y.pieces, sub);
            mu[s] = mean[row];
            r[s] = rstd[row];
        }
#pragma unroll
        for (uint32_t s = 0; s < kSets; ++s) {
            const uint64_t row = first + s * kRows + lane_id() / kLanes;
            const bool inside = row < rows;
            const uint64_t minus_mu = pack2(-mu[s], -mu[s]), by_r = pack2(r[s], r[s]);
            uint64_t h[E / 2], g[E / 2], sum_g = 0, sum_gh = 0;
            unit_pairs<T>(raw_x[s], left, 0.0f, h);
            unit_pairs<T>(raw_y[s], inside ? left : 0u, 0.0f, g);           // (a row again at the end adds nothing)
#pragma unroll
            for (uint32_t q = 0; q < E / 2; ++q) {
                h[q] = mul2(add2(h[q], minus_mu), by_r);
                if (inside) dw[q] = fma2(g[q], h[q], dw[q]);
                db[q] = add2(db[q], g[q]);
                g[q] = mul2(g[q], w[q]);
                sum_g = add2(sum_g, g[q]);
                sum_gh = fma2(g[q], h[q], sum_gh);
            }
            float p0, p1;
            unpack2(sum_g, p0, p1);
            const float m1 = __fmul_rn(lanes_sum<kLanes>(__fadd_rn(p0, p1)), per_column);
            unpack2(sum_gh, p0, p1);
            const float m2 = __fmul_rn(lanes_sum<kLanes>(__fadd_rn(p0, p1)), per_column);
            const uint64_t minus_m1 = pack2(-m1, -m1), minus_m2 = pack2(-m2, -m2);
#pragma unroll
            for (uint32_t q = 0; q < E / 2; ++q) g[q] = mul2(by_r, fma2(h[q], minus_m2, add2(g[q], minus_m1)));
            if (inside && left) store_narrow(dx + row * ld_dx + col, pack_unit<T>(g), left);
        }
    }
    if (!parts) return;
    // the warp's sums over its rows' places, then the CTA's over its warps
    float v[2][E];
#pragma unroll
    for (uint32_t q = 0; q < E / 2; ++q) {
        unpack2(dw[q], v[0][2 * q], v[0][2 * q + 1]);
        unpack2(db[q], v[1][2 * q], v[1][2 * q + 1]);
    }
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k) {
#pragma unroll
        for (uint32_t e = 0; e < E; ++e)
#pragma unroll
            for (uint32_t o = 16; o >= kLanes; o >>= 1) v[k][e] = __fadd_rn(v[k][e], __shfl_xor_sync(0xFFFFFFFFu, v[k][e], o));
        if (lane_id() < kLanes) {
#pragma unroll
            for (uint32_t e = 0; e < E; e += 4)
                sums[threadIdx.x >> 5][k][(col + e) / 4] = make_float4(v[k][e], v[k][e + 1], v[k][e + 2], v[k][e + 3]);
        }
    }
    __syncthreads();
    const uint32_t width = (d + E - 1) / E * E;
    float4* cta = reinterpret_cast<float4*>(parts + static_cast<size_t>(blockIdx.x) * 2 * width);
    for (uint32_t i = threadIdx.x; i < 2 * width / 4; i += 256) {
        const uint32_t k = i / (width / 4), c = i % (width / 4);
        float4 t = sums[0][k][c];
#pragma unroll
        for (uint32_t n = 1; n < 8; ++n) {
            const float4 o = sums[n][k][c];
            t.x = __fadd_rn(t.x, o.x);
            t.y = __fadd_rn(t.y, o.y);
            t.z = __fadd_rn(t.z, o.z);
            t.w = __fadd_rn(t.w, o.w);
        }
        cta[i] = t;
    }
}

// Forward by the same rules for as many rows as a grid that stays has groups for: the rows come through a ring of bulk copies,
// kFwdRing ahead of the one being worked on, and the parameters lie in shared memory, so that a row's only waits are its two sums.
// (more rows on their way make the reads outrun the writes, and both slower: 16384 rows of 4096 fp32 with 2 / 3 / 4: 88 / 96 / 107 us)
constexpr uint32_t kFwdRing = 2u;

// the parameters as they lie in shared memory: 16-byte pieces (fp32 where a unit's bf16 parameters would be less than that),
// piece q of unit u at [q][u]
template <typename P, uint32_t kE> struct ParamImage {
    static constexpr bool kWide = kE * sizeof(P) < 16;
    static constexpr uint32_t kPieces = kWide ? 1 : kE * sizeof(P) / 16;
    static constexpr uint32_t kPerPiece = kE / kPieces;
    __device__ __forceinline__ static void fill(uint4* image, const P* params, uint32_t d, uint32_t units, float none) {
        for (uint32_t i = threadIdx.x; i < kPieces * units; i += blockDim.x) {
            const uint32_t col = i % units * kE + i / units * kPerPiece;
            float v[kPerPiece];
#pragma unroll
            for (uint32_t e = 0; e < kPerPiece; ++e) v[e] = params && col + e < d ? to_f32(params[col + e]) : none;
            if constexpr (kPerPiece == 4) image[i] = Unit<float>::pack(v);
            else image[i] = Unit<__nv_bfloat16>::pack(v);                   // (exact: bf16 already)
        }
    }
    __device__ __forceinline__ static void pairs(const uint4* image, uint32_t u, uint32_t units, uint64_t (&x)[kE / 2]) {
#pragma unroll
        for (uint32_t q = 0; q < kPieces; ++q) {
            const uint4 v = image[q * units + u];
#pragma unroll
            for (uint32_t e = 0; e < kPerPiece; e += 2) {
                if constexpr (kPerPiece == 4) x[(q * kPerPiece + e) / 2] = pack2(Unit<float>::get(v, e), Unit<float>::get(v, e + 1));
                else x[(q * kPerPiece + e) / 2] = pack2(Unit<__nv_bfloat16>::get(v, e), Unit<__nv_bfloat16>::get(v, e + 1));
            }
        }
    }
};

// What a CTA knows of its waits for rows of a ring.  gave_up: a bounded wait ran out, and that row is NaN; stuck: its copy did not come at
// all, no more are asked for and what is left is NaN.
struct RingWaits {
    uint32_t gave_up, stuck;
    __device__ __forceinline__ bool is_stuck() const { return *const_cast<const volatile uint32_t*>(&stuck); }
    // false: what lies in the slot is not to be used.  (A thread that knows of a copy that did not come never looks at a barrier
    // again, its limit is 0 from then on: the phase after the one that is due would seem to be over.)
    __device__ __forceinline__ bool row_is_here(uint64_t* full, uint32_t phase, uint32_t& spin_limit) {
        if (mbar_wait_bounded(full, phase, spin_limit, &gave_up)) return true;
        *const_cast<volatile uint32_t*>(&gave_up) = 1;
        if (!is_stuck() && !mbar_drain(full, phase)) *const_cast<volatile uint32_t*>(&stuck) = 1;
        if (is_stuck()) spin_limit = 0;
        return false;
    }
};
// CTAs of the forward kernel an SM's registers are asked to hold
template <uint32_t kThreads, uint32_t kUnits> constexpr uint32_t fwd_ctas() { return (kUnits == 4 ? 512 : 1024) / kThreads; }

// shared memory of a CTA of it: the parameters for `all` units; per group its slots and two images of an unaligned y
template <typename P, uint32_t kE, uint32_t kGroups> constexpr size_t fwd_shared(uint32_t all, uint32_t slot_units, bool whole) {
    return 16 * (2 * static_cast<size_t>(ParamImage<P, kE>::kPieces) * all + static_cast<size_t>(kGroups) * (kFwdRing + (whole ? 0 : 2)) * slot_units);
}

template <typename T, typename P, uint32_t kGroup, uint32_t kThreads, uint32_t kUnits, bool kWhole>
__global__ void __launch_bounds__(kThreads, fwd_ctas<kThreads, kUnits>())
norm_fwd_ring_kernel(const T* x, uint32_t rows, uint32_t d, uint32_t ld, const P* __restrict__ weight,
                     const P* __restrict__ bias, float eps, T* y, uint32_t ld_y, float* __restrict__ mean_out,
                     float* __restrict__ rstd_out, uint32_t slot_units, float per_column, uint32_t spin_limit) {
    constexpr uint32_t E = Unit<T>::kElems, kGroups = kGroup ? kThreads / kGroup : 1;
    using Image = ParamImage<P, E>;
    extern __shared__ __align__(128) uint4 shared[];       // parameters; per group its slots and two images of an unaligned y
    __shared__ float slots[128];
    __shared__ uint64_t full[kGroups][kFwdRing];
    __shared__ RingWaits waits;
    const uint32_t all = group_size<kGroup>() * kUnits;    // units the group's lanes hold
    const uint32_t lane = kGroup ? threadIdx.x % 32 : threadIdx.x, group = kGroup ? threadIdx.x / 32 : 0, units = (d + E - 1) / E;
    uint4 *const weights = shared, *const biases = shared + Image::kPieces * all;
    uint4* const mine = shared + 2 * Image::kPieces * all + group * (kFwdRing + (kWhole ? 0 : 2)) * slot_units;
    uint4* const image = mine + kFwdRing * slot_units;
    const uint64_t stride = static_cast<uint64_t>(gridDim.x) * kGroups;
    const uint64_t first = static_cast<uint64_t>(blockIdx.x) * kGroups + group;

    if (threadIdx.x == 0) waits = RingWaits{0, 0};
    if (lane == 0) {
        for (uint32_t s = 0; s < kFwdRing; ++s) mbar_init(&full[group][s], 1);
        mbar_init_fence();
        fence_proxy_async_smem();
    }
    __syncthreads();
    auto fetch = [&](uint64_t row, uint32_t slot) {          // by one thread
        if (row >= rows || waits.is_stuck()) return;
        const NormRow<T> a(x + row * ld, d);
        mbar_arrive_expect_tx(&full[group][slot], 16 * a.pieces);
        bulk_load(mine + slot * slot_units, a.base, 16 * a.pieces, &full[group][slot]);
    };
    if (lane == 0)
        for (uint32_t s = 0; s < kFwdRing; ++s) fetch(first + s * stride, s);
    Image::fill(weights, weight, d, all, 1.0f);
    Image::fill(biases, bias, d, all, 0.0f);
    __syncthreads();

    uint32_t slot = 0, phase = 0, turn = 0;
    const T* x_row = x + first * ld;
    T* y_row = y + first * ld_y;
    for (uint64_t row = first; row < rows; row += stride, x_row += stride * ld, y_row += stride * ld_y) {
        const NormRow<T> in(x_row, d);
        // (a thread that misses the row makes its sum NaN, and with it all the group writes of it)
        const bool missed = !waits.row_is_here(&full[group][slot], phase, spin_limit);
        uint4 raw[kUnits];
        const uint4* from = mine + slot * slot_units;
        load_units<kGroup, kUnits, kWhole>(raw, lane, units, in.off, in.pieces, [&](uint32_t p) { return from[p]; });
        uint64_t v[kUnits][E / 2];
        uint64_t sum = 0;
#pragma unroll
        for (uint32_t i = 0; i < kUnits; ++i) {
            const uint32_t u = lane + i * group_size<kGroup>();
            unit_pairs<T>(raw[i], kWhole ? E : u < units ? d - u * E : 0u, 0.0f, v[i]);
#pragma unroll
            for (uint32_t q = 0; q < E / 2; ++q) sum = add2(sum, v[i][q]);
        }
        float s0, s1, total;
        unpack2(sum, s0, s1);
        total = missed ? __uint_as_float(0x7FFFFFFFu) : __fadd_rn(s0, s1);
        group_sum<kGroup>(total, slots, turn++);
        if (kGroup == 32) __syncwarp();
        if (lane == 0) fetch(row + kFwdRing * stride, slot);      // every thread has its part of the row: the slot is free
        const float mean = __fmul_rn(total, per_column);
        const uint64_t minus_mean = pack2(-mean, -mean);
        uint64_t squares = 0;
#pragma unroll
        for (uint32_t i = 0; i < kUnits; ++i) {
            const uint32_t u = lane + i * group_size<kGroup>(), left = kWhole ? E : u < units ? d - u * E : 0u;
#pragma unroll
            for (uint32_t q = 0; q < E / 2; ++q) v[i][q] = add2(v[i][q], minus_mean);
            if (left < E) {                        // what is past the end does not deviate
#pragma unroll
                for (uint32_t q = 0; q < E / 2; ++q) {
                    float p0, p1;
                    unpack2(v[i][q], p0, p1);
                    v[i][q] = pack2(2 * q < left ? p0 : 0.0f, 2 * q + 1 < left ? p1 : 0.0f);
                }
            }
#pragma unroll
            for (uint32_t q = 0; q < E / 2; ++q) squares = fma2(v[i][q], v[i][q], squares);
        }
        unpack2(squares, s0, s1);
        float deviation = __fadd_rn(s0, s1);
        group_sum<kGroup>(deviation, slots, turn++);
        const float rstd = rsqrtf(fmaf(deviation, per_column, eps));
        const uint64_t by_rstd = pack2(rstd, rstd);
        RowWriter<T, kGroup, kWhole> out(y_row, d, image, slot_units, turn / 2);
#pragma unroll
        for (uint32_t i = 0; i < kUnits; ++i) {
            uint64_t w[E / 2], b[E / 2];
            Image::pairs(weights, lane + i * group_size<kGroup>(), all, w);
            Image::pairs(biases, lane + i * group_size<kGroup>(), all, b);
#pragma unroll
            for (uint32_t q = 0; q < E / 2; ++q) v[i][q] = fma2(mul2(v[i][q], by_rstd), w[q], b[q]);
            out.put(lane + i * group_size<kGroup>(), pack_unit<T>(v[i]));
        }
        out.finish(lane);
        if (lane == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
        if (++slot == kFwdRing) {
            slot = 0;
            phase ^= 1u;
        }
    }
    RowWriter<T, kGroup, kWhole>::drain(lane);
    if (lane == 0 && waits.is_stuck()) copies_settle();
}

// Backward: dx = r (g - mean(g) - h mean(g h)) with g = dy w, h = (x - mu) r; dweight = sum dy h, dbias = sum dy.
// A group's rows come through a ring of bulk copies (x and dy of a row to a slot); the row is taken into registers, added to
// the group's columns of the parameter gradients, summed over, and dx is written from the registers while the slot is
// filled again.
// (2 / 3 / 4 rows ahead: 73 / 68 / 69 us for 16384 rows of 4096 bf16.  Rows of more than 16 KiB go two ahead: with three, beside the images
// that an unaligned dx needs, slots of 32 KiB would not fit a CTA, and where they do, it is slower: 8192 rows of 8192 fp32 133 us with
// two and 137 with three, of 7000 108 and 118.)
template <uint32_t kThreads, uint32_t kUnits> constexpr uint32_t kBwdRing = kThreads * kUnits > 1024 ? 2 : 3;
// shared memory of a backward CTA whose rows span slot_units pieces at most: per group the slots of (x, dy) and two images of an unaligned dx
template <uint32_t kGroups, uint32_t kThreads, uint32_t kUnits, bool kWhole> constexpr size_t bwd_shared(uint32_t slot_units) {
    return static_cast<size_t>(kGroups) * (2 * kBwdRing<kThreads, kUnits> + (kWhole ? 0 : 2)) * slot_units * 16;
}
// CTAs of the backward kernel an SM's registers are asked to hold
template <uint32_t kThreads, uint32_t kUnits> constexpr uint32_t bwd_ctas() {
    return kUnits == 1 ? 768 / kThreads : kThreads <= 320 ? 640 / kThreads : 1;
}

template <typename T, typename P, uint32_t kGroup, uint32_t kThreads, uint32_t kUnits, bool kWhole>
__global__ void __launch_bounds__(kThreads, bwd_ctas<kThreads, kUnits>())
norm_bwd_units_kernel(const T* dy, uint32_t ld_dy, const T* x, uint32_t rows, uint32_t d, uint32_t ld,
                      const P* __restrict__ weight, const float* __restrict__ mean, const float* __restrict__ rstd, T* dx,
                      uint32_t ld_dx, float* __restrict__ parts, uint32_t slot_units, float per_column, uint32_t spin_limit) {
    constexpr uint32_t E = Unit<T>::kElems, kGroups = kGroup ? kThreads / kGroup : 1, kRing = kBwdRing<kThreads, kUnits>;
    extern __shared__ __align__(128) uint4 ring[];        // per group: kRing slots of (x, dy), and two images of an unaligned dx
    __shared__ float slots[128];
    __shared__ uint64_t full[kGroups][kRing];
    __shared__ RingWaits waits;
    const uint32_t lane = kGroup ? threadIdx.x % 32 : threadIdx.x, group = kGroup ? threadIdx.x / 32 : 0, units = (d + E - 1) / E;
    uint4* const mine = ring + group * (2 * kRing + (kWhole ? 0 : 2)) * slot_units;
    uint4* const image = mine + 2 * kRing * slot_units;
    const uint64_t stride = static_cast<uint64_t>(gridDim.x) * kGroups;
    const uint64_t first = static_cast<uint64_t>(blockIdx.x) * kGroups + group;

    chain_release_next();                  // the CTAs that join the partial sums may come and wait
    if (threadIdx.x == 0) waits = RingWaits{0, 0};
    if (lane == 0) {
        for (uint32_t s = 0; s < kRing; ++s) mbar_init(&full[group][s], 1);
        mbar_init_fence();
        fence_proxy_async_smem();
    }
    __syncthreads();
    auto fetch = [&](uint64_t row, uint32_t slot) {          // by one thread
        if (row >= rows || waits.is_stuck()) return;
        const NormRow<T> a(x + row * ld, d), b(dy + row * ld_dy, d);
        mbar_arrive_expect_tx(&full[group][slot], 16 * (a.pieces + b.pieces));
        bulk_load(mine + 2 * slot * slot_units, a.base, 16 * a.pieces, &full[group][slot]);
        bulk_load(mine + (2 * slot + 1) * slot_units, b.base, 16 * b.pieces, &full[group][slot]);
    };
    if (lane == 0)
        for (uint32_t s = 0; s < kRing; ++s) fetch(first + s * stride, s);

    uint64_t w[kUnits][E / 2], dw[kUnits][E / 2], db[kUnits][E / 2];
#pragma unroll
    for (uint32_t i = 0; i < kUnits; ++i) {
        param_pairs<P, E>(weight, false, vector_params(weight), (lane + i * group_size<kGroup>()) * E, d, 1.0f, w[i]);
#pragma unroll
        for (uint32_t q = 0; q < E / 2; ++q) dw[i][q] = db[i][q] = 0;
    }
    uint32_t slot = 0, phase = 0, turn = 0;
    float mu = first < rows ? mean[first] : 0.0f, r = first < rows ? rstd[first] : 0.0f;
    const T *x_row = x + first * ld, *dy_row = dy + first * ld_dy;
    T* dx_row = dx + first * ld_dx;
    for (uint64_t row = first; row < rows; row += stride, x_row += stride * ld, dy_row += stride * ld_dy, dx_row += stride * ld_dx) {
        const uint64_t next = row + stride;
        const float next_mu = next < rows ? mean[next] : 0.0f, next_r = next < rows ? rstd[next] : 0.0f;
        const NormRow<T> ax(x_row, d), ay(dy_row, d);
        // (a thread that misses the row makes its h NaN, and with it the sum of g h: all the group writes of it)
        if (!waits.row_is_here(&full[group][slot], phase, spin_limit)) r = __uint_as_float(0x7FFFFFFFu);
        const uint64_t minus_mu = pack2(-mu, -mu), by_r = pack2(r, r);
        uint64_t h[kUnits][E / 2], g[kUnits][E / 2], sum_g = 0, sum_gh = 0;
        const uint4* sx = mine + 2 * slot * slot_units;
        const uint4* sy = sx + slot_units;
        uint4 raw_x[kUnits], raw_y[kUnits];
        load_units<kGroup, kUnits, kWhole>(raw_x, lane, units, ax.off, ax.pieces, [&](uint32_t p) { return sx[p]; });
        load_units<kGroup, kUnits, kWhole>(raw_y, lane, units, ay.off, ay.pieces, [&](uint32_t p) { return sy[p]; });
#pragma unroll
        for (uint32_t i = 0; i < kUnits; ++i) {
            const uint32_t u = lane + i * group_size<kGroup>(), left = kWhole ? E : u < units ? d - u * E : 0u;
            unit_pairs<T>(raw_x[i], left, 0.0f, h[i]);
            unit_pairs<T>(raw_y[i], left, 0.0f, g[i]);
#pragma unroll
            for (uint32_t q = 0; q < E / 2; ++q) {
                h[i][q] = mul2(add2(h[i][q], minus_mu), by_r);
                dw[i][q] = fma2(g[i][q], h[i][q], dw[i][q]);
                db[i][q] = add2(db[i][q], g[i][q]);
                g[i][q] = mul2(g[i][q], w[i][q]);
                sum_g = add2(sum_g, g[i][q]);
                sum_gh = fma2(g[i][q], h[i][q], sum_gh);
            }
        }
        float p, q0, a, b;
        unpack2(sum_g, p, q0);
        a = __fadd_rn(p, q0);
        unpack2(sum_gh, p, q0);
        b = __fadd_rn(p, q0);
        group_sums<kGroup>(a, b, slots, turn++);
        if (kGroup == 32) __syncwarp();
        // every thread has its part of the row: the slot is free
        if (lane == 0) fetch(row + kRing * stride, slot);
        const float m1 = __fmul_rn(a, per_column), m2 = __fmul_rn(b, per_column);
        const uint64_t minus_m1 = pack2(-m1, -m1), minus_m2 = pack2(-m2, -m2);
        RowWriter<T, kGroup, kWhole> out(dx_row, d, image, slot_units, turn);
#pragma unroll
        for (uint32_t i = 0; i < kUnits; ++i) {
#pragma unroll
            for (uint32_t q = 0; q < E / 2; ++q)
                g[i][q] = mul2(by_r, fma2(h[i][q], minus_m2, add2(g[i][q], minus_m1)));
            out.put(lane + i * group_size<kGroup>(), pack_unit<T>(g[i]));
        }
        out.finish(lane);
        mu = next_mu;
        r = next_r;
        if (++slot == kRing) {
            slot = 0;
            phase ^= 1u;
        }
    }
    RowWriter<T, kGroup, kWhole>::drain(lane);
    if (lane == 0 && waits.is_stuck()) copies_settle();
    if (!parts) return;
    __syncthreads();                                       // every copy has arrived and been used, a wait that ran out is known
    // the CTA's partial sums: dweight, then dbias, `width` apart (a wait that ran out: NaN)
    const uint32_t width = units * E;
    float* cta = parts + static_cast<size_t>(blockIdx.x) * 2 * width;
    const float broken = waits.gave_up ? __uint_as_float(0x7FFFFFFFu) : 0.0f;
    float* to = cta;
    if (kGroups > 1) to = reinterpret_cast<float*>(ring) + group * 2 * width;
#pragma unroll
    for (uint32_t i = 0; i < kUnits; ++i) {
        const uint32_t u = lane + i * group_size<kGroup>();
        if (u >= units) break;
#pragma unroll
        for (uint32_t q = 0; q < E / 2; q += 2) {
            float4 v, t;
            unpack2(dw[i][q], v.x, v.y);
            unpack2(dw[i][q + 1], v.z, v.w);
            unpack2(db[i][q], t.x, t.y);
            unpack2(db[i][q + 1], t.z, t.w);
            v = make_float4(v.x + broken, v.y + broken, v.z + broken, v.w + broken);
            t = make_float4(t.x + broken, t.y + broken, t.z + broken, t.w + broken);
            *reinterpret_cast<float4*>(to + u * E + 2 * q) = v;
            *reinterpret_cast<float4*>(to + width + u * E + 2 * q) = t;
        }
    }
    if (kGroups > 1) {
        __syncthreads();
        const float4* from = reinterpret_cast<const float4*>(ring);
        for (uint32_t c = threadIdx.x; c < 2 * width / 4; c += kThreads) {
            float4 v = from[c];
#pragma unroll
            for (uint32_t k = 1; k < kGroups; ++k) {
                const float4 t = from[c + k * (2 * width / 4)];
                v.x = __fadd_rn(v.x, t.x);
                v.y = __fadd_rn(v.y, t.y);
                v.z = __fadd_rn(v.z, t.z);
                v.w = __fadd_rn(v.w, t.w);
            }
            reinterpret_cast<float4*>(cta)[c] = v;
        }
    }
}

// dweight, dbias from the CTAs' partial sums, in a fixed order: 32 columns to a CTA, a run of partial sums to each of its warps.
// Its launch overlaps the backward kernel; what it adds is the partial sums' way through L2 (16384 rows of 4096: 5.5 us)
constexpr uint32_t kJoinRuns = 32u, kJoinBatch = 5u;      // (ten would take the registers of an SM's second CTA)
__global__ void __launch_bounds__(32 * kJoinRuns, 2)
norm_param_join_kernel(const float* __restrict__ parts, uint32_t num, uint32_t d, uint32_t width,
                       float* __restrict__ dweight, float* __restrict__ dbias) {
    __shared__ float s[2][kJoinRuns][33];
    chain_wait_previous();
    const uint32_t lane = threadIdx.x & 31u, run = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float w = 0.0f, b = 0.0f;
    if (col < d) {
        for (uint32_t first = run; first < num; first += kJoinBatch * kJoinRuns) {
            float ws[kJoinBatch], bs[kJoinBatch];
#pragma unroll
            for (uint32_t k = 0; k < kJoinBatch; ++k) {
                const uint32_t i = first + k * kJoinRuns;
                const float* p = parts + static_cast<size_t>(i) * 2 * width + col;
                ws[k] = i < num ? __ldcg(p) : 0.0f;
                bs[k] = i < num ? __ldcg(p + width) : 0.0f;
            }
#pragma unroll
            for (uint32_t k = 0; k < kJoinBatch; ++k) {
                w = __fadd_rn(w, ws[k]);
                b = __fadd_rn(b, bs[k]);
            }
        }
    }
    s[0][run][lane] = w;
    s[1][run][lane] = b;
    __syncthreads();
    // warp r adds up column r of this CTA's: dweight, then dbias
    float v = warp_join<SumOp>(s[0][lane][run]), u = warp_join<SumOp>(s[1][lane][run]);
    const uint32_t mine = blockIdx.x * 32 + run;
    if (lane == 0 && mine < d) {
        if (dweight) dweight[mine] = v;
        if (dbias) dbias[mine] = u;
    }
}

// Rows too wide for a CTA's registers: 4096 rows of 16384 bf16 backward 365 us (1.1 TB/s) ---------------------------------------------------------------------------

template <typename T, typename P>
__global__ void __launch_bounds__(kNormThreads)
norm_fwd_kernel(const T* x, uint32_t rows, uint32_t d, uint32_t ld, const P* __restrict__ weight,
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
        auto result = [&](float x_j, uint32_t j) {
            const float w = weight ? to_f32(weight[j]) : 1.0f, b = bias ? to_f32(bias[j]) : 0.0f;
            return from_f32<T>(fmaf((x_j - mean) * rstd, w, b));
        };
        // (y may be x, so a load cannot be moved over a store: eight elements at a time, 129 us for 2048 rows of 32768 bf16; one by one 172)
        uint32_t j = threadIdx.x;
        for (; j + 7 * kNormThreads < d; j += 8 * kNormThreads) {
            T out[8];
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) out[k] = result(to_f32(xr[j + k * kNormThreads]), j + k * kNormThreads);
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) yr[j + k * kNormThreads] = out[k];
        }
        for (; j < d; j += kNormThreads) yr[j] = result(to_f32(xr[j]), j);
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

// warps that hold `units` with `each` to a lane
uint32_t warps_for(uint32_t units, uint32_t each) { return (units + 32 * each - 1) / (32 * each); }
// every row of a matrix starts on a 16-byte boundary
bool on_boundaries(const void* p, uint32_t rows, uint32_t ld, size_t es) {
    return aligned_to(p, 16) && (rows == 1 || static_cast<size_t>(ld) * es % 16 == 0);
}

// CTAs that may leave partial sums (the general kernels' rows are so wide that fewer do)
uint32_t norm_parts(uint32_t rows, uint32_t d) {
    const uint32_t most = d <= 8192 ? kMaxParts : 148u;
    return rows < most ? (rows ? rows : 1) : most;
}

template <typename T, typename P>
dct_status_t launch_fwd_units(const T* x, uint32_t rows, uint32_t d, uint32_t ld, const P* weight, const P* bias, float eps, T* y,
                              uint32_t ld_y, float* mean_out, float* rstd_out, cudaStream_t stream) {
    const uint32_t units = (d + Unit<T>::kElems - 1) / Unit<T>::kElems, threads = warps_for(units, 4) * 32;
    auto kernel = norm_fwd_units_kernel<T, P>;
    // an image only if some row of y does not start on a boundary
    const size_t smem = on_boundaries(y, rows, ld_y, sizeof(T)) ? 0 : 2 * static_cast<size_t>(units + 2) * 16;
    static SharedLimit allowed;
    const dct_status_t allowed_st = allow_shared(kernel, smem, allowed);
    if (allowed_st != DCT_OK) return allowed_st;
    kernel<<<rows < 1u << 30 ? rows : 1u << 30, threads, smem, stream>>>(x, rows, d, ld, weight, bias, eps, y, ld_y, mean_out, rstd_out);
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}

template <typename T, typename P, uint32_t kGroup, uint32_t kThreads, uint32_t kUnits>
dct_status_t launch_fwd_ring(const T* x, uint32_t rows, uint32_t d, uint32_t ld, const P* weight, const P* bias, float eps, T* y,
                             uint32_t ld_y, float* mean_out, float* rstd_out, cudaStream_t stream) {
    constexpr uint32_t kGroups = kGroup ? kThreads / kGroup : 1, E = Unit<T>::kElems;
    const int sms = sm_count();
    if (sms <= 0) return DCT_ERR_CUDA;
    const uint32_t threads = kGroup ? kThreads : warps_for((d + E - 1) / E, kUnits) * 32, all = (kGroup ? kGroup : threads) * kUnits;
    const bool whole = d == E * all && on_boundaries(x, rows, ld, sizeof(T)) && on_boundaries(y, rows, ld_y, sizeof(T));
    auto kernel = whole ? norm_fwd_ring_kernel<T, P, kGroup, kThreads, kUnits, true> : norm_fwd_ring_kernel<T, P, kGroup, kThreads, kUnits, false>;
    const uint32_t slot_units = (d + E - 1) / E + 2;       // (an unaligned row touches one piece more; its image half a word beyond)
    const size_t smem = fwd_shared<P, E, kGroups>(all, slot_units, whole);
    constexpr uint32_t kMostUnits = (kGroup ? kGroup : kThreads) * kUnits;
    static_assert(fwd_shared<P, E, kGroups>(kMostUnits, kMostUnits + 2, false) <= kMostShared, "a width of this kernel would be refused at launch");
    static SharedLimit allowed[2];
    const dct_status_t allowed_st = allow_shared(kernel, smem, allowed[whole]);
    if (allowed_st != DCT_OK) return allowed_st;
    uint32_t per_sm = static_cast<uint32_t>(227 * 1024 / (smem + 2048));
    const uint32_t by_registers = fwd_ctas<kThreads, kUnits>() * kThreads / threads;
    per_sm = per_sm < 1 ? 1 : per_sm < by_registers ? per_sm : by_registers;
    const uint64_t wanted = (static_cast<uint64_t>(rows) + kGroups - 1) / kGroups, room = static_cast<uint64_t>(sms) * per_sm;
    kernel<<<static_cast<uint32_t>(wanted < room ? wanted : room), threads, smem, stream>>>(
        x, rows, d, ld, weight, bias, eps, y, ld_y, mean_out, rstd_out, slot_units, 1.0f / static_cast<float>(d), debug_config().spin_limit);
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}

template <typename T, typename P, uint32_t kLanes>
dct_status_t launch_fwd_narrow(const T* x, uint32_t rows, uint32_t d, uint32_t ld, const P* weight, const P* bias, float eps, T* y,
                               uint32_t ld_y, float* mean_out, float* rstd_out, cudaStream_t stream) {
    const int sms = sm_count();
    if (sms <= 0) return DCT_ERR_CUDA;
    constexpr uint32_t per_cta = 8 * (32 / kLanes) * kSets;
    const uint64_t wanted = (static_cast<uint64_t>(rows) + per_cta - 1) / per_cta, room = static_cast<uint64_t>(sms) * 16;
    norm_fwd_narrow_kernel<T, P, kLanes><<<static_cast<uint32_t>(wanted < room ? wanted : room), 256, 0, stream>>>(
        x, rows, d, ld, weight, bias, eps, y, ld_y, mean_out, rstd_out, 1.0f / static_cast<float>(d));
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}

template <typename T, typename P>
dct_status_t launch_norm_fwd(const void* x_, uint32_t rows, uint32_t d, uint32_t ld, const void* weight_, const void* bias_,
                             float eps, void* y_, uint32_t ld_y, float* mean_out, float* rstd_out, cudaStream_t stream) {
    const T* x = static_cast<const T*>(x_);
    T* y = static_cast<T*>(y_);
    const P *weight = static_cast<const P*>(weight_), *bias = static_cast<const P*>(bias_);
    const uint32_t units = (d + Unit<T>::kElems - 1) / Unit<T>::kElems;
    auto go = [&](auto launch) { return launch(x, rows, d, ld, weight, bias, eps, y, ld_y, mean_out, rstd_out, stream); };
    if (units <= 8) return go(launch_fwd_narrow<T, P, 8>);
    if (units <= 16) return go(launch_fwd_narrow<T, P, 16>);
    if (units <= 32) {
        // (rows of exactly 32 units on boundaries: 17 us by the ring, 20 by this, for 65536 rows of 256 bf16; of 200: 27 and 22)
        const bool whole = d == 32 * Unit<T>::kElems && on_boundaries(x, rows, ld, sizeof(T)) && on_boundaries(y, rows, ld_y, sizeof(T));
        return whole ? go(launch_fwd_ring<T, P, 32, 256, 1>) : go(launch_fwd_narrow<T, P, 32>);
    }
    if (units <= 64) return go(launch_fwd_ring<T, P, 32, 256, 2>);
    if (units <= 128) return go(launch_fwd_ring<T, P, 32, 256, 4>);
    if (units <= 512) return go(launch_fwd_ring<T, P, 0, 256, 2>);
    if (units <= 1024) return go(launch_fwd_ring<T, P, 0, 256, 4>);
    if (units <= 2048) {
        // (the ring and both arrays of parameters fit an SM's shared memory unless fp32 parameters come with bf16 rows)
        if constexpr (sizeof(P) <= sizeof(T)) return go(launch_fwd_ring<T, P, 0, 512, 4>);
        else return go(launch_fwd_units<T, P>);
    }
    const uint32_t grid = rows < 4096u ? rows : 4096u;
    norm_fwd_kernel<T, P><<<grid, kNormThreads, 0, stream>>>(x, rows, d, ld, weight, bias, eps, y, ld_y, mean_out, rstd_out);
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}

dct_status_t launch_param_join(const float* parts, uint32_t num, uint32_t d, uint32_t width, float* dweight, float* dbias, cudaStream_t stream) {
    DCT_CUDA_TRY(launch_chained(norm_param_join_kernel, (d + 31) / 32, 32 * kJoinRuns, stream, parts, num, d, width, dweight, dbias));
    return DCT_OK;
}

template <typename T, typename P, uint32_t kGroup, uint32_t kThreads, uint32_t kUnits>
dct_status_t launch_bwd_units(const T* dy, uint32_t ld_dy, const T* x, uint32_t rows, uint32_t d, uint32_t ld, const P* weight,
                              const float* mean, const float* rstd, T* dx, uint32_t ld_dx, float* dweight, float* dbias,
                              float* parts, cudaStream_t stream) {
    constexpr uint32_t kGroups = kGroup ? kThreads / kGroup : 1, E = Unit<T>::kElems;
    const int sms = sm_count();
    if (sms <= 0) return DCT_ERR_CUDA;
    const uint32_t threads = kGroup ? kThreads : warps_for((d + E - 1) / E, kUnits) * 32;
    const bool whole = d == E * (kGroup ? kGroup : threads) * kUnits && on_boundaries(x, rows, ld, sizeof(T)) &&
                       on_boundaries(dy, rows, ld_dy, sizeof(T)) && on_boundaries(dx, rows, ld_dx, sizeof(T));
    auto kernel = whole ? norm_bwd_units_kernel<T, P, kGroup, kThreads, kUnits, true> : norm_bwd_units_kernel<T, P, kGroup, kThreads, kUnits, false>;
    const uint32_t slot_units = (d + E - 1) / E + 2;       // (an unaligned row touches one piece more; its image half a word beyond)
    const size_t smem = whole ? bwd_shared<kGroups, kThreads, kUnits, true>(slot_units) : bwd_shared<kGroups, kThreads, kUnits, false>(slot_units);
    constexpr uint32_t kMostUnits = (kGroup ? kGroup : kThreads) * kUnits + 2;
    static_assert(bwd_shared<kGroups, kThreads, kUnits, true>(kMostUnits) <= kMostShared && bwd_shared<kGroups, kThreads, kUnits, false>(kMostUnits) <= kMostShared,
                  "a width of this kernel would be refused at launch");
    static SharedLimit allowed[2];
    const dct_status_t allowed_st = allow_shared(kernel, smem, allowed[whole]);
    if (allowed_st != DCT_OK) return allowed_st;
    const uint64_t wanted = (static_cast<uint64_t>(rows) + kGroups - 1) / kGroups;
    uint64_t room = static_cast<uint64_t>(sms) * (bwd_ctas<kThreads, kUnits>() * kThreads / threads);
    if (room > kMaxParts) room = kMaxParts;
    const uint32_t grid = static_cast<uint32_t>(wanted < room ? wanted : room);
    const bool params = dweight || dbias;
    kernel<<<grid, threads, smem, stream>>>(dy, ld_dy, x, rows, d, ld, weight, mean, rstd, dx, ld_dx,
                                             params ? parts : nullptr, slot_units, 1.0f / static_cast<float>(d), debug_config().spin_limit);
    DCT_CUDA_TRY(cudaGetLastError());
    return params ? launch_param_join(parts, grid, d, (d + E - 1) / E * E, dweight, dbias, stream) : DCT_OK;
}

template <typename T, typename P, uint32_t kLanes>
dct_status_t launch_bwd_narrow(const T* dy, uint32_t ld_dy, const T* x, uint32_t rows, uint32_t d, uint32_t ld, const P* weight,
                               const float* mean, const float* rstd, T* dx, uint32_t ld_dx, float* dweight, float* dbias,
                               float* parts, cudaStream_t stream) {
    const int sms = sm_count();
    if (sms <= 0) return DCT_ERR_CUDA;
    constexpr uint32_t per_cta = 8 * (32 / kLanes) * kSets, E = Unit<T>::kElems;
    const uint64_t wanted = (static_cast<uint64_t>(rows) + per_cta - 1) / per_cta;
    uint64_t room = static_cast<uint64_t>(sms) * 3;
    if (room > norm_parts(rows, d)) room = norm_parts(rows, d);
    const uint32_t grid = static_cast<uint32_t>(wanted < room ? wanted : room);
    const bool params = dweight || dbias;
    norm_bwd_narrow_kernel<T, P, kLanes><<<grid, 256, 0, stream>>>(dy, ld_dy, x, rows, d, ld, weight, mean, rstd, dx, ld_dx,
                                                                   params ? parts : nullptr, 1.0f / static_cast<float>(d));
    DCT_CUDA_TRY(cudaGetLastError());
    return params ? launch_param_join(parts, grid, d, (d + E - 1) / E * E, dweight, dbias, stream) : DCT_OK;
}

template <typename T, typename P>
dct_status_t launch_norm_bwd(const void* dy_, uint32_t ld_dy, const void* x_, uint32_t rows, uint32_t d, uint32_t ld,
                             const void* weight_, const float* mean, const float* rstd, void* dx_, uint32_t ld_dx,
                             float* dweight, float* dbias, float* parts, cudaStream_t stream) {
    const T *dy = static_cast<const T*>(dy_), *x = static_cast<const T*>(x_);
    T* dx = static_cast<T*>(dx_);
    const P* weight = static_cast<const P*>(weight_);
    const uint32_t units = (d + Unit<T>::kElems - 1) / Unit<T>::kElems;
    auto go = [&](auto launch) { return launch(dy, ld_dy, x, rows, d, ld, weight, mean, rstd, dx, ld_dx, dweight, dbias, parts, stream); };
    if (units <= 8) return go(launch_bwd_narrow<T, P, 8>);
    if (units <= 16) return go(launch_bwd_narrow<T, P, 16>);
    if (units <= 32) {
        const bool whole = d == 32 * Unit<T>::kElems && on_boundaries(x, rows, ld, sizeof(T)) &&
                           on_boundaries(dy, rows, ld_dy, sizeof(T)) && on_boundaries(dx, rows, ld_dx, sizeof(T));
        return whole ? go(launch_bwd_units<T, P, 32, 256, 1>) : go(launch_bwd_narrow<T, P, 32>);
    }
    if (units <= 64) return go(launch_bwd_units<T, P, 32, 256, 2>);
    if (units <= 128) {
        if constexpr (sizeof(T) == 4) return go(launch_bwd_units<T, P, 32, 256, 4>);
        else return go(launch_bwd_units<T, P, 0, 128, 1>);
    }
    if (units <= 256) return go(launch_bwd_units<T, P, 0, 256, 1>);
    if (units <= 512) return go(launch_bwd_units<T, P, 0, 256, 2>);
    if (units <= 640) return go(launch_bwd_units<T, P, 0, 320, 2>);
    if (units <= 1024) return go(launch_bwd_units<T, P, 0, 512, 2>);
    if constexpr (sizeof(T) == 4)
        if (units <= 2048) return go(launch_bwd_units<T, P, 0, 512, 4>);
    if (dweight || dbias) {        // before dx, which may take the place of dy or x
        const uint32_t cols = (d + kNormThreads - 1) / kNormThreads, num = norm_parts(rows, d);
        norm_param_parts_kernel<T><<<dim3(cols, num), kNormThreads, 0, stream>>>(dy, ld_dy, x, rows, d, ld, mean, rstd, parts);
        DCT_CUDA_TRY(cudaGetLastError());
        const dct_status_t st = launch_param_join(parts, num, d, d, dweight, dbias, stream);
        if (st != DCT_OK) return st;
    }
    const uint32_t grid = rows < 4096u ? rows : 4096u;
    norm_bwd_kernel<T, P><<<grid, kNormThreads, 0, stream>>>(dy, ld_dy, x, rows, d, ld, weight, mean, rstd, dx, ld_dx);
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
    return (static_cast<size_t>(norm_parts(rows, d)) * 2 * ((d + 7) / 8 * 8) * sizeof(float) + 255) & ~static_cast<size_t>(255);
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
