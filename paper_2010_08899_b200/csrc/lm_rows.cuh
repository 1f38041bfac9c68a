// Pieces shared by the layer norm and by the calls on rows of logits: element types, sums over a CTA in a fixed
// order, the order of logits, and the host's argument checks.
#pragma once
#include <cmath>

#include "common.cuh"
#include "launch_words.h"

namespace dct {

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

__device__ __forceinline__ float minus_inf() { return __uint_as_float(0xFF800000u); }

// The order of logits as unsigned integers: a < b exactly when order_key(a) < order_key(b), -0 and +0 alike, NaN
// (key 0) below everything, -inf (key 0x007FFFFF) the lowest of the others.
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t u = __float_as_uint(__fadd_rn(x, 0.0f));       // -0 + 0 = +0
    const uint32_t key = u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
    return x == x ? key : 0u;
}

struct SumOp {
    static constexpr float kNeutral = 0.0f;
    __device__ static __forceinline__ float join(float a, float b) { return __fadd_rn(a, b); }
};
struct MaxOp {     // NaN loses
    __device__ static __forceinline__ float join(float a, float b) { return fmaxf(a, b); }
};
template <typename Op> __device__ __forceinline__ float warp_join(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = Op::join(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}
// The same value in every thread of the CTA.  scratch: 32 floats that nothing else uses between two calls' barriers.
template <typename Op> __device__ __forceinline__ float cta_join(float v, float* scratch) {
    const uint32_t warps = blockDim.x >> 5;
    v = warp_join<Op>(v);
    __syncthreads();                 // the last call's readers are done
    if (lane_id() == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = scratch[0];
    for (uint32_t w = 1; w < warps; ++w) v = Op::join(v, scratch[w]);
    return v;
}

// Sum of whole numbers over the CTA, the same in every thread.  scratch: 32 words, as above.
__device__ __forceinline__ uint32_t cta_count(uint32_t v, uint32_t* scratch) {
    v = __reduce_add_sync(0xFFFFFFFFu, v);
    __syncthreads();
    if (lane_id() == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0;
    for (uint32_t w = 0; w < (blockDim.x >> 5); ++w) v += scratch[w];
    return v;
}

// A row as 16-byte units ----------------------------------------------------------------------------------------
// A row starts and ends anywhere; it is read in whole 16-byte units from the boundary at or before its first element
// (the unit lies in the same page, so the elements outside the row are readable), and what lies outside the row
// is replaced before it is used.

constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {            // 2^x within 2 ulp; results below 2^-126 are 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// two fp32 in a 64-bit register: one instruction for both
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

template <typename T> struct Unit {};
template <> struct Unit<float> {
    static constexpr int kElems = 4;
    static constexpr uint32_t kMinusInf = 0xFF800000u;
    __device__ static __forceinline__ float get(const uint4& v, int i) {
        return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w);
    }
    __device__ static __forceinline__ void set(uint4& v, int i, float x) {
        const uint32_t u = __float_as_uint(x);
        if (i == 0) v.x = u; else if (i == 1) v.y = u; else if (i == 2) v.z = u; else v.w = u;
    }
    __device__ static __forceinline__ uint4 pack(const float (&g)[4]) {
        return make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3]));
    }
    // the largest element, NaN only if all are
    __device__ static __forceinline__ float best(const uint4& a) {
        return fmaxf(fmaxf(get(a, 0), get(a, 1)), fmaxf(get(a, 2), get(a, 3)));
    }
    __device__ static __forceinline__ float best(const uint4& a, const uint4& b) { return fmaxf(best(a), best(b)); }
};
template <> struct Unit<__nv_bfloat16> {
    static constexpr int kElems = 8;
    static constexpr uint32_t kMinusInf = 0xFF80FF80u;
    __device__ static __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
    __device__ static __forceinline__ float get(const uint4& v, int i) {
        const uint32_t w = word(v, i >> 1);
        return __uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
    }
    __device__ static __forceinline__ void set(uint4& v, int i, float x) {
        const uint32_t u = __bfloat16_as_ushort(__float2bfloat16_rn(x));
        uint32_t w = word(v, i >> 1);
        w = i & 1 ? (w & 0xFFFFu) | u << 16 : (w & 0xFFFF0000u) | u;
        if (i >> 1 == 0) v.x = w; else if (i >> 1 == 1) v.y = w; else if (i >> 1 == 2) v.z = w; else v.w = w;
    }
    __device__ static __forceinline__ uint4 pack(const float (&g)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(g[2 * i], g[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ static __forceinline__ __nv_bfloat162 pair(uint32_t w) { return *reinterpret_cast<__nv_bfloat162*>(&w); }
    __device__ static __forceinline__ __nv_bfloat162 best2(const uint4& v) {
        return __hmax2(__hmax2(pair(v.x), pair(v.y)), __hmax2(pair(v.z), pair(v.w)));
    }
    __device__ static __forceinline__ float best(const uint4& a) {
        const __nv_bfloat162 m = best2(a);
        return fmaxf(__low2float(m), __high2float(m));
    }
    __device__ static __forceinline__ float best(const uint4& a, const uint4& b) {
        const __nv_bfloat162 m = __hmax2(best2(a), best2(b));
        return fmaxf(__low2float(m), __high2float(m));
    }
};

__device__ __forceinline__ uint4 ld_unit(const uint4* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

__device__ __forceinline__ void st_unit(void* p, const uint4& v) {
    asm volatile("st.global.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void st_unit_stream(void* p, const uint4& v) {        // the first to leave L2
    asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void copy_word_async(void* smem, const void* global) {        // 4 bytes, both 4-byte aligned
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_addr(smem)), "l"(global) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory"); }
__device__ __forceinline__ float max_nan(float a, float b) {     // NaN if either is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

template <typename T> struct RowView {
    static constexpr uint32_t kElems = Unit<T>::kElems;
    const uint4* base;       // the boundary at or before the first element
    uint32_t lead;           // elements of the first unit that lie before the row
    uint32_t units;
    uint32_t width;          // elements of the row
    bool ragged;             // a unit at an end holds elements outside the row

    __device__ __forceinline__ RowView(const T* row, uint32_t width_) { at(row, width_); }
    __device__ __forceinline__ void at(const T* row, uint32_t width_) {
        width = width_;
        const uintptr_t a = reinterpret_cast<uintptr_t>(row);
        lead = static_cast<uint32_t>(a & 15u) / static_cast<uint32_t>(sizeof(T));
        base = reinterpret_cast<const uint4*>(a & ~static_cast<uintptr_t>(15));
        units = (lead + width + kElems - 1) / kElems;
        ragged = lead != 0 || width % kElems != 0;
    }
    // column of element i of unit u; >= width (as unsigned) outside the row
    __device__ __forceinline__ uint32_t column(uint32_t u, uint32_t i) const { return u * kElems + i - lead; }
    __device__ __forceinline__ bool at_an_end(uint32_t u) const { return u == 0 || u + 1 == units; }
    // -inf in the place of what lies outside the row (only the first and the last unit can hold such elements)
    __device__ __forceinline__ void mask(uint4& v, uint32_t u) const {
        if (at_an_end(u)) {
#pragma unroll
            for (uint32_t i = 0; i < kElems; ++i)
                if (column(u, i) >= width) Unit<T>::set(v, i, minus_inf());
        }
    }
};

// Writes unit u of a row laid out as `row`, element by element where the unit holds anything else, too (or everywhere, if
// the output row sits differently against the 16-byte boundaries: `aligned` is false then).
template <typename T>
__device__ __forceinline__ void store_unit(const RowView<T>& row, T* out, uint32_t u, const float (&g)[Unit<T>::kElems], bool aligned) {
    constexpr uint32_t E = Unit<T>::kElems;
    if (aligned && !row.at_an_end(u)) {
        st_unit(out + row.column(u, 0), Unit<T>::pack(g));
    } else {
#pragma unroll
        for (uint32_t i = 0; i < E; ++i) {
            const uint32_t col = row.column(u, i);
            if (col < row.width) out[col] = from_f32<T>(g[i]);
        }
    }
}
inline __device__ bool same_boundary(const void* a, const void* b) {      // alike against the 16-byte boundaries
    return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) & 15u) == 0;
}

__device__ __forceinline__ float warp_max(float v) {               // NaN only if every lane's is
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xFFFFFFFF;" : "=f"(r) : "f"(v));
    return r;
}

// 1 / T and log2 e / T
struct Scale {
    float inv_t, c;
};

// Rows whose largest z = x / T lies 2^26 or more from zero (a mask's value throughout, as a rule) are far off.  The exact z is then up to
// 2 and more away from the nearest fp32 number, and for the masks in use, -1e9 to the type's lowest value, so far that 2^z
// relative to that number overflows.  z there is the product rounded to fp32 everywhere: in the largest, in the sums, in log p and in the gradients.
// Below that, z enters as the exact product (one fma).
constexpr float kFar = 67108864.0f, kFarLog2 = 2.0f * kFar;          // (kFarLog2 > log2 e kFar)
__device__ __forceinline__ bool far_off(float z) { return !(fabsf(z) < kFar); }            // infinities and NaN, too
// z - m; m: the row's largest z, rounded (-inf, a row without a number: z itself)
__device__ __forceinline__ float less_max(float x, float inv_t, float m) {
    if (m == minus_inf()) m = 0.0f;
    return far_off(m) ? __fadd_rn(__fmul_rn(x, inv_t), -m) : fmaf(x, inv_t, -m);
}
// what the exact largest z is beyond m
__device__ __forceinline__ float beyond_max(float xmax, float inv_t, float m) { return far_off(m) ? 0.0f : fmaf(xmax, inv_t, -m); }

// What is known of a part of a row: its largest x, and relative to that the sums s = sum 2^y and st = sum 2^y y with
// y = (x - xmax) c, c = log2 e / T.  st / s is the mean of log2 p + log2 s.  An empty part has xmax = -inf, s = 0.
struct RowPart {
    float xmax, s, st;
    // the same sums relative to a larger x, which is `apart` (binary powers) above this one
    __device__ __forceinline__ void raise(float to, float apart) {
        if (s == 0.0f) {
            st = 0.0f;
        } else {
            // (from -1e4 on the factor is 0, and no difference may be so large that s * d overflows)
            const float d = xmax == to ? 0.0f : max_nan(apart, -1.0e4f), f = exp2_fast(d);
            st = __fmul_rn(f, fmaf(s, d, st));
            s = __fmul_rn(f, s);
        }
        xmax = to;
    }
    template <int kLanes, bool kMoment> __device__ __forceinline__ void add_lanes() {
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) {
            s = __fadd_rn(s, __shfl_xor_sync(0xFFFFFFFFu, s, o));
            if (kMoment) st = __fadd_rn(st, __shfl_xor_sync(0xFFFFFFFFu, st, o));
        }
    }
    // joins the parts of kLanes (a power of two) neighbouring lanes, in a fixed order; all lanes get the result.  (Every group of
    // kLanes lanes holds the same parts, so the warp's largest x is the group's.)
    template <int kLanes, bool kMoment> __device__ __forceinline__ void join_lanes(float c) {
        const float to = kLanes == 1 ? xmax : warp_max(xmax);
        raise(to, __fmul_rn(__fadd_rn(xmax, -to), c));
        add_lanes<kLanes, kMoment>();
    }
    // the same for whole slices of a row, each summed as its own largest x asks for
    template <int kLanes, bool kMoment> __device__ __forceinline__ void join_slices(const Scale& by) {
        const float to = warp_max(xmax), z = __fmul_rn(to, by.inv_t);
        raise(to, far_off(z) && z > minus_inf() ? __fmul_rn(__fadd_rn(__fmul_rn(xmax, by.inv_t), -z), kLog2E) : __fmul_rn(__fadd_rn(xmax, -to), by.c));
        add_lanes<kLanes, kMoment>();
    }
};

// One warp's share of the part of a row whose largest z is far off, from z as rounded: the units first + lane, `step` on, below u1.
// keep(u, i): whether element i of unit u counts.  (Out of line, with four loads under way: 4096 such rows of 32768 bf16 99 us in all, one load at a
// time and one warp to a slice 153.)
template <typename T, typename Keep>
__device__ __noinline__ RowPart far_part(const RowView<T> row, uint32_t first, uint32_t step, uint32_t u1, float xmax, const Scale by, const Keep keep) {
    constexpr uint32_t E = Unit<T>::kElems;
    const float m = __fmul_rn(xmax, by.inv_t), less = m == minus_inf() ? 0.0f : -m;
    uint64_t sum = 0, moment = 0;
    for (uint32_t u = first + lane_id(); u < u1; u += 4 * step) {
        uint4 v[4];
#pragma unroll
        for (uint32_t n = 0; n < 4; ++n) v[n] = ld_unit(row.base + min(u + n * step, u1 - 1));
#pragma unroll
        for (uint32_t n = 0; n < 4; ++n) {
            const uint32_t at = u + n * step;
            if (at >= u1) break;
            row.mask(v[n], at);
#pragma unroll
            for (uint32_t i = 0; i < E; ++i)
                if (!keep(at, i)) Unit<T>::set(v[n], i, minus_inf());
#pragma unroll
            for (uint32_t i = 0; i < E; i += 2) {
                // (one by one: of a product and a sum of pairs the compiler makes one fma, whose product is not rounded)
                const float d0 = __fadd_rn(__fmul_rn(Unit<T>::get(v[n], i), by.inv_t), less);
                const float d1 = __fadd_rn(__fmul_rn(Unit<T>::get(v[n], i + 1), by.inv_t), less);
                const float y0 = max_nan(__fmul_rn(d0, kLog2E), -200.0f), y1 = max_nan(__fmul_rn(d1, kLog2E), -200.0f);
                const uint64_t y = pack2(y0, y1), e = pack2(exp2_fast(y0), exp2_fast(y1));
                sum = add2(sum, e);
                moment = fma2(e, y, moment);
            }
        }
    }
    RowPart p{xmax, 0.0f, 0.0f};
    float p0, p1;
    unpack2(sum, p0, p1);
    p.s = __fadd_rn(p0, p1);
    unpack2(moment, p0, p1);
    p.st = __fadd_rn(p0, p1);
    __syncwarp();
    p.join_lanes<32, true>(by.c);          // (alike in their xmax)
    return p;
}

// One thread's share of sum 2^y and sum 2^y y over a row, y = x c - ref.  The reference is the warp's: the largest x c of its
// first batch, replaced only when a batch exceeds it by kSlack, so that an element costs one product-sum, one power of
// two and two sums.  Rounding c and ref moves nothing but the reference: what counts is (x - xmax) c, and the
// distance of xmax c to ref is formed by one fma at the end.  A reference is below kFarLog2 in size, so that no y exceeds kSlack by more
// than the 4 its rounding can be off.  Batches whose largest x is further down add nothing; where it is all the row has, or
// where there is one further up, the row is far off and these sums are not used.
struct RowSums {
    static constexpr float kSlack = 4.0f;
    float ref, s, st;
    bool masked;                   // several of the warp's lanes met -inf beside numbers in the last batch
    __device__ __forceinline__ RowSums() : ref(minus_inf()), s(0.0f), st(0.0f), masked(false) {}

    // sums over four units.  kClamp: y at least -200, so that a masked column (2^y = 0, y = -inf) adds 0 to the moment and not NaN
    template <typename T, bool kMoment, bool kClamp>
    __device__ __forceinline__ void batch(const uint4 (&v)[4], float c, float& sum, float& moment) const {
        constexpr int E = Unit<T>::kElems;
        const uint64_t scale = pack2(c, c), shift = pack2(-ref, -ref);
        uint64_t sb = 0, stb = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < E; i += 2) {
                uint64_t y = fma2(pack2(Unit<T>::get(v[u], i), Unit<T>::get(v[u], i + 1)), scale, shift);
                float y0, y1;
                unpack2(y, y0, y1);
                if (kClamp) y = pack2(y0 = max_nan(y0, -200.0f), y1 = max_nan(y1, -200.0f));
                const uint64_t e = pack2(exp2_fast(y0), exp2_fast(y1));
                sb = add2(sb, e);
                if (kMoment) stb = fma2(e, y, stb);
            }
        float p, q;
        unpack2(sb, p, q);
        sum = __fadd_rn(p, q);
        unpack2(stb, p, q);
        moment = __fadd_rn(p, q);
    }
    // best: the largest of this thread's four units; all lanes of the warp take part
    template <typename T, bool kMoment> __device__ __forceinline__ void add(const uint4 (&v)[4], float best, float c) {
        if (__any_sync(0xFFFFFFFFu, !(__fmul_rn(best, c) <= __fadd_rn(ref, kSlack)))) {
            const float to = __fmul_rn(warp_max(best), c);
            if (to > ref && fabsf(to) < kFarLog2) {
                if (ref != minus_inf()) {
                    const float d = max_nan(__fadd_rn(ref, -to), -1.0e4f), f = exp2_fast(d);
                    st = __fmul_rn(f, fmaf(s, d, st));
                    s = __fmul_rn(f, s);
                }
                ref = to;
            }
        }
        if (ref == minus_inf()) {        // nothing but -inf, NaN and values far off so far
            float any = 0.0f;
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int i = 0; i < Unit<T>::kElems; ++i) any = __fadd_rn(any, Unit<T>::get(v[u], i));
            if (any != any) s = any;
            return;
        }
        float sum, moment = 0.0f;
        if (!kMoment) {
            batch<T, false, false>(v, c, sum, moment);
        } else {
            // (the ends of a row put -inf into one lane's units of one batch: no reason to clamp from there on)
            if (!masked) batch<T, true, false>(v, c, sum, moment);
            const bool clamp = masked || moment != moment;
            masked = __popc(__ballot_sync(0xFFFFFFFFu, clamp)) >= 8;
            if (clamp) batch<T, true, true>(v, c, sum, moment);
        }
        s = __fadd_rn(s, sum);
        if (kMoment) st = __fadd_rn(st, moment);
    }
    // the warp's sums as a part; xmax: the warp's largest x
    template <bool kMoment> __device__ __forceinline__ RowPart part(float xmax, float c) const {
        RowPart r{xmax, warp_join<SumOp>(s), kMoment ? warp_join<SumOp>(st) : 0.0f};
        if (ref != minus_inf()) {
            // |xmax c - ref| <= kSlack + 4; the factor puts the sums where 2^y of the largest x is 1
            const float d = fmaf(xmax, c, -ref), f = exp2_fast(-d);
            r.st = __fmul_rn(f, fmaf(-d, r.s, r.st));
            r.s = __fmul_rn(f, r.s);
        }
        return r;
    }
};

// Streams the units [u0, u1) of a row through the CTA, in batches of four units per thread (first + tid + i kThreads).
// each(v, first) takes the four units, -inf where there is no element of the row or the slice, and the first one's number.
template <typename T, uint32_t kThreads, typename Each>
__device__ __forceinline__ void stream_units(const RowView<T>& row, uint32_t u0, uint32_t u1, Each&& each) {
    constexpr uint32_t kInf = Unit<T>::kMinusInf;
    for (uint32_t batch = u0; batch < u1; batch += 4 * kThreads) {
        const uint32_t first = batch + threadIdx.x;
        uint4 v[4];
        if (batch + 4 * kThreads <= u1) {                  // the same for the whole CTA: no bounds to look at
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = ld_unit(row.base + first + i * kThreads);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = make_uint4(kInf, kInf, kInf, kInf);
                if (first + i * kThreads < u1) v[i] = ld_unit(row.base + first + i * kThreads);
            }
        }
        if (row.ragged && (batch == 0 || batch + 4 * kThreads >= row.units)) {      // can hold an end of the row
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (first + i * kThreads < u1) row.mask(v[i], first + i * kThreads);
        }
        each(v, first);
    }
}

// The units of one row that one of `ctas` CTAs takes.
struct Slice {
    uint32_t u0, u1;
    __device__ __forceinline__ Slice(uint32_t units, uint32_t rank, uint32_t ctas) {
        const uint32_t share = (units + ctas - 1) / ctas;
        u0 = min(units, rank * share);
        u1 = min(units, u0 + share);
    }
    // the row's columns that lie in it
    template <typename Row> __device__ __forceinline__ uint32_t columns(const Row& row) const {
        if (u0 == u1) return 0;
        return min(row.width, u1 * Row::kElems - row.lead) - (u0 == 0 ? 0u : u0 * Row::kElems - row.lead);
    }
};

// After a bounded wait that ran out (what depends on it becomes NaN): waits for the same phase once more, for up to a second by the
// clock and whatever the first limit was, so that nothing is on its way when shared memory is used again or given up, and the
// barrier is in step with its copies.  False if that ran out, too.
__device__ __forceinline__ bool mbar_drain(uint64_t* bar, uint32_t parity) {
    uint64_t start, now;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(start));
    for (uint32_t i = 0; i < 1u << 24; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
        if (now - start > 1000000000ull) break;
    }
    return false;
}

// A second by the clock, before shared memory is given up or used for something else, for copies that may be on their way after one did not come.
static __device__ __noinline__ void copies_settle() {
    uint64_t start, now;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(start));
    for (uint32_t i = 0; i < 1u << 20; ++i) {
        __nanosleep(1000u);
        asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
        if (now - start > 1000000000ull) break;
    }
}

// Clusters of CTAs -------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
// every CTA of the cluster has arrived, and what each wrote to its shared memory before is visible to all
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// its two halves, for work in between that needs neither.  The first tells of reads that are over (or of what a fence of its own
// covers): nothing this CTA wrote is waited for.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ uint32_t remote_smem(const void* p, uint32_t rank) {      // p's counterpart in CTA `rank`
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
    return a;
}
// four values into another CTA's shared memory (16-byte aligned), counted there on that CTA's mbarrier; both by remote_smem
__device__ __forceinline__ void push_remote(uint32_t to, float x, float y, float z, float w, uint32_t bar) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                 ::"r"(to), "f"(x), "f"(y), "f"(z), "f"(w), "r"(bar) : "memory");
}
__device__ __forceinline__ void push_remote(uint32_t to, uint64_t x, uint32_t bar) {          // 8-byte aligned
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];" ::"r"(to), "l"(x), "r"(bar) : "memory");
}

// Host side ---------------------------------------------------------------------------------------------------

// the current device, as an index into what is kept per device
inline dct_status_t current_device(int* out) {
    DCT_CUDA_TRY(cudaGetDevice(out));
    return *out >= 0 && *out < kMaxDevices ? DCT_OK : DCT_ERR_CUDA;
}

// How many clusters of `cluster` (2, 4 or 8) CTAs the current device holds at a time.  A GPC's SMs are no multiple of a cluster, so
// this is less than the CTAs that fit divided by the cluster; a persistent grid of more would run its last clusters after
// all others.
template <typename... Params>
inline dct_status_t clusters_at_once(void (*kernel)(Params...), unsigned block, unsigned cluster, size_t smem,
                                     ClusterCounts& kept, uint32_t* out) {
    int dev = 0;
    const dct_status_t st = current_device(&dev);
    if (st != DCT_OK) return st;
    cudaError_t error = cudaSuccess;
    *out = kept.get(dev, cluster, [&]() -> uint32_t {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(cluster);
        cfg.blockDim = dim3(block);
        cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute shape = {};
        shape.id = cudaLaunchAttributeClusterDimension;
        shape.val.clusterDim.x = cluster;
        shape.val.clusterDim.y = 1;
        shape.val.clusterDim.z = 1;
        cfg.attrs = &shape;
        cfg.numAttrs = 1;
        int found = 0;
        error = cudaOccupancyMaxActiveClusters(&found, kernel, &cfg);
        return error != cudaSuccess ? 0u : found > 0 ? static_cast<uint32_t>(found) : 1u;
    });
    DCT_CUDA_TRY(error);
    return DCT_OK;
}

// launches `kernel` in clusters of `cluster` CTAs
template <typename... Params, typename... Args>
cudaError_t launch_clusters(void (*kernel)(Params...), unsigned grid, unsigned block, unsigned cluster, size_t smem,
                            cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute shape = {};
    shape.id = cudaLaunchAttributeClusterDimension;
    shape.val.clusterDim.x = cluster;
    shape.val.clusterDim.y = 1;
    shape.val.clusterDim.z = 1;
    cfg.attrs = &shape;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}

inline size_t element_size(dct_dtype_t t) { return t == DCT_F32 ? 4 : 2; }
inline bool known_dtype(dct_dtype_t t) { return t == DCT_F32 || t == DCT_BF16; }

// [rows, ld] of which d columns count: the bytes from the first to one past the last
inline size_t span_bytes(uint32_t rows, uint32_t d, uint32_t ld, size_t es) {
    return rows == 0 ? 0 : (static_cast<size_t>(rows - 1) * ld + d) * es;
}
inline bool spans_overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}
// an output matrix may be an input matrix itself (same address, same stride) or lie apart from it
inline bool in_place_or_apart(const void* in, uint32_t ld_in, const void* out, uint32_t ld_out, uint32_t rows,
                              uint32_t d, size_t es) {
    return (in == out && ld_in == ld_out) ||
           !spans_overlap(in, span_bytes(rows, d, ld_in, es), out, span_bytes(rows, d, ld_out, es));
}
// lets `kernel` have `bytes` of dynamic shared memory.  Without asking it has 48 KiB, of which static
// shared memory is a part: `unasked` of them are had anyway.  allowed: the kernel's own.
template <typename... Params>
inline dct_status_t allow_shared(void (*kernel)(Params...), size_t bytes, SharedLimit& allowed, size_t unasked = 32 * 1024) {
    if (bytes <= unasked) return DCT_OK;
    int dev = 0;
    const dct_status_t st = current_device(&dev);
    if (st != DCT_OK) return st;
    DCT_CUDA_TRY(static_cast<cudaError_t>(allowed.raise(dev, static_cast<uint32_t>(bytes), [&](uint32_t most) {
        return static_cast<int>(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most)));
    })));
    return DCT_OK;
}

inline float log2_scale(float inv_t) { return static_cast<float>(1.4426950408889634 * inv_t); }
inline bool usable_temperature(float inv_t) { return std::isfinite(inv_t) && inv_t > 0.0f; }

}  // namespace dct
