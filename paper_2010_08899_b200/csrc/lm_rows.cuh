// Pieces shared by the layer norm and by the calls on rows of logits: element types, sums over a CTA in a fixed
// order, the order of logits, and the host's argument checks.
#pragma once
#include <cmath>

#include "common.cuh"

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

// Host side ---------------------------------------------------------------------------------------------------

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
inline bool usable_temperature(float inv_t) { return std::isfinite(inv_t) && inv_t > 0.0f; }

}  // namespace dct
