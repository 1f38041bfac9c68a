// Products of matrices in 8 bits, and the gated feed-forward block's first half.
#include "act8.cuh"

namespace dct {
namespace {

constexpr uint32_t kThreads = 256, kRows = 64, kCols = 128, kDepth = 32;

struct Pair {
    Act8 a, b;
};

__device__ __forceinline__ float value_at(const Act8& m, uint32_t row, uint32_t col) {
    if (row >= m.rows || col >= m.cols) return 0.0f;
    float lo, hi;
    act8_values2(m.codes[static_cast<size_t>(row) * m.ld + col], lo, hi);
    return __fmul_rn(lo, act8_power(m.scales[act8_scale_offset(m.row_tiles, row, col >> 7)]));
}

// acc += the tile's part of A B^T; a thread has rows 4 rg .. and columns 8 cx ..
__device__ void multiply(float (&acc)[4][8], const Act8& a, const Act8& b, uint32_t row0, uint32_t col0) {
    __shared__ float sa[kDepth][kRows + 1], sb[kDepth][kCols + 1];
    const uint32_t cx = threadIdx.x & 15u, rg = threadIdx.x >> 4;
    for (uint32_t k0 = 0; k0 < a.cols; k0 += kDepth) {
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < kRows * kDepth; i += kThreads) sa[i % kDepth][i / kDepth] = value_at(a, row0 + i / kDepth, k0 + i % kDepth);
        for (uint32_t i = threadIdx.x; i < kCols * kDepth; i += kThreads) sb[i % kDepth][i / kDepth] = value_at(b, col0 + i / kDepth, k0 + i % kDepth);
        __syncthreads();
        for (uint32_t k = 0; k < kDepth; ++k) {
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r)
#pragma unroll
                for (uint32_t c = 0; c < 8; ++c) acc[r][c] = fmaf(sa[k][rg * 4 + r], sb[k][cx * 8 + c], acc[r][c]);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) gemm8_kernel(const Pair one, const Pair two, T* c, uint32_t m, uint32_t n, uint32_t ld_c, bool accumulate) {
    const uint32_t row0 = blockIdx.y * kRows, col0 = blockIdx.x * kCols;
    float acc[4][8] = {};
    multiply(acc, one.a, one.b, row0, col0);
    if (two.a.codes) multiply(acc, two.a, two.b, row0, col0);
    const uint32_t cx = threadIdx.x & 15u, rg = threadIdx.x >> 4;
    for (uint32_t r = 0; r < 4; ++r)
        for (uint32_t k = 0; k < 8; ++k) {
            const uint32_t row = row0 + rg * 4 + r, col = col0 + cx * 8 + k;
            if (row >= m || col >= n) continue;
            T* to = c + static_cast<size_t>(row) * ld_c + col;
            *to = from_f32<T>(accumulate ? __fadd_rn(to_f32(*to), acc[r][k]) : acc[r][k]);
        }
}

__device__ void hold(const float (&v)[8], const Act8& out, uint32_t row, uint32_t col) {
    uint32_t m = 0;
    for (uint32_t k = 0; k < 8; ++k) m = max(m, col + k < out.cols ? magnitude(v[k]) : 0u);
    for (uint32_t o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    if (row >= out.rows) return;
    const uint32_t byte = act8_byte(m);
    for (uint32_t k = 0; k < 8; ++k)
        if (col + k < out.cols) out.codes[static_cast<size_t>(row) * out.ld + col + k] = static_cast<uint8_t>(act8_finite4(act8_codes2(__fmul_rn(v[k], act8_inverse(byte)), 0.0f), byte));
    if (col % 128 == 0) out.scales[act8_scale_offset(out.row_tiles, row, col >> 7)] = static_cast<uint8_t>(byte);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) gated8_kernel(const Act8 x, const Act8 w_gate, const Act8 w_up, bool gelu, const Act8 h, T* dense,
                                                          uint32_t ld_h, const Act8 gate, const Act8 up) {
    const uint32_t row0 = blockIdx.y * kRows, col0 = blockIdx.x * kCols;
    float g[4][8] = {}, u[4][8] = {};
    multiply(g, x, w_gate, row0, col0);
    multiply(u, x, w_up, row0, col0);
    const uint32_t cx = threadIdx.x & 15u, rg = threadIdx.x >> 4;
    for (uint32_t r = 0; r < 4; ++r) {
        const uint32_t row = row0 + rg * 4 + r, col = col0 + cx * 8;
        float v[8];
        for (uint32_t k = 0; k < 8; ++k) v[k] = Gate(g[r][k], gelu).times(u[r][k]);
        if (gate.codes) {
            hold(g[r], gate, row, col);
            hold(u[r], up, row, col);
        }
        if (h.codes) hold(v, h, row, col);
        if (dense && row < x.rows)
            for (uint32_t k = 0; k < 8; ++k)
                if (col + k < w_gate.rows) dense[static_cast<size_t>(row) * ld_h + col + k] = from_f32<T>(v[k]);
    }
}

}  // namespace
}  // namespace dct

using namespace dct;

extern "C" dct_status_t dct_gemm8(const dct_act8_t* a, const dct_act8_t* b, const dct_act8_t* a2, const dct_act8_t* b2, void* c,
                                  dct_dtype_t dtype, uint32_t ld_c, int accumulate, dct_stream_t stream_) {
    if (!known_dtype(dtype)) return DCT_ERR_UNSUPPORTED;
    if (!a || !b || !usable(a) || !usable(b) || a->cols != b->cols || (a2 == nullptr) != (b2 == nullptr)) return DCT_ERR_INVALID_ARG;
    const uint32_t m = a->rows, n = b->rows;
    if (a2 && (!usable(a2) || !usable(b2) || a2->cols != b2->cols || a2->rows != m || b2->rows != n)) return DCT_ERR_INVALID_ARG;
    if (ld_c < n) return DCT_ERR_INVALID_ARG;
    if (m == 0 || n == 0) return DCT_OK;
    const size_t es = element_size(dtype);
    if (!c || !aligned_to(c, es)) return DCT_ERR_INVALID_ARG;
    Buffers all;
    all.write(c, m, n * es, ld_c * es);
    all.read(a);
    all.read(b);
    all.read(a2);
    all.read(b2);
    if (all.clash()) return DCT_ERR_INVALID_ARG;
    const dim3 grid(ceil_div(n, kCols), ceil_div(m, kRows));
    if (grid.y > 65535u) return DCT_ERR_UNSUPPORTED;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const Pair one{device_view(a), device_view(b)}, two{device_view(a2), device_view(b2)};
    if (dtype == DCT_F32)
        gemm8_kernel<<<grid, kThreads, 0, stream>>>(one, two, static_cast<float*>(c), m, n, ld_c, accumulate != 0);
    else
        gemm8_kernel<<<grid, kThreads, 0, stream>>>(one, two, static_cast<__nv_bfloat16*>(c), m, n, ld_c, accumulate != 0);
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}

extern "C" dct_status_t dct_gated8_fwd(const dct_act8_t* x, const dct_act8_t* w_gate, const dct_act8_t* w_up, dct_activation_t activation,
                                       const dct_act8_t* h, void* h_dense, dct_dtype_t dtype, uint32_t ld_h, const dct_act8_t* gate,
                                       const dct_act8_t* up, dct_stream_t stream_) {
    if (!known_dtype(dtype) || (activation != DCT_ACT_SILU && activation != DCT_ACT_GELU)) return DCT_ERR_UNSUPPORTED;
    if (!x || !w_gate || !w_up || !usable(x) || !usable(w_gate) || !usable(w_up)) return DCT_ERR_INVALID_ARG;
    const uint32_t rows = x->rows, d = x->cols, f = w_gate->rows;
    const auto is = [](const dct_act8_t* m, uint32_t r, uint32_t c) { return usable(m) && m->rows == r && m->cols == c; };
    if (w_gate->cols != d || !is(w_up, f, d) || (!h && !h_dense) || (gate == nullptr) != (up == nullptr) || (h && !is(h, rows, f)) ||
        (gate && (!is(gate, rows, f) || !is(up, rows, f))))
        return DCT_ERR_INVALID_ARG;
    const size_t es = element_size(dtype);
    if (h_dense && (ld_h < f || !aligned_to(h_dense, es))) return DCT_ERR_INVALID_ARG;
    if (rows == 0 || f == 0) return DCT_OK;
    Buffers all;
    all.read(x);
    all.read(w_gate);
    all.read(w_up);
    all.write(h);
    all.write(h_dense, rows, f * es, ld_h * es);
    all.write(gate);
    all.write(up);
    if (all.clash()) return DCT_ERR_INVALID_ARG;
    const dim3 grid(ceil_div(f, kCols), ceil_div(rows, kRows));
    if (grid.y > 65535u) return DCT_ERR_UNSUPPORTED;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (dtype == DCT_F32)
        gated8_kernel<<<grid, kThreads, 0, stream>>>(device_view(x), device_view(w_gate), device_view(w_up), activation == DCT_ACT_GELU,
            device_view(h), static_cast<float*>(h_dense), ld_h, device_view(gate), device_view(up));
    else
        gated8_kernel<<<grid, kThreads, 0, stream>>>(device_view(x), device_view(w_gate), device_view(w_up), activation == DCT_ACT_GELU,
            device_view(h), static_cast<__nv_bfloat16*>(h_dense), ld_h, device_view(gate), device_view(up));
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}
