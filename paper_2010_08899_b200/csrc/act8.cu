// Checkpoints in 8 bits: written from fp32 or bf16 by rows and / or transposed, read back, transposed; and the backward pass of the gated
// block, which reads two of them and writes up to five.
//
// A CTA takes tiles of 128 x 128 elements, so that both a row's block and, in the transpose, a column's block are its own.  A thread holds a
// patch of eight rows and eight columns in registers: sixteen neighbouring lanes hold a row's block, and the thread's own eight bytes of a
// column are contiguous in the transpose.  The largest magnitude of a row's block is a maximum over sixteen lanes; that of a column's block
// goes through shared memory, as do the transposed codes, which leave it as whole rows of 128 bytes.
#include "act8.cuh"

namespace dct {
namespace {

constexpr uint32_t kTileThreads = 256;
constexpr uint32_t kPatch = 8;

struct Place {
    uint32_t row0, col0;         // of the tile
    uint32_t row, col;           // of the thread's patch
    uint32_t cx, rg;             // the patch's number among the columns and the rows
};
__device__ __forceinline__ Place place_of(uint32_t tile_row, uint32_t tile_col) {
    const uint32_t lane = threadIdx.x & 31u, cx = lane & 15u, rg = (threadIdx.x >> 5) * 2u + (lane >> 4);
    return Place{tile_row * 128u, tile_col * 128u, tile_row * 128u + rg * kPatch, tile_col * 128u + cx * kPatch, cx, rg};
}

struct TileShared {
    uint32_t largest[8][128];          // per warp and column, then row 0: the columns' bytes
    uint8_t codes[128 * 128];          // transposed: [column][row], groups of eight rows exchanged by column
};

// The patch's rows as blocks of 128 columns
__device__ __forceinline__ void write_rows(const float (&v)[kPatch][kPatch], const Act8& out, const Place& at) {
    const uint32_t block = at.col0 >> 7;
#pragma unroll
    for (uint32_t r = 0; r < kPatch; ++r) {
        uint32_t m = 0;
#pragma unroll
        for (uint32_t c = 0; c < kPatch; ++c) m = max(m, magnitude(v[r][c]));
#pragma unroll
        for (uint32_t o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        const uint32_t byte = act8_byte(m), row = at.row + r;
        if (row >= out.rows) continue;
        const float inverse = act8_inverse(byte);
        uint2 q;
        q.x = act8_codes4(__fmul_rn(v[r][0], inverse), __fmul_rn(v[r][1], inverse), __fmul_rn(v[r][2], inverse), __fmul_rn(v[r][3], inverse));
        q.y = act8_codes4(__fmul_rn(v[r][4], inverse), __fmul_rn(v[r][5], inverse), __fmul_rn(v[r][6], inverse), __fmul_rn(v[r][7], inverse));
        q = make_uint2(act8_finite4(q.x, byte), act8_finite4(q.y, byte));
        uint8_t* to = out.codes + static_cast<size_t>(row) * out.ld + at.col;
        if (at.col + kPatch <= out.cols) {
            *reinterpret_cast<uint2*>(to) = q;
        } else {
            for (uint32_t c = 0; at.col + c < out.cols; ++c) to[c] = static_cast<uint8_t>((c < 4 ? q.x >> (8 * c) : q.y >> (8 * c - 32)));
        }
        if (at.cx == 0) out.scales[act8_scale_offset(out.row_tiles, row, block)] = static_cast<uint8_t>(byte);
    }
}

// The patch's columns as blocks of 128 rows of the transpose
__device__ __forceinline__ void write_columns(const float (&v)[kPatch][kPatch], const Act8& out, const Place& at, TileShared& sh) {
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    __syncthreads();                 // the last plane's readers are done
#pragma unroll
    for (uint32_t c = 0; c < kPatch; ++c) {
        uint32_t m = 0;
#pragma unroll
        for (uint32_t r = 0; r < kPatch; ++r) m = max(m, magnitude(v[r][c]));
        m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
        if (lane < 16) sh.largest[warp][at.cx * kPatch + c] = m;
    }
    __syncthreads();
    if (threadIdx.x < 128) {
        uint32_t m = 0;
#pragma unroll
        for (uint32_t w = 0; w < 8; ++w) m = max(m, sh.largest[w][threadIdx.x]);
        const uint32_t byte = act8_byte(m), row = at.col0 + threadIdx.x;
        if (row < out.rows) out.scales[act8_scale_offset(out.row_tiles, row, at.row0 >> 7)] = static_cast<uint8_t>(byte);
        sh.largest[0][threadIdx.x] = byte;
    }
    __syncthreads();
#pragma unroll
    for (uint32_t c = 0; c < kPatch; ++c) {
        const uint32_t byte = sh.largest[0][at.cx * kPatch + c];
        const float inverse = act8_inverse(byte);
        uint2 q;
        q.x = act8_codes4(__fmul_rn(v[0][c], inverse), __fmul_rn(v[1][c], inverse), __fmul_rn(v[2][c], inverse), __fmul_rn(v[3][c], inverse));
        q.y = act8_codes4(__fmul_rn(v[4][c], inverse), __fmul_rn(v[5][c], inverse), __fmul_rn(v[6][c], inverse), __fmul_rn(v[7][c], inverse));
        q = make_uint2(act8_finite4(q.x, byte), act8_finite4(q.y, byte));
        // (a half-warp's sixteen patches write sixteen different groups: no two to the same bank)
        *reinterpret_cast<uint2*>(sh.codes + (at.cx * kPatch + c) * 128u + ((at.rg ^ at.cx) << 3)) = q;
    }
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        const uint32_t c = i * 16u + (threadIdx.x >> 4), group = threadIdx.x & 15u;
        const uint32_t row = at.col0 + c, col = at.row0 + group * 8u;           // of the transpose
        if (row >= out.rows || col >= out.cols) continue;
        const uint2 q = *reinterpret_cast<const uint2*>(sh.codes + c * 128u + ((group ^ (c >> 3)) << 3));
        uint8_t* to = out.codes + static_cast<size_t>(row) * out.ld + col;
        if (col + 8 <= out.cols) {
            *reinterpret_cast<uint2*>(to) = q;
        } else {
            for (uint32_t k = 0; col + k < out.cols; ++k) to[k] = static_cast<uint8_t>((k < 4 ? q.x >> (8 * k) : q.y >> (8 * k - 32)));
        }
    }
}

// A dense matrix: eight elements of one row, zeros outside.  aligned: rows start on 16-byte boundaries.
template <typename T> struct Dense {
    const T* x;
    uint32_t rows, cols, ld;
    bool aligned;
    __device__ __forceinline__ void load(float (&v)[kPatch], uint32_t row, uint32_t col) const {
        const T* p = x + static_cast<size_t>(row) * ld + col;
        if (row < rows && aligned && col + kPatch <= cols) {
            constexpr uint32_t E = Unit<T>::kElems;
#pragma unroll
            for (uint32_t u = 0; u < kPatch / E; ++u) {
                const uint4 w = ld_unit(reinterpret_cast<const uint4*>(p) + u);
#pragma unroll
                for (uint32_t i = 0; i < E; ++i) v[u * E + i] = Unit<T>::get(w, i);
            }
        } else {
#pragma unroll
            for (uint32_t i = 0; i < kPatch; ++i) v[i] = row < rows && col + i < cols ? to_f32(p[i]) : 0.0f;
        }
    }
};

// Eight values of a row of a matrix in 8 bits, zeros outside.  (Rows start on 16-byte boundaries and are as long as a multiple of 16, so
// the eight codes can be read together wherever one of them counts.)
__device__ __forceinline__ uint2 act8_load(const Act8& m, uint32_t row, uint32_t col) {
    if (row >= m.rows || col >= m.cols) return make_uint2(0, 0);
    uint2 q = *reinterpret_cast<const uint2*>(m.codes + static_cast<size_t>(row) * m.ld + col);
    if (col + kPatch > m.cols) {
        const uint32_t n = m.cols - col;          // 1 to 7
        q.x = n >= 4 ? q.x : q.x & ((1u << 8 * n) - 1u);
        q.y = n <= 4 ? 0u : q.y & ((1u << (8 * n - 32)) - 1u);
    }
    return q;
}
__device__ __forceinline__ float act8_power_at(const Act8& m, uint32_t row, uint32_t col) {
    return row < m.rows && col < m.cols ? act8_power(m.scales[act8_scale_offset(m.row_tiles, row, col >> 7)]) : 0.0f;
}
__device__ __forceinline__ void act8_values(float (&v)[kPatch], const uint2& q, float power) {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t w = i < 2 ? q.x : q.y;
        float lo, hi;
        act8_values2(i & 1 ? w >> 16 : w & 0xFFFFu, lo, hi);
        v[2 * i] = __fmul_rn(lo, power);
        v[2 * i + 1] = __fmul_rn(hi, power);
    }
}

struct Held {
    Act8 a;
    __device__ __forceinline__ void load(float (&v)[kPatch], uint32_t row, uint32_t col) const {
        act8_values(v, act8_load(a, row, col), act8_power_at(a, row, col));
    }
};

template <typename Source>
__global__ void __launch_bounds__(kTileThreads, 2) act8_write_kernel(const Source source, const Act8 out, const Act8 out_t) {
    __shared__ TileShared sh;
    const Place at = place_of(blockIdx.y, blockIdx.x);
    float v[kPatch][kPatch];
#pragma unroll
    for (uint32_t r = 0; r < kPatch; ++r) source.load(v[r], at.row + r, at.col);
    if (out.codes) write_rows(v, out, at);
    if (out_t.codes) write_columns(v, out_t, at, sh);
}

template <typename T>
__global__ void __launch_bounds__(kTileThreads) act8_unpack_kernel(const Act8 a, T* y, const uint32_t ld_y, const bool aligned) {
    const Place at = place_of(blockIdx.y, blockIdx.x);
#pragma unroll
    for (uint32_t r = 0; r < kPatch; ++r) {
        const uint32_t row = at.row + r;
        if (row >= a.rows || at.col >= a.cols) continue;
        float v[kPatch];
        act8_values(v, act8_load(a, row, at.col), act8_power_at(a, row, at.col));
        T* to = y + static_cast<size_t>(row) * ld_y + at.col;
        if (aligned && at.col + kPatch <= a.cols) {
            constexpr uint32_t E = Unit<T>::kElems;
#pragma unroll
            for (uint32_t u = 0; u < kPatch / E; ++u) {
                float g[E];
#pragma unroll
                for (uint32_t i = 0; i < E; ++i) g[i] = v[u * E + i];
                st_unit(to + u * E, Unit<T>::pack(g));
            }
        } else {
#pragma unroll
            for (uint32_t i = 0; i < kPatch; ++i)
                if (at.col + i < a.cols) to[i] = from_f32<T>(v[i]);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kTileThreads, 1)
gated_bwd_kernel(const Dense<T> dh, const Act8 gate, const Act8 up, const bool gelu, const Act8 dgate, const Act8 dup,
                 const Act8 dgate_t, const Act8 dup_t, const Act8 h_t) {
    __shared__ TileShared sh;
    const Place at = place_of(blockIdx.y, blockIdx.x);
    const bool want_gate = dgate.codes || dgate_t.codes, want_up = dup.codes || dup_t.codes;
    float v[kPatch][kPatch];
    for (uint32_t plane = 0; plane < 3; ++plane) {
        if (plane == 0 ? !want_gate : plane == 1 ? !want_up : h_t.codes == nullptr) continue;
#pragma unroll
        for (uint32_t r = 0; r < kPatch; ++r) {
            float g[kPatch], u[kPatch], d[kPatch];
            act8_values(g, act8_load(gate, at.row + r, at.col), act8_power_at(gate, at.row + r, at.col));
            if (plane != 1) act8_values(u, act8_load(up, at.row + r, at.col), act8_power_at(up, at.row + r, at.col));
            if (plane != 2) dh.load(d, at.row + r, at.col);
#pragma unroll
            for (uint32_t c = 0; c < kPatch; ++c) {
                const Gate a(g[c], gelu);
                v[r][c] = plane == 0 ? a.slope_times(__fmul_rn(d[c], u[c])) : a.times(plane == 1 ? d[c] : u[c]);
            }
        }
        if (plane == 0 && dgate.codes) write_rows(v, dgate, at);
        if (plane == 1 && dup.codes) write_rows(v, dup, at);
        const Act8& turned = plane == 0 ? dgate_t : plane == 1 ? dup_t : h_t;
        if (turned.codes) write_columns(v, turned, at, sh);
    }
}

// the grid of 128 x 128 tiles; false if it is beyond what one launch takes
bool tile_grid(uint32_t rows, uint32_t cols, dim3* grid) {
    *grid = dim3(ceil_div(cols, 128), ceil_div(rows, 128));
    return grid->y <= 65535u;
}

template <typename T> bool unit_rows(const void* p, uint32_t ld) {
    return aligned_to(p, 16) && static_cast<size_t>(ld) * sizeof(T) % 16 == 0;
}
template <typename T> Dense<T> dense(const void* x, uint32_t rows, uint32_t cols, uint32_t ld) {
    return Dense<T>{static_cast<const T*>(x), rows, cols, ld, unit_rows<T>(x, ld)};
}

bool sized(const dct_act8_t* m, uint32_t rows, uint32_t cols) { return m->rows == rows && m->cols == cols && usable(m); }

}  // namespace
}  // namespace dct

using namespace dct;

extern "C" size_t dct_act8_scale_bytes(uint32_t rows, uint32_t cols) {
    return rows > DCT_ACT8_MAX_DIM || cols > DCT_ACT8_MAX_DIM ? 0 : act8_scale_bytes(rows, cols);
}

extern "C" dct_status_t dct_act8_pack(const void* x, dct_dtype_t dtype, uint32_t rows, uint32_t cols, uint32_t ld,
                                      const dct_act8_t* out, const dct_act8_t* out_t, dct_stream_t stream_) {
    if (!known_dtype(dtype)) return DCT_ERR_UNSUPPORTED;
    if ((!out && !out_t) || ld < cols || (out && !sized(out, rows, cols)) || (out_t && !sized(out_t, cols, rows)) ||
        rows > DCT_ACT8_MAX_DIM || cols > DCT_ACT8_MAX_DIM)
        return DCT_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return DCT_OK;
    const size_t es = element_size(dtype);
    if (!x || !aligned_to(x, es)) return DCT_ERR_INVALID_ARG;
    Buffers all;
    all.read(x, rows, cols * es, ld * es);
    all.write(out);
    all.write(out_t);
    if (all.clash()) return DCT_ERR_INVALID_ARG;
    dim3 grid;
    if (!tile_grid(rows, cols, &grid)) return DCT_ERR_UNSUPPORTED;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (dtype == DCT_F32)
        act8_write_kernel<<<grid, kTileThreads, 0, stream>>>(dense<float>(x, rows, cols, ld), device_view(out), device_view(out_t));
    else
        act8_write_kernel<<<grid, kTileThreads, 0, stream>>>(dense<__nv_bfloat16>(x, rows, cols, ld), device_view(out), device_view(out_t));
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}

extern "C" dct_status_t dct_act8_unpack(const dct_act8_t* a, void* y, dct_dtype_t dtype, uint32_t ld_y, dct_stream_t stream_) {
    if (!known_dtype(dtype)) return DCT_ERR_UNSUPPORTED;
    if (!a || !usable(a) || ld_y < a->cols) return DCT_ERR_INVALID_ARG;
    if (a->rows == 0 || a->cols == 0) return DCT_OK;
    const size_t es = element_size(dtype);
    if (!y || !aligned_to(y, es)) return DCT_ERR_INVALID_ARG;
    Buffers all;
    all.read(a);
    all.write(y, a->rows, a->cols * es, ld_y * es);
    if (all.clash()) return DCT_ERR_INVALID_ARG;
    dim3 grid;
    if (!tile_grid(a->rows, a->cols, &grid)) return DCT_ERR_UNSUPPORTED;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (dtype == DCT_F32)
        act8_unpack_kernel<<<grid, kTileThreads, 0, stream>>>(device_view(a), static_cast<float*>(y), ld_y, unit_rows<float>(y, ld_y));
    else
        act8_unpack_kernel<<<grid, kTileThreads, 0, stream>>>(device_view(a), static_cast<__nv_bfloat16*>(y), ld_y,
                                                              unit_rows<__nv_bfloat16>(y, ld_y));
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}

extern "C" dct_status_t dct_act8_transpose(const dct_act8_t* a, const dct_act8_t* out_t, dct_stream_t stream_) {
    if (!a || !out_t || !usable(a) || !sized(out_t, a->cols, a->rows)) return DCT_ERR_INVALID_ARG;
    if (a->rows == 0 || a->cols == 0) return DCT_OK;
    Buffers all;
    all.read(a);
    all.write(out_t);
    if (all.clash()) return DCT_ERR_INVALID_ARG;
    dim3 grid;
    if (!tile_grid(a->rows, a->cols, &grid)) return DCT_ERR_UNSUPPORTED;
    act8_write_kernel<<<grid, kTileThreads, 0, static_cast<cudaStream_t>(stream_)>>>(Held{device_view(a)}, device_view(nullptr), device_view(out_t));
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}

extern "C" dct_status_t dct_gated8_bwd(const void* dh, dct_dtype_t dtype, uint32_t ld_dh, const dct_act8_t* gate, const dct_act8_t* up,
                                       dct_activation_t activation, const dct_act8_t* dgate, const dct_act8_t* dup,
                                       const dct_act8_t* dgate_t, const dct_act8_t* dup_t, const dct_act8_t* h_t, dct_stream_t stream_) {
    if (!known_dtype(dtype) || (activation != DCT_ACT_SILU && activation != DCT_ACT_GELU)) return DCT_ERR_UNSUPPORTED;
    if (!gate || !up || !usable(gate) || !sized(up, gate->rows, gate->cols)) return DCT_ERR_INVALID_ARG;
    const uint32_t rows = gate->rows, f = gate->cols;
    const dct_act8_t* outs[5] = {dgate, dup, dgate_t, dup_t, h_t};
    bool any = false;
    for (int i = 0; i < 5; ++i) {
        if (!outs[i]) continue;
        any = true;
        if (!(i < 2 ? sized(outs[i], rows, f) : sized(outs[i], f, rows))) return DCT_ERR_INVALID_ARG;
    }
    const bool gradients = dgate || dup || dgate_t || dup_t;
    if (!any || (gradients && ld_dh < f)) return DCT_ERR_INVALID_ARG;
    if (rows == 0 || f == 0) return DCT_OK;
    const size_t es = element_size(dtype);
    if (gradients && (!dh || !aligned_to(dh, es))) return DCT_ERR_INVALID_ARG;
    Buffers all;
    if (gradients) all.read(dh, rows, f * es, ld_dh * es);
    all.read(gate);
    all.read(up);
    for (const dct_act8_t* m : outs) all.write(m);
    if (all.clash()) return DCT_ERR_INVALID_ARG;
    dim3 grid;
    if (!tile_grid(rows, f, &grid)) return DCT_ERR_UNSUPPORTED;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const bool gelu = activation == DCT_ACT_GELU;
    if (dtype == DCT_F32)
        gated_bwd_kernel<<<grid, kTileThreads, 0, stream>>>(dense<float>(dh, rows, f, ld_dh), device_view(gate), device_view(up), gelu,
            device_view(dgate), device_view(dup), device_view(dgate_t), device_view(dup_t), device_view(h_t));
    else
        gated_bwd_kernel<<<grid, kTileThreads, 0, stream>>>(dense<__nv_bfloat16>(dh, rows, f, ld_dh), device_view(gate), device_view(up), gelu,
            device_view(dgate), device_view(dup), device_view(dgate_t), device_view(dup_t), device_view(h_t));
    DCT_CUDA_TRY(cudaGetLastError());
    return DCT_OK;
}
