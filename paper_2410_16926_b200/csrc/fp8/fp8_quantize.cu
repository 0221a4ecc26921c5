// Values to the 8-bit format and back.
#include <algorithm>

#include "fp8_rows.cuh"

namespace pvq {
namespace fp8 {
namespace {

constexpr int kThreads = 256;

// Blocks along rows.  A half warp takes a block; `pairs` blocks of two lie side by side in a row.
template <class T>
__global__ void __launch_bounds__(kThreads) quantize_rows_kernel(const T* x, int64_t ld, Matrix q, Division pairs, uint32_t tasks) {
    const int lane = threadIdx.x & 31, half = lane >> 4;
    const uint32_t task = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (task >= tasks) return;
    const uint32_t row = divide(task, pairs);
    const int block = static_cast<int>(task - row * pairs.d) * 2 + half;
    const int64_t col = int64_t(block) * kBlock + (lane & 15) * 8;
    float v[8];
    load8(x + row * ld, col, q.cols, v);
    uint2 w;
    const uint32_t byte = quantize_block(v, &w);
    store_codes(q.codes + row * q.ld_codes, col, q.cols, w);
    if ((lane & 15) == 0 && block < q.blocks) q.scales[row * q.ld_scales + block] = static_cast<uint8_t>(byte);
}

// Tiles of 128 x 128: a thread block takes one, and holds it in registers between the search and the rounding.
template <class T>
__global__ void __launch_bounds__(kThreads) quantize_tiles_kernel(const T* x, int64_t ld, Matrix q) {
    __shared__ uint32_t found[2];
    constexpr int kRounds = 128 * 16 / kThreads;
    const int64_t row0 = int64_t(blockIdx.y) * 128, col = int64_t(blockIdx.x) * 128 + (threadIdx.x & 15) * 8;
    if (threadIdx.x < 2) found[threadIdx.x] = 0u;
    __syncthreads();
    float v[kRounds][8];
    uint32_t m = 0u;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int64_t row = row0 + r * (kThreads / 16) + (threadIdx.x >> 4);
        if (row < q.rows) {
            load8(x + row * ld, col, q.cols, v[r]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[r][i] = 0.0f;
        }
    }
#pragma unroll
    for (int r = 0; r < kRounds; ++r) m = max(m, magnitude(v[r]));
    atomicMax(&found[0], __reduce_max_sync(0xffffffffu, m));
    __syncthreads();
    const bool finite = found[0] < kFiniteEnd;
    m = found[0];
    if (!finite) {
        m = 0u;
#pragma unroll
        for (int r = 0; r < kRounds; ++r) m = max(m, finite_magnitude(v[r]));
        atomicMax(&found[1], __reduce_max_sync(0xffffffffu, m));
        __syncthreads();
        m = found[1];
    }
    const uint32_t byte = scale_byte(m);
    const float inverse = inverse_of(byte);
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int64_t row = row0 + r * (kThreads / 16) + (threadIdx.x >> 4);
        if (row < q.rows) store_codes(q.codes + row * q.ld_codes, col, q.cols, encode8(v[r], inverse, finite));
    }
    if (threadIdx.x == 0) q.scales[blockIdx.y * q.ld_scales + blockIdx.x] = static_cast<uint8_t>(byte);
}

template <class T>
__global__ void __launch_bounds__(kThreads) dequantize_kernel(Matrix q, T* out, int64_t ld, Division pairs, uint32_t tasks) {
    const int lane = threadIdx.x & 31, half = lane >> 4;
    const uint32_t task = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (task >= tasks) return;
    const uint32_t row = divide(task, pairs);
    const int block = static_cast<int>(task - row * pairs.d) * 2 + half;
    if (block >= q.blocks) return;
    const int64_t col = int64_t(block) * kBlock + (lane & 15) * 8;
    const float scale = scale_of(q.scales[(row >> q.shift) * q.ld_scales + block]);
    float v[8];
    decode8(load_codes(q.codes + row * q.ld_codes, col, q.cols), scale, v);
    store8(out + row * ld, col, q.cols, v);
}

}  // namespace

int quantize(const void* x, bool bf16, int64_t ld, const Matrix& q, cudaStream_t s) {
    if (q.shift) {
        const dim3 grid(static_cast<unsigned>(q.blocks), static_cast<unsigned>((q.rows + 127) / 128));
        if (grid.y > 65535u) return PVQ_ERR_UNSUPPORTED;
        if (bf16) quantize_tiles_kernel<<<grid, kThreads, 0, s>>>(static_cast<const __nv_bfloat16*>(x), ld, q);
        else quantize_tiles_kernel<<<grid, kThreads, 0, s>>>(static_cast<const float*>(x), ld, q);
    } else {
        const int64_t pairs = (q.blocks + 1) / 2, tasks = q.rows * pairs;
        const unsigned grid = static_cast<unsigned>((tasks + kThreads / 32 - 1) / (kThreads / 32));
        const Division d = division_by(pairs);
        if (bf16) quantize_rows_kernel<<<grid, kThreads, 0, s>>>(static_cast<const __nv_bfloat16*>(x), ld, q, d, static_cast<uint32_t>(tasks));
        else quantize_rows_kernel<<<grid, kThreads, 0, s>>>(static_cast<const float*>(x), ld, q, d, static_cast<uint32_t>(tasks));
    }
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? PVQ_OK : set_cuda_error(e);
}

int dequantize(const Matrix& q, void* out, bool bf16, int64_t ld, cudaStream_t s) {
    const int64_t pairs = (q.blocks + 1) / 2, tasks = q.rows * pairs;
    const unsigned grid = static_cast<unsigned>((tasks + kThreads / 32 - 1) / (kThreads / 32));
    const Division d = division_by(pairs);
    if (bf16) dequantize_kernel<<<grid, kThreads, 0, s>>>(q, static_cast<__nv_bfloat16*>(out), ld, d, static_cast<uint32_t>(tasks));
    else dequantize_kernel<<<grid, kThreads, 0, s>>>(q, static_cast<float*>(out), ld, d, static_cast<uint32_t>(tasks));
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? PVQ_OK : set_cuda_error(e);
}

}  // namespace fp8
}  // namespace pvq
