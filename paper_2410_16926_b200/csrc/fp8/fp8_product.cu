// The products of 8-bit matrices, in plain form: tiles of 64 x 64 in shared memory, a 4 x 4 part a thread, fp32
// multiply-adds on the dequantised values.
#include "fp8_rows.cuh"

namespace pvq {
namespace fp8 {
namespace {

constexpr int kTile = 64, kStep = 16, kThreads = 256;

__device__ __forceinline__ float value_at(const Matrix& m, int64_t row, int64_t col) {
    return values_of(m.codes[row * m.ld_codes + col]).x * scale_of(m.scales[(row >> m.shift) * m.ld_scales + col / kBlock]);
}

// operand(i, k): its value; out[i][j] = sum_k a(i,k) b(j,k)
template <class A, class B, class T>
__device__ __forceinline__ void product(const A& a, const B& b, int64_t m, int64_t n, int64_t k, T* out, int64_t ld) {
    __shared__ float as[kStep][kTile + 1], bs[kStep][kTile + 1];
    const int64_t i0 = int64_t(blockIdx.y) * kTile, j0 = int64_t(blockIdx.x) * kTile;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int64_t k0 = 0; k0 < k; k0 += kStep) {
        for (int e = threadIdx.x; e < kTile * kStep; e += kThreads) {
            const int i = a.k_inner ? e / kStep : e % kTile, kk = a.k_inner ? e % kStep : e / kTile;
            as[kk][i] = i0 + i < m && k0 + kk < k ? a(i0 + i, k0 + kk) : 0.0f;
            const int j = b.k_inner ? e / kStep : e % kTile, kb = b.k_inner ? e % kStep : e / kTile;
            bs[kb][j] = j0 + j < n && k0 + kb < k ? b(j0 + j, k0 + kb) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < kStep; ++kk)
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[p][q] = __fmaf_rn(as[kk][ty * 4 + p], bs[kk][tx + 16 * q], acc[p][q]);
        __syncthreads();
    }
    for (int p = 0; p < 4; ++p)
        for (int q = 0; q < 4; ++q) {
            const int64_t i = i0 + ty * 4 + p, j = j0 + tx + 16 * q;
            if (i < m && j < n) out[i * ld + j] = T(acc[p][q]);
        }
}

struct Rows {  // (i, k) of a matrix by rows
    Matrix m;
    static constexpr bool k_inner = true;
    __device__ float operator()(int64_t i, int64_t k) const { return value_at(m, i, k); }
};
struct Columns {  // (i, k) of a matrix [k][i]
    Matrix m;
    static constexpr bool k_inner = false;
    __device__ float operator()(int64_t i, int64_t k) const { return value_at(m, k, i); }
};
struct Bf16Columns {
    const __nv_bfloat16* p;
    int64_t ld;
    static constexpr bool k_inner = false;
    __device__ float operator()(int64_t i, int64_t k) const { return __bfloat162float(p[k * ld + i]); }
};

template <class A, class B, class T>
__global__ void __launch_bounds__(kThreads) product_kernel(A a, B b, int64_t m, int64_t n, int64_t k, T* out, int64_t ld) {
    product(a, b, m, n, k, out, ld);
}

template <class A, class B>
int launch(const A& a, const B& b, int64_t m, int64_t n, int64_t k, void* out, bool bf16, int64_t ld, cudaStream_t s) {
    const dim3 grid(static_cast<unsigned>((n + kTile - 1) / kTile), static_cast<unsigned>((m + kTile - 1) / kTile));
    if (grid.y > 65535u) return PVQ_ERR_UNSUPPORTED;
    if (bf16) product_kernel<<<grid, kThreads, 0, s>>>(a, b, m, n, k, static_cast<__nv_bfloat16*>(out), ld);
    else product_kernel<<<grid, kThreads, 0, s>>>(a, b, m, n, k, static_cast<float*>(out), ld);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? PVQ_OK : set_cuda_error(e);
}

}  // namespace

int matmul(const Matrix& a, const Matrix& b, bool transposed, void* out, bool bf16, int64_t ld, uint32_t*, cudaStream_t s) {
    if (transposed) return launch(Rows{a}, Columns{b}, a.rows, b.cols, a.cols, out, bf16, ld, s);
    return launch(Rows{a}, Rows{b}, a.rows, b.rows, a.cols, out, bf16, ld, s);
}

int weight_grad(const void* dy, int64_t outer, int64_t ld_dy, const Matrix& x, void* out, bool bf16, int64_t ld, uint32_t*, cudaStream_t s) {
    return launch(Bf16Columns{static_cast<const __nv_bfloat16*>(dy), ld_dy}, Columns{x}, outer, x.cols, x.rows, out, bf16, ld, s);
}

}  // namespace fp8
}  // namespace pvq
