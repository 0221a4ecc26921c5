// What the kernels of the 8-bit floating-point operators share: the format (e4m3 codes, one power of two a block
// of 128), conversions, launch arguments.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <utility>

#include "pvq.h"

namespace pvq {
// pvq_host.cu
int set_cuda_error(cudaError_t e);
bool is_aligned(const void* p, size_t a);

namespace fp8 {

constexpr int kBlock = 128;              // values that share a scale, along a row
constexpr int kSms = 148;
constexpr uint32_t kFiniteEnd = 0x7f800000u;  // the magnitude bits of an fp32 from which on it is not finite

// A matrix of the format as the kernels see it.  `shift`: a row's scales are those of row >> shift (7: tiles of 128 rows).
struct Matrix {
    uint8_t* codes;
    uint8_t* scales;
    int64_t rows, cols, ld_codes, ld_scales;
    int shift;
    int blocks;  // of a row
};

// i / d for 0 <= i < 2^31, 1 <= d < 2^31: the upper word of a product, shifted.  With s = ceil(log2 d) and
// mul = ceil(2^(31+s) / d) < 2^32, i * mul / 2^(31+s) exceeds i / d by less than 1 / d, so the floors agree.
struct Division {
    uint32_t mul, d;
    int shift;
};
inline Division division_by(int64_t d) {
    int s = 0;
    while ((int64_t(1) << s) < d) ++s;
    if (s == 0) return {0u, 1u, 0};
    const unsigned long long one = 1ull << (31 + s), dd = static_cast<unsigned long long>(d);
    return {static_cast<uint32_t>((one + dd - 1) / dd), static_cast<uint32_t>(d), s - 1};
}
__device__ __forceinline__ uint32_t divide(uint32_t i, const Division& v) { return v.mul ? __umulhi(i, v.mul) >> v.shift : i; }

// The exponent byte (e8m0, 2^(byte - 127)) of a block whose largest finite magnitude has the bits `amax`: the smallest
// power of two s, from 2^-126, with amax <= 448 s; 1 for a block of zeros.  448 = 1.75 * 2^8, so the exponent is amax's
// less 8, and one more where the mantissa is above 1.75 (the addition carries then).
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
    const int e = static_cast<int>((amax + 0x1fffffu) >> 23) - 8;
    return amax == 0u ? 127u : static_cast<uint32_t>(e < 1 ? 1 : e);
}
// 1 / scale: exact, and so is its product with the block's values (those that leave the normal range are far below
// half of e4m3's smallest step).
__device__ __forceinline__ float inverse_of(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// The scale itself; byte 0 is 2^-127 (subnormal), byte 255 NaN.
__device__ __forceinline__ float scale_of(uint32_t byte) {
    return __uint_as_float(byte == 0u ? 0x00400000u : (byte == 255u ? 0x7fffffffu : byte << 23));
}

// Two values to two codes, rounded to nearest even (the first in the low byte); NaN to NaN.
__device__ __forceinline__ uint32_t codes_of(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// Two codes to two values, exact.
__device__ __forceinline__ float2 values_of(uint32_t two) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(two)));
    return __half22float2(*reinterpret_cast<__half2*>(&h));
}

__device__ __forceinline__ uint32_t bf16x2_of(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// As the library's other hot kernels, those here may be set up while the kernel before them in the stream still runs: every
// thread calls dependency_wait() before it touches global memory, and launch_dependents() once what it holds of the SM
// (tensor memory above all) is its own, so that an early block of the next kernel takes nothing that this one waits for.
__device__ __forceinline__ void dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
template <typename... Params, typename... Args>
inline int launch_early(void (*kernel)(Params...), dim3 grid, unsigned threads, size_t shared, unsigned cluster, cudaStream_t s, Args&&... args) {
    cudaLaunchConfig_t config = {};
    config.gridDim = grid;
    config.blockDim = dim3(threads);
    config.dynamicSmemBytes = shared;
    config.stream = s;
    cudaLaunchAttribute attrs[2];
    attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[0].val.programmaticStreamSerializationAllowed = 1;
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = cluster, attrs[1].val.clusterDim.y = 1, attrs[1].val.clusterDim.z = 1;
    config.attrs = attrs;
    config.numAttrs = cluster > 0 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&config, kernel, std::forward<Args>(args)...);
    return e == cudaSuccess ? PVQ_OK : set_cuda_error(e);
}

// launches
int quantize(const void* x, bool bf16, int64_t ld, const Matrix& q, cudaStream_t s);
int dequantize(const Matrix& q, void* out, bool bf16, int64_t ld, cudaStream_t s);
struct GatedArgs {
    const void *gate, *up;
    int64_t ld_gate, ld_up;
    Matrix h, gate8, up8;  // gate8.codes null: no checkpoint
};
int gated(const GatedArgs& a, bool bf16, int act, cudaStream_t s);
struct GatedBackwardArgs {
    const void* dh;
    int64_t ld_dh;
    Matrix gate8, up8;
    void *dgate, *dup;
    int64_t ld_dgate, ld_dup;
};
int gated_backward(const GatedBackwardArgs& a, bool bf16, int act, cudaStream_t s);
int matmul(const Matrix& a, const Matrix& b, bool transposed, void* out, bool bf16, int64_t ld, uint32_t* status, cudaStream_t s);
size_t weight_grad_workspace(int64_t rows, int64_t inner, int64_t outer);
int weight_grad(const void* dy, int64_t outer, int64_t ld_dy, const Matrix& x, void* out, bool bf16, int64_t ld, void* workspace, uint32_t* status,
                cudaStream_t s);

}  // namespace fp8
}  // namespace pvq
