// The middle of a gated feed-forward block, h = act(gate) * up, with its result and its checkpoints in the 8-bit format,
// and its backward pass from the checkpoints.
//
// Both activations are g * sigma(w(g)): silu with w = g, gelu (the form with tanh) with w = 2 sqrt(2/pi) (g + 0.044715 g^3),
// since (1 + tanh z) / 2 = sigma(2 z).  Their slope is s + g s (1 - s) w'(g), s = sigma(w).
#include "fp8_rows.cuh"

namespace pvq {
namespace fp8 {
namespace {

constexpr int kThreads = 256;

constexpr float kGelu = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float kCubic = 0.044715f;

// 1 / (1 + e^-w): the exponential and the reciprocal by the special function unit, within 2^-22 and 2^-23 of their
// values; e^-w may be infinite (the result is zero then).
__device__ __forceinline__ float sigma(float w) {
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(w * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    return r;
}

template <int ACT>
__device__ __forceinline__ float activation(float g) {
    return g * sigma(ACT == PVQ_ACT_SILU ? g : kGelu * g * __fmaf_rn(kCubic * g, g, 1.0f));
}
// The activation and its slope.
template <int ACT>
__device__ __forceinline__ float2 activation_slope(float g) {
    if (ACT == PVQ_ACT_SILU) {
        const float s = sigma(g), a = g * s;
        return make_float2(a, __fmaf_rn(a, 1.0f - s, s));
    }
    const float square = fminf(g * g, 1e30f);  // (no infinity to be multiplied by s (1 - s) = 0)
    const float s = sigma(kGelu * g * __fmaf_rn(kCubic, square, 1.0f)), a = g * s;
    return make_float2(a, __fmaf_rn(a * (1.0f - s), kGelu * __fmaf_rn(3.0f * kCubic, square, 1.0f), s));
}

template <class T, int ACT, bool KEEP>
__global__ void __launch_bounds__(kThreads) gated_kernel(GatedArgs a, Division pairs, uint32_t tasks) {
    const int lane = threadIdx.x & 31, half = lane >> 4;
    const uint32_t task = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (task >= tasks) return;
    const uint32_t row = divide(task, pairs);
    const int block = static_cast<int>(task - row * pairs.d) * 2 + half;
    const int64_t col = int64_t(block) * kBlock + (lane & 15) * 8;
    const bool first = (lane & 15) == 0 && block < a.h.blocks;
    float g[8], u[8], h[8];
    load8(static_cast<const T*>(a.gate) + row * a.ld_gate, col, a.h.cols, g);
    load8(static_cast<const T*>(a.up) + row * a.ld_up, col, a.h.cols, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = activation<ACT>(g[i]) * u[i];
    uint2 w;
    uint32_t byte = quantize_block(h, &w);
    store_codes(a.h.codes + row * a.h.ld_codes, col, a.h.cols, w);
    if (first) a.h.scales[row * a.h.ld_scales + block] = static_cast<uint8_t>(byte);
    if (KEEP) {
        byte = quantize_block(g, &w);
        store_codes(a.gate8.codes + row * a.gate8.ld_codes, col, a.h.cols, w);
        if (first) a.gate8.scales[row * a.gate8.ld_scales + block] = static_cast<uint8_t>(byte);
        byte = quantize_block(u, &w);
        store_codes(a.up8.codes + row * a.up8.ld_codes, col, a.h.cols, w);
        if (first) a.up8.scales[row * a.up8.ld_scales + block] = static_cast<uint8_t>(byte);
    }
}

template <class T, int ACT>
__global__ void __launch_bounds__(kThreads) gated_backward_kernel(GatedBackwardArgs a, Division pairs, uint32_t tasks) {
    const int lane = threadIdx.x & 31, half = lane >> 4;
    const uint32_t task = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (task >= tasks) return;
    const uint32_t row = divide(task, pairs);
    const int block = static_cast<int>(task - row * pairs.d) * 2 + half;
    if (block >= a.gate8.blocks) return;
    const int64_t col = int64_t(block) * kBlock + (lane & 15) * 8, cols = a.gate8.cols;
    float dh[8], g[8], u[8];
    load8(static_cast<const T*>(a.dh) + row * a.ld_dh, col, cols, dh);
    decode8(load_codes(a.gate8.codes + row * a.gate8.ld_codes, col, cols),
            scale_of(a.gate8.scales[row * a.gate8.ld_scales + block]), g);
    decode8(load_codes(a.up8.codes + row * a.up8.ld_codes, col, cols), scale_of(a.up8.scales[row * a.up8.ld_scales + block]), u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 as = activation_slope<ACT>(g[i]);
        g[i] = dh[i] * u[i] * as.y;
        u[i] = dh[i] * as.x;
    }
    store8(static_cast<T*>(a.dgate) + row * a.ld_dgate, col, cols, g);
    store8(static_cast<T*>(a.dup) + row * a.ld_dup, col, cols, u);
}

template <class T, int ACT>
void launch_gated(const GatedArgs& a, unsigned grid, const Division& d, uint32_t tasks, cudaStream_t s) {
    if (a.gate8.codes) gated_kernel<T, ACT, true><<<grid, kThreads, 0, s>>>(a, d, tasks);
    else gated_kernel<T, ACT, false><<<grid, kThreads, 0, s>>>(a, d, tasks);
}

}  // namespace

int gated(const GatedArgs& a, bool bf16, int act, cudaStream_t s) {
    const int64_t pairs = (a.h.blocks + 1) / 2, tasks = a.h.rows * pairs;
    const unsigned grid = static_cast<unsigned>((tasks + kThreads / 32 - 1) / (kThreads / 32));
    const Division d = division_by(pairs);
    const uint32_t n = static_cast<uint32_t>(tasks);
    if (act == PVQ_ACT_SILU) {
        if (bf16) launch_gated<__nv_bfloat16, PVQ_ACT_SILU>(a, grid, d, n, s);
        else launch_gated<float, PVQ_ACT_SILU>(a, grid, d, n, s);
    } else {
        if (bf16) launch_gated<__nv_bfloat16, PVQ_ACT_GELU>(a, grid, d, n, s);
        else launch_gated<float, PVQ_ACT_GELU>(a, grid, d, n, s);
    }
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? PVQ_OK : set_cuda_error(e);
}

int gated_backward(const GatedBackwardArgs& a, bool bf16, int act, cudaStream_t s) {
    const int64_t pairs = (a.gate8.blocks + 1) / 2, tasks = a.gate8.rows * pairs;
    const unsigned grid = static_cast<unsigned>((tasks + kThreads / 32 - 1) / (kThreads / 32));
    const Division d = division_by(pairs);
    const uint32_t n = static_cast<uint32_t>(tasks);
    if (act == PVQ_ACT_SILU) {
        if (bf16) gated_backward_kernel<__nv_bfloat16, PVQ_ACT_SILU><<<grid, kThreads, 0, s>>>(a, d, n);
        else gated_backward_kernel<float, PVQ_ACT_SILU><<<grid, kThreads, 0, s>>>(a, d, n);
    } else {
        if (bf16) gated_backward_kernel<__nv_bfloat16, PVQ_ACT_GELU><<<grid, kThreads, 0, s>>>(a, d, n);
        else gated_backward_kernel<float, PVQ_ACT_GELU><<<grid, kThreads, 0, s>>>(a, d, n);
    }
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? PVQ_OK : set_cuda_error(e);
}

}  // namespace fp8
}  // namespace pvq
