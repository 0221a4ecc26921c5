// The middle of a gated feed-forward block, h = act(gate) * up, with its result and its checkpoints in the 8-bit format,
// and its backward pass from the checkpoints.
//
// Both activations are g * sigma(w(g)): silu with w = g, gelu (the form with tanh) with w = 2 sqrt(2/pi) (g + 0.044715 g^3),
// since (1 + tanh z) / 2 = sigma(2 z).  Their slope is s + g s (1 - s) w'(g), s = sigma(w).
//
// Bound by memory, near the issue of instructions (56% of the slots): forward with checkpoints 16384 x 14336 bf16 295 us, 87% of
// the copy rate, backward 1999 x 14336 40.0 us, 89%.
#include "fp8_rows.cuh"

namespace pvq {
namespace fp8 {
namespace {

constexpr float kGelu = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float kCubic = 0.044715f;

// 1 / (1 + e^-w), from -w / ln 2: the exponential and the reciprocal by the special function unit, within 2^-22 and 2^-23 of
// their values; e^-w may be infinite (the result is zero then).
__device__ __forceinline__ float2 sigma(float2 minus_w) {
    float2 e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(minus_w.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(minus_w.y));
    e = add2(e, both(1.0f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(e.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(e.y));
    return r;
}

constexpr float kMinusLog2E = -1.4426950408889634f;

template <int ACT>
__device__ __forceinline__ float2 activation(float2 g) {
    if (ACT == PVQ_ACT_SILU) return mul2(g, sigma(mul2(g, both(kMinusLog2E))));
    const float2 w = mul2(mul2(g, both(kGelu)), fma2(mul2(g, both(kCubic)), g, both(1.0f)));
    return mul2(g, sigma(mul2(w, both(kMinusLog2E))));
}
// The activation and its slope.
template <int ACT>
__device__ __forceinline__ void activation_slope(float2 g, float2* value, float2* slope) {
    if (ACT == PVQ_ACT_SILU) {
        const float2 s = sigma(mul2(g, both(kMinusLog2E)));
        *value = mul2(g, s);
        *slope = fma2(*value, fma2(s, both(-1.0f), both(1.0f)), s);
        return;
    }
    const float2 square = make_float2(fminf(g.x * g.x, 1e30f), fminf(g.y * g.y, 1e30f));  // (no infinity to be multiplied by s (1 - s) = 0)
    const float2 s = sigma(mul2(mul2(mul2(g, both(kGelu)), fma2(square, both(kCubic), both(1.0f))), both(kMinusLog2E)));
    *value = mul2(g, s);
    const float2 steep = mul2(fma2(square, both(3.0f * kCubic), both(1.0f)), both(kGelu));
    *slope = fma2(mul2(*value, fma2(s, both(-1.0f), both(1.0f))), steep, s);
}

// Thread blocks an SM that the registers are limited for: 9 of 128 threads (bf16, 56 registers) is 296 us for 16384 x 14336 with
// its checkpoints, 8 and 10 are 302 and 301, no limit (62) 318; in blocks of 256 threads 306 at best, 344 without a limit.
// Backward, silu: 8 is 41.2 us for 1999 x 14336, no limit 42.8, 9 to 12 45; gelu: 7 is 82.9 for 4096 x 14336, 8 97.7, 6 90.5, 10 83.3.
template <class T>
constexpr int kGatedBlocks = sizeof(T) == 2 ? 9 : 6;
template <class T, int ACT>
constexpr int kBackwardBlocks = sizeof(T) == 2 ? (ACT == PVQ_ACT_SILU ? 8 : 7) : 6;

template <class T, int ACT, bool KEEP>
__global__ void __launch_bounds__(kRowThreads, kGatedBlocks<T>) gated_kernel(GatedArgs a, Work work) {
    launch_dependents();
    dependency_wait();
    const Unit at = unit_at<1>(work, a.h.cols, 0);
    Values<T> g, u;
    load_unit(&g, static_cast<const T*>(a.gate) + at.row * a.ld_gate, at, a.h.cols);
    load_unit(&u, static_cast<const T*>(a.up) + at.row * a.ld_up, at, a.h.cols);
    Codes c;
    uint32_t byte;
    if (KEEP) {
        byte = quantize_block(g, &c);
        store_unit(a.gate8, at, c, byte);
        byte = quantize_block(u, &c);
        store_unit(a.up8, at, c, byte);
    }
    Values<float> h;
#pragma unroll
    for (int i = 0; i < 8; ++i) h.v[i] = mul2(activation<ACT>(g.pair(i)), u.pair(i));
    byte = quantize_block(h, &c);
    store_unit(a.h, at, c, byte);
}

template <class T, int ACT>
__global__ void __launch_bounds__(kRowThreads, kBackwardBlocks<T, ACT>) gated_backward_kernel(GatedBackwardArgs a, Work work) {
    launch_dependents();
    dependency_wait();
    const int64_t cols = a.gate8.cols;
    const Unit at = unit_at<1>(work, cols, 0);
    if (!at.there) return;
    Values<T> dh;
    Codes gate, up;
    load_unit(&dh, static_cast<const T*>(a.dh) + at.row * a.ld_dh, at, cols);
    load_unit(&gate, a.gate8.codes + at.row * a.gate8.ld_codes, at, cols);
    load_unit(&up, a.up8.codes + at.row * a.up8.ld_codes, at, cols);
    const float2 gate_scale = both(scale_of(__ldg(a.gate8.scales + at.row * a.gate8.ld_scales + at.block)));
    const float2 up_scale = both(scale_of(__ldg(a.up8.scales + at.row * a.up8.ld_scales + at.block)));
    float2 dgate[8], dup[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float2 value, slope;
        activation_slope<ACT>(mul2(gate.pair(i), gate_scale), &value, &slope);
        dgate[i] = mul2(mul2(dh.pair(i), mul2(up.pair(i), up_scale)), slope);
        dup[i] = mul2(dh.pair(i), value);
    }
    store_unit(static_cast<T*>(a.dgate) + at.row * a.ld_dgate, at, cols, dgate);
    store_unit(static_cast<T*>(a.dup) + at.row * a.ld_dup, at, cols, dup);
}

template <class T, int ACT>
int launch_gated(const GatedArgs& a, cudaStream_t s) {
    const Work w = work_of(a.h);
    return launch_early(a.gate8.codes ? gated_kernel<T, ACT, true> : gated_kernel<T, ACT, false>, dim3(grid_of<1>(w)), kRowThreads, 0, 0, s, a, w);
}
template <class T, int ACT>
int launch_backward(const GatedBackwardArgs& a, cudaStream_t s) {
    const Work w = work_of(a.gate8);
    return launch_early(gated_backward_kernel<T, ACT>, dim3(grid_of<1>(w)), kRowThreads, 0, 0, s, a, w);
}

}  // namespace

int gated(const GatedArgs& a, bool bf16, int act, cudaStream_t s) {
    if (act == PVQ_ACT_SILU) return bf16 ? launch_gated<__nv_bfloat16, PVQ_ACT_SILU>(a, s) : launch_gated<float, PVQ_ACT_SILU>(a, s);
    return bf16 ? launch_gated<__nv_bfloat16, PVQ_ACT_GELU>(a, s) : launch_gated<float, PVQ_ACT_GELU>(a, s);
}

int gated_backward(const GatedBackwardArgs& a, bool bf16, int act, cudaStream_t s) {
    if (act == PVQ_ACT_SILU) return bf16 ? launch_backward<__nv_bfloat16, PVQ_ACT_SILU>(a, s) : launch_backward<float, PVQ_ACT_SILU>(a, s);
    return bf16 ? launch_backward<__nv_bfloat16, PVQ_ACT_GELU>(a, s) : launch_backward<float, PVQ_ACT_GELU>(a, s);
}

}  // namespace fp8
}  // namespace pvq
