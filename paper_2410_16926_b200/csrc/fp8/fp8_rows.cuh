// Eight values of a row a thread, sixteen threads a block of 128: what the kernels that go over rows of the format share.
#pragma once
#include "fp8_internal.cuh"

namespace pvq {
namespace fp8 {

// Values col .. col+7 of a row (16-byte aligned); those from `cols` on are zeros and are not read.
__device__ __forceinline__ void load8(const __nv_bfloat16* row, int64_t col, int64_t cols, float (&v)[8]) {
    if (col + 8 <= cols) {
        const uint4 w = __ldg(reinterpret_cast<const uint4*>(row + col));
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < cols ? __bfloat162float(row[col + i]) : 0.0f;
    }
}
__device__ __forceinline__ void load8(const float* row, int64_t col, int64_t cols, float (&v)[8]) {
    if (col + 8 <= cols) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(row + col)), b = __ldg(reinterpret_cast<const float4*>(row + col + 4));
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < cols ? row[col + i] : 0.0f;
    }
}
__device__ __forceinline__ void store8(__nv_bfloat16* row, int64_t col, int64_t cols, const float (&v)[8]) {
    if (col + 8 <= cols) {
        *reinterpret_cast<uint4*>(row + col) =
            make_uint4(bf16x2_of(v[0], v[1]), bf16x2_of(v[2], v[3]), bf16x2_of(v[4], v[5]), bf16x2_of(v[6], v[7]));
    } else {
        for (int i = 0; i < 8 && col + i < cols; ++i) row[col + i] = __float2bfloat16_rn(v[i]);
    }
}
__device__ __forceinline__ void store8(float* row, int64_t col, int64_t cols, const float (&v)[8]) {
    if (col + 8 <= cols) {
        *reinterpret_cast<float4*>(row + col) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4*>(row + col + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        for (int i = 0; i < 8 && col + i < cols; ++i) row[col + i] = v[i];
    }
}

// Eight codes, as two words; codes from `cols` on are zeros and are not read.
__device__ __forceinline__ uint2 load_codes(const uint8_t* row, int64_t col, int64_t cols) {
    if (col + 8 <= cols) return __ldg(reinterpret_cast<const uint2*>(row + col));
    uint32_t w[2] = {0u, 0u};
    for (int i = 0; i < 8 && col + i < cols; ++i) w[i >> 2] |= static_cast<uint32_t>(row[col + i]) << (8 * (i & 3));
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void store_codes(uint8_t* row, int64_t col, int64_t cols, uint2 w) {
    if (col + 8 <= cols) {
        *reinterpret_cast<uint2*>(row + col) = w;
    } else {
        for (int i = 0; i < 8 && col + i < cols; ++i) row[col + i] = static_cast<uint8_t>((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    }
}

// The largest magnitude of eight values, as bits; not finite ones give kFiniteEnd or more.
__device__ __forceinline__ uint32_t magnitude(const float (&v)[8]) {
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
}
// ... of the finite ones alone
__device__ __forceinline__ uint32_t finite_magnitude(const float (&v)[8]) {
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
        m = max(m, b < kFiniteEnd ? b : 0u);
    }
    return m;
}
// The largest of sixteen neighbouring threads' (all of them have it).
__device__ __forceinline__ uint32_t max16(uint32_t m) {
#pragma unroll
    for (int d = 8; d; d >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
    return m;
}

// Eight values to codes; what is not finite becomes NaN (Inf * 0 is NaN; e4m3 has no infinity, and a saturated one would
// pass for a value).
__device__ __forceinline__ uint2 encode8(const float (&v)[8], float inverse, bool finite) {
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = v[i] * inverse;
    if (!finite) {
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = __fmaf_rn(v[i], 0.0f, t[i]);
    }
    return make_uint2(codes_of(t[0], t[1]) | codes_of(t[2], t[3]) << 16, codes_of(t[4], t[5]) | codes_of(t[6], t[7]) << 16);
}
__device__ __forceinline__ void decode8(uint2 w, float scale, float (&v)[8]) {
    const float2 a = values_of(w.x & 0xffffu), b = values_of(w.x >> 16), c = values_of(w.y & 0xffffu), d = values_of(w.y >> 16);
    v[0] = a.x * scale, v[1] = a.y * scale, v[2] = b.x * scale, v[3] = b.y * scale;
    v[4] = c.x * scale, v[5] = c.y * scale, v[6] = d.x * scale, v[7] = d.y * scale;
}

// A block's sixteen threads quantise it: returns its scale byte, `w` the thread's codes.  All 32 lanes call it.
__device__ __forceinline__ uint32_t quantize_block(const float (&v)[8], uint2* w) {
    uint32_t m = max16(magnitude(v));
    const bool finite = m < kFiniteEnd;
    if (__any_sync(0xffffffffu, !finite)) {  // rare: once more without what is not finite
        const uint32_t f = max16(finite_magnitude(v));
        if (!finite) m = f;
    }
    const uint32_t byte = scale_byte(m);
    *w = encode8(v, inverse_of(byte), finite);
    return byte;
}

}  // namespace fp8
}  // namespace pvq
