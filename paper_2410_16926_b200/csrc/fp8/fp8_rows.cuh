// Eight threads a block of 128 values, a thread eight of the first 64 and eight of the last 64: what the kernels that go over
// rows of the format share.  (Sixteen threads with eight values each took 4 shuffles for 8 values where this takes 3 for 16.)
//
// All of them are bound by memory, and near enough to the issue of instructions that those are counted: values stay as they
// were loaded until they are needed, magnitudes are compared two or three at a time, products are made in pairs.
#pragma once
#include "fp8_internal.cuh"

namespace pvq {
namespace fp8 {

__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("mul.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<unsigned long long&>(r))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<unsigned long long&>(r))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<unsigned long long&>(r))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)), "l"(reinterpret_cast<unsigned long long&>(c)));
    return r;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// ---- a thread's share of a block

// Sixteen values as they were loaded: columns col .. col+7 and col+64 .. col+71 of a row.
template <class T>
struct Values;
template <>
struct Values<__nv_bfloat16> {
    uint32_t w[8];
    __device__ __forceinline__ float2 pair(int i) const { return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)); }
    // The largest magnitude, as the bits of an fp32; kFiniteEnd or more where one is not finite.
    __device__ __forceinline__ uint32_t magnitude() const {
        uint32_t m = w[0] & 0x7fff7fffu;
#pragma unroll
        for (int i = 1; i < 8; ++i) asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(w[i] & 0x7fff7fffu));
        return max(m << 16, m & 0xffff0000u);
    }
    __device__ __forceinline__ void load(const __nv_bfloat16* row, int col) {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(row + col)), b = __ldg(reinterpret_cast<const uint4*>(row + col + 64));
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
    }
    __device__ __forceinline__ void load_some(const __nv_bfloat16* row, int col, int64_t cols) {
        const uint16_t* r = reinterpret_cast<const uint16_t*>(row);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = col + (i / 4) * 64 + (i % 4) * 2;
            w[i] = (c < cols ? r[c] : 0u) | (c + 1 < cols ? uint32_t(r[c + 1]) << 16 : 0u);
        }
    }
};
// The largest of three magnitudes; NaN where one of them is.
__device__ __forceinline__ float max_abs(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
template <>
struct Values<float> {
    float2 v[8];
    __device__ __forceinline__ float2 pair(int i) const { return v[i]; }
    __device__ __forceinline__ uint32_t magnitude() const {
        float m = max_abs(v[0].x, v[0].x, v[0].y);
#pragma unroll
        for (int i = 1; i < 8; ++i) m = max_abs(m, v[i].x, v[i].y);
        return __float_as_uint(m);
    }
    __device__ __forceinline__ void load(const float* row, int col) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(row + col + (i / 2) * 64 + (i % 2) * 4));
            v[2 * i] = make_float2(a.x, a.y), v[2 * i + 1] = make_float2(a.z, a.w);
        }
    }
    __device__ __forceinline__ void load_some(const float* row, int col, int64_t cols) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = col + (i / 4) * 64 + (i % 4) * 2;
            v[i] = make_float2(c < cols ? row[c] : 0.0f, c + 1 < cols ? row[c + 1] : 0.0f);
        }
    }
};

// Sixteen codes: four words.
struct Codes {
    uint32_t w[4];
    __device__ __forceinline__ float2 pair(int i) const { return values_of(i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu); }
    __device__ __forceinline__ void load(const uint8_t* row, int col) {
        const uint2 a = __ldg(reinterpret_cast<const uint2*>(row + col)), b = __ldg(reinterpret_cast<const uint2*>(row + col + 64));
        w[0] = a.x, w[1] = a.y, w[2] = b.x, w[3] = b.y;
    }
    __device__ __forceinline__ void load_some(const uint8_t* row, int col, int64_t cols) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = 0u;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int c = col + (i / 8) * 64 + i % 8;
            if (c < cols) w[i / 4] |= static_cast<uint32_t>(row[c]) << (8 * (i % 4));
        }
    }
    __device__ __forceinline__ void store(uint8_t* row, int col) const {
        *reinterpret_cast<uint2*>(row + col) = make_uint2(w[0], w[1]);
        *reinterpret_cast<uint2*>(row + col + 64) = make_uint2(w[2], w[3]);
    }
    __device__ __forceinline__ void store_some(uint8_t* row, int col, int64_t cols) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int c = col + (i / 8) * 64 + i % 8;
            if (c < cols) row[c] = static_cast<uint8_t>(w[i / 4] >> (8 * (i % 4)));
        }
    }
};

// Sixteen computed values to memory.
__device__ __forceinline__ void store_values(__nv_bfloat16* row, int col, const float2 (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
        *reinterpret_cast<uint4*>(row + col + 64 * j) =
            make_uint4(bf16x2_of(v[4 * j].x, v[4 * j].y), bf16x2_of(v[4 * j + 1].x, v[4 * j + 1].y), bf16x2_of(v[4 * j + 2].x, v[4 * j + 2].y),
                       bf16x2_of(v[4 * j + 3].x, v[4 * j + 3].y));
}
__device__ __forceinline__ void store_values(float* row, int col, const float2 (&v)[8]) {
    // 32 bytes at a time where the row allows it: two stores of 16 each leave half of every sector to the other (14336 x 4096
    // codes to fp32 57 us, so 45.5)
    if ((reinterpret_cast<uintptr_t>(row) & 31) == 0) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
            asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(row + col + 64 * j), "f"(v[4 * j].x), "f"(v[4 * j].y), "f"(v[4 * j + 1].x),
                         "f"(v[4 * j + 1].y), "f"(v[4 * j + 2].x), "f"(v[4 * j + 2].y), "f"(v[4 * j + 3].x), "f"(v[4 * j + 3].y)
                         : "memory");
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(row + col + (i / 2) * 64 + (i % 2) * 4) = make_float4(v[2 * i].x, v[2 * i].y, v[2 * i + 1].x, v[2 * i + 1].y);
}
template <class T>
__device__ __forceinline__ void store_some(T* row, int col, int64_t cols, const float2 (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = col + (i / 4) * 64 + (i % 4) * 2;
        if (c < cols) row[c] = T(v[i].x);
        if (c + 1 < cols) row[c + 1] = T(v[i].y);
    }
}

// ---- quantisation of a block by its eight threads

// The largest of eight neighbouring threads' (all of them have it).
__device__ __forceinline__ uint32_t max8(uint32_t m) {
#pragma unroll
    for (int d = 4; d; d >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
    return m;
}
// Sixteen values (pair(i) gives two) to codes.
template <class V>
__device__ __forceinline__ Codes encode(const V& v, float inverse) {
    Codes c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 a = mul2(v.pair(2 * i), both(inverse)), b = mul2(v.pair(2 * i + 1), both(inverse));
        c.w[i] = codes_of(a.x, a.y) | codes_of(b.x, b.y) << 16;
    }
    return c;
}
// A block's eight threads quantise it: the scale's byte, and the thread's codes.  All 32 lanes call it.
template <class V>
__device__ __forceinline__ uint32_t quantize_block(const V& v, Codes* codes) {
    uint32_t m = max8(v.magnitude());
    // Rare: where some are not finite, the others' magnitude counts, and these become NaN (e4m3 has no infinity, and a
    // saturated one would pass for a value).
    if (__any_sync(0xffffffffu, m >= kFiniteEnd)) {
        Values<float> t;
        uint32_t f = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            t.v[i] = v.pair(i);
            const uint32_t a = __float_as_uint(t.v[i].x) & 0x7fffffffu, b = __float_as_uint(t.v[i].y) & 0x7fffffffu;
            f = max(f, max(a < kFiniteEnd ? a : 0u, b < kFiniteEnd ? b : 0u));
            t.v[i].x = a < kFiniteEnd ? t.v[i].x : __uint_as_float(0x7fffffffu);
            t.v[i].y = b < kFiniteEnd ? t.v[i].y : __uint_as_float(0x7fffffffu);
        }
        const uint32_t byte = scale_byte(max8(f));
        *codes = encode(t, inverse_of(byte));
        return byte;
    }
    const uint32_t byte = scale_byte(m);
    *codes = encode(v, inverse_of(byte));
    return byte;
}

// ---- blocks of a matrix, one after another, to groups of eight threads: UNITS a thread, a thread block's threads side by side

constexpr int kRowThreads = 128;
struct Work {
    Division blocks;  // of a row
    uint32_t count;
};
inline Work work_of(const Matrix& m) { return {division_by(m.blocks), static_cast<uint32_t>(m.rows * m.blocks)}; }
template <int UNITS>
inline unsigned grid_of(const Work& w) {
    constexpr uint32_t each = UNITS * kRowThreads / 8;
    return w.count / each + (w.count % each != 0);
}
struct Unit {
    bool there, whole;  // whole: all sixteen values lie in the row
    uint32_t row;
    int block, col;
};
template <int UNITS>
__device__ __forceinline__ Unit unit_at(const Work& w, int64_t cols, int i) {
    const uint32_t b = (blockIdx.x * UNITS + i) * (kRowThreads / 8) + threadIdx.x / 8;
    Unit u;
    u.there = b < w.count;
    u.row = divide(u.there ? b : 0u, w.blocks);
    u.block = static_cast<int>((u.there ? b : 0u) - u.row * w.blocks.d);
    u.col = u.block * kBlock + (threadIdx.x & 7) * 8;
    u.whole = u.there && u.col <= cols - 72;  // (64 bits: the last block's col + 72 may be 2^31)
    return u;
}
// What is not there is zeros.
template <class V, class P>
__device__ __forceinline__ void load_unit(V* v, const P* row, const Unit& u, int64_t cols) {
    if (u.whole) v->load(row, u.col);
    else v->load_some(row, u.col, u.there ? cols : 0);
}
__device__ __forceinline__ void store_unit(const Matrix& q, const Unit& u, const Codes& c, uint32_t byte) {
    if (!u.there) return;
    uint8_t* row = q.codes + u.row * q.ld_codes;
    if (u.whole) c.store(row, u.col);
    else c.store_some(row, u.col, q.cols);
    if ((threadIdx.x & 7) == 0) q.scales[u.row * q.ld_scales + u.block] = static_cast<uint8_t>(byte);
}
template <class T>
__device__ __forceinline__ void store_unit(T* row, const Unit& u, int64_t cols, const float2 (&v)[8]) {
    if (u.whole) store_values(row, u.col, v);
    else store_some(row, u.col, cols, v);
}

}  // namespace fp8
}  // namespace pvq
