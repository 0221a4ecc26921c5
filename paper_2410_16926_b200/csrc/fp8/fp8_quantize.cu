// Values to the 8-bit format and back.  Bound by memory: 16384 x 4096 bf16 to codes 32.1 us and 14336 x 4096 codes to bf16 27.9 us,
// 97 and 98% of the copy rate.
#include "fp8_rows.cuh"

namespace pvq {
namespace fp8 {
namespace {

template <class T, int UNITS>
__global__ void __launch_bounds__(kRowThreads) quantize_rows_kernel(const T* x, int64_t ld, Matrix q, Work work) {
    launch_dependents();
    dependency_wait();
    Unit at[UNITS];
    Values<T> v[UNITS];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        at[i] = unit_at<UNITS>(work, q.cols, i);
        load_unit(&v[i], x + at[i].row * ld, at[i], q.cols);
    }
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        Codes c;
        const uint32_t byte = quantize_block(v[i], &c);
        store_unit(q, at[i], c, byte);
    }
}

// Tiles of 128 x 128: a thread block takes one, and holds it in registers between the search and the rounding.
constexpr int kTileThreads = 256, kTileRows = kTileThreads / 8, kRounds = 128 / kTileRows;
template <class T>
__global__ void __launch_bounds__(kTileThreads) quantize_tiles_kernel(const T* x, int64_t ld, Matrix q, Division across) {
    __shared__ uint32_t found[2];
    const uint32_t down = divide(blockIdx.x, across);
    const int block = static_cast<int>(blockIdx.x - down * across.d), col = block * kBlock + (threadIdx.x & 7) * 8;
    const int64_t row0 = int64_t(down) * 128 + threadIdx.x / 8;
    const bool whole = col <= q.cols - 72;
    if (threadIdx.x < 2) found[threadIdx.x] = 0u;
    launch_dependents();
    __syncthreads();
    dependency_wait();
    Values<T> v[kRounds];
    uint32_t m = 0u;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int64_t row = row0 + r * kTileRows;
        if (whole && row < q.rows) v[r].load(x + row * ld, col);
        else v[r].load_some(x + row * ld, col, row < q.rows ? q.cols : 0);
    }
#pragma unroll
    for (int r = 0; r < kRounds; ++r) m = max(m, v[r].magnitude());
    m = __reduce_max_sync(0xffffffffu, m);
    if ((threadIdx.x & 31) == 0) atomicMax(&found[0], m);
    __syncthreads();
    m = found[0];
    const bool finite = m < kFiniteEnd;
    if (!finite) {  // (as in quantize_block)
        m = 0u;
#pragma unroll
        for (int r = 0; r < kRounds; ++r)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t a = __float_as_uint(v[r].pair(i).x) & 0x7fffffffu, b = __float_as_uint(v[r].pair(i).y) & 0x7fffffffu;
                m = max(m, max(a < kFiniteEnd ? a : 0u, b < kFiniteEnd ? b : 0u));
            }
        m = __reduce_max_sync(0xffffffffu, m);
        if ((threadIdx.x & 31) == 0) atomicMax(&found[1], m);
        __syncthreads();
        m = found[1];
    }
    const uint32_t byte = scale_byte(m);
    const float inverse = inverse_of(byte);
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int64_t row = row0 + r * kTileRows;
        Codes c;
        if (finite) {
            c = encode(v[r], inverse);
        } else {
            Values<float> t;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 p = v[r].pair(i);
                t.v[i] = make_float2(__fmaf_rn(p.x, 0.0f, p.x), __fmaf_rn(p.y, 0.0f, p.y));  // (Inf * 0 is NaN)
            }
            c = encode(t, inverse);
        }
        if (row >= q.rows) continue;
        if (whole) c.store(q.codes + row * q.ld_codes, col);
        else c.store_some(q.codes + row * q.ld_codes, col, q.cols);
    }
    if (threadIdx.x == 0) q.scales[down * q.ld_scales + block] = static_cast<uint8_t>(byte);
}

template <class T, int UNITS>
__global__ void __launch_bounds__(kRowThreads) dequantize_kernel(Matrix q, T* out, int64_t ld, Work work) {
    launch_dependents();
    dependency_wait();
    Unit at[UNITS];
    Codes c[UNITS];
    uint32_t byte[UNITS];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        at[i] = unit_at<UNITS>(work, q.cols, i);
        load_unit(&c[i], q.codes + at[i].row * q.ld_codes, at[i], q.cols);
        byte[i] = __ldg(q.scales + (at[i].row >> q.shift) * q.ld_scales + at[i].block);
    }
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        if (!at[i].there) continue;
        const float2 scale = both(scale_of(byte[i]));
        float2 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = mul2(c[i].pair(k), scale);
        store_unit(out + at[i].row * ld, at[i], q.cols, v);
    }
}

template <class T>
int launch_quantize(const void* x, int64_t ld, const Matrix& q, cudaStream_t s) {
    const T* from = static_cast<const T*>(x);
    const Work w = work_of(q);
    if (q.shift) {
        const int64_t tiles = (q.rows + 127) / 128 * q.blocks;
        return launch_early(quantize_tiles_kernel<T>, dim3(static_cast<unsigned>(tiles)), kTileThreads, 0, 0, s, from, ld, q, w.blocks);
    }
    constexpr int kUnits = sizeof(T) == 2 ? 2 : 1;
    return launch_early(quantize_rows_kernel<T, kUnits>, dim3(grid_of<kUnits>(w)), kRowThreads, 0, 0, s, from, ld, q, w);
}
template <class T>
int launch_dequantize(const Matrix& q, void* out, int64_t ld, cudaStream_t s) {
    constexpr int kUnits = 2;
    const Work w = work_of(q);
    return launch_early(dequantize_kernel<T, kUnits>, dim3(grid_of<kUnits>(w)), kRowThreads, 0, 0, s, q, static_cast<T*>(out), ld, w);
}

}  // namespace

int quantize(const void* x, bool bf16, int64_t ld, const Matrix& q, cudaStream_t s) {
    return bf16 ? launch_quantize<__nv_bfloat16>(x, ld, q, s) : launch_quantize<float>(x, ld, q, s);
}

int dequantize(const Matrix& q, void* out, bool bf16, int64_t ld, cudaStream_t s) {
    return bf16 ? launch_dequantize<__nv_bfloat16>(q, out, ld, s) : launch_dequantize<float>(q, out, ld, s);
}

}  // namespace fp8
}  // namespace pvq
