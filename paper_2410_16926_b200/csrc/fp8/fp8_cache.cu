// The 8-bit key and value cache: new tokens quantised into their sequences' pages, and read back.
#include "fp8_cache.cuh"

namespace pvq {
namespace fp8 {
namespace {

constexpr int kThreads = 256;

// Eight values as fp32.
template <class T>
__device__ __forceinline__ void load_eight(const T* p, float (&x)[8]) {
    if constexpr (sizeof(T) == 2) {
        const uint4 w = __ldg(reinterpret_cast<const uint4*>(p));
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(u[i] << 16), x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    } else {
        const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    }
}

__device__ __forceinline__ uint32_t finite_bits(float x) {
    const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
    return u < kFiniteEnd ? u : 0u;
}

// Eight codes of values times `inverse`, a power of two; what is not finite becomes NaN, what is beyond the largest code that.
__device__ __forceinline__ uint2 eight_codes(const float (&x)[8], float inverse) {
    uint32_t two[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = x[2 * i] * inverse, b = x[2 * i + 1] * inverse;
        if ((__float_as_uint(x[2 * i]) & 0x7fffffffu) >= kFiniteEnd) a = __uint_as_float(0x7fffffffu);
        if ((__float_as_uint(x[2 * i + 1]) & 0x7fffffffu) >= kFiniteEnd) b = __uint_as_float(0x7fffffffu);
        two[i] = codes_of(a, b);
    }
    return make_uint2(two[0] | two[1] << 16, two[2] | two[3] << 16);
}

// Eight codes for a scale that has grown by 1 / factor: e4m3(code * factor), to nearest even.
__device__ __forceinline__ uint2 rescaled(uint2 c, float factor) {
    uint32_t two[4] = {c.x & 0xffffu, c.x >> 16, c.y & 0xffffu, c.y >> 16};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 v = values_of(two[i]);
        two[i] = codes_of(v.x * factor, v.y * factor);
    }
    return make_uint2(two[0] | two[1] << 16, two[2] | two[3] << 16);
}

// A unit is a page that the step writes to, of a head, keys or values: 16 tokens a warp, their values in registers between the
// search for the largest and the codes.
//
// A sequence with rows a to b gets b / page - a / page + 2 places for its pages, at least as many as it can touch wherever it
// begins, from a / page + 2 s on: no sum over the sequences is needed, only a search for the last s with such a beginning.
template <class T>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(const Cache c, const Step p, const Rows x, int64_t units, uint32_t* status) {
    __shared__ uint32_t most[kThreads / 32];
    dependency_wait();
    launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, page = 1 << c.page_shift, warps = page >> 4;  // (of a unit)
    const int64_t unit = (int64_t(blockIdx.x) * (kThreads / 32) + warp) / warps;
    bool mine = unit < units;
    int s = 0, nth = 0, head = 0, which = 0;
    if (mine) {
        const int64_t place = unit / (2 * c.heads);
        which = static_cast<int>(unit - place * 2 * c.heads);
        head = which >> 1;
        which &= 1;
        if (p.starts) {
            int lo = 0, hi = p.seqs;  // beginning(lo) <= place
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if ((min(max(__ldg(p.starts + mid), 0), p.rows) >> c.page_shift) + 2ll * mid <= place) lo = mid;
                else hi = mid;
            }
            s = lo;
            nth = static_cast<int>(place - (min(max(__ldg(p.starts + s), 0), p.rows) >> c.page_shift) - 2ll * s);
        } else {
            s = static_cast<int>(place);
        }
    }
    Sequence q{};
    int begin = 0, end = 0, row = 0;  // tokens of the page that are written, and the first one's row
    uint8_t *codes = nullptr, *scale = nullptr;
    if (mine) {
        q = sequence_of(p, s, c.page_shift);
        const int from = max(q.first, 0), all = q.first + q.n, to = min(all, q.held);
        if (status && lane == 0 && nth == 0 && which == 0 && head == 0 && q.n > 0 && (q.first < 0 || to < all)) atomicOr(status, PVQ_STATUS_BAD_PAGE);
        const int nth_page = (from >> c.page_shift) + nth;  // of the sequence
        mine = q.n > 0 && nth >= 0 && from < to && nth_page <= (to - 1) >> c.page_shift;  // (nth < 0: rows in front of the first sequence)
        if (mine) {
            const int at = nth_page << c.page_shift;  // the page's first position
            begin = max(from, at) - at, end = min(to - at, page);
            row = q.row + (at + begin - q.first);
            const int id = __ldg(p.table + s * p.ld + nth_page);
            if (id < 0 || id >= c.pages) {
                mine = false;
                if (status && lane == 0) atomicOr(status, PVQ_STATUS_BAD_PAGE);
            } else {
                codes = (which ? c.v : c.k) + id * c.page_step + head * c.head_step;
                scale = (which ? c.v_scales : c.k_scales) + id * c.scale_step + head;
            }
        }
    }
    const int chunks = c.dim >> 3, within = (warp % warps) * 16;  // eight values each; the warp's first token
    const T* values = static_cast<const T*>(which ? x.v : x.k) + head * (which ? x.v_head : x.k_head);
    const int64_t step = which ? x.v_row : x.k_row;
    float v[8][8];
    uint32_t top = 0u;
    uint32_t had = 0u;
    if (mine && begin > 0) had = *scale;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = i * 32 + lane, token = within + at / chunks;
        if (mine && at < 16 * chunks && token >= begin && token < end) {
            load_eight(values + (row + token - begin) * step + (at % chunks) * 8, v[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) top = max(top, finite_bits(v[i][j]));
        }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (warps > 1) {
        if (lane == 0) most[warp] = top;
        __syncthreads();
        for (int i = 0; i < warps; ++i) top = max(top, most[warp / warps * warps + i]);
    }
    if (!mine) return;
    int byte = page_scale_byte(top);
    if (begin > 0) {
        const int before = min(max(static_cast<int>(had), kLeastScale), kMostScale);
        byte = max(byte, before);
        if (byte > before) {  // what the page holds, in the new scale
            const float factor = __uint_as_float(static_cast<uint32_t>(127 - (byte - before)) << 23);
#pragma unroll 1
            for (int i = 0; i < 8; ++i) {
                const int at = i * 32 + lane, token = within + at / chunks;
                if (at < 16 * chunks && token < begin) {
                    uint2* to = reinterpret_cast<uint2*>(codes + token * c.token_step + (at % chunks) * 8);
                    *to = rescaled(*to, factor);
                }
            }
        }
    }
    if (lane == 0 && warp % warps == 0) *scale = static_cast<uint8_t>(byte);
    const float inverse = inverse_of(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = i * 32 + lane, token = within + at / chunks;
        if (at < 16 * chunks && token >= begin && token < end)
            *reinterpret_cast<uint2*>(codes + token * c.token_step + (at % chunks) * 8) = eight_codes(v[i], inverse);
    }
}

constexpr int kReadRows = 16;  // of a block

// Sixteen values a thread; a block finds its rows' places first.
template <class T>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const Cache c, const Step p, const Rows x, uint32_t* status) {
    __shared__ int64_t places[kReadRows][2];  // of codes and scales; -1: none, -2: a row of no sequence
    dependency_wait();
    launch_dependents();
    const int64_t row0 = int64_t(blockIdx.x) * kReadRows;
    if (threadIdx.x < kReadRows) {
        const int64_t row = row0 + threadIdx.x;
        int64_t codes = -2, scale = -2;
        int s = static_cast<int>(row);
        if (p.starts) {
            int lo = 0, hi = p.seqs;  // the last sequence that begins at the row or before
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (__ldg(p.starts + mid) <= row) lo = mid;
                else hi = mid;
            }
            s = lo;
        }
        if (row < p.rows && s < p.seqs) {
            const Sequence q = sequence_of(p, s, c.page_shift);
            if (row >= q.row && row < q.row + q.n) {
                const int at = q.first + static_cast<int>(row - q.row);
                codes = -1;
                if (at >= 0 && at < q.held) {
                    const int id = __ldg(p.table + s * p.ld + (at >> c.page_shift));
                    if (id >= 0 && id < c.pages) {
                        codes = id * c.page_step + (at & ((1 << c.page_shift) - 1)) * c.token_step;
                        scale = id * c.scale_step;
                    }
                }
                if (codes < 0 && status) atomicOr(status, PVQ_STATUS_BAD_PAGE);
            }
        }
        places[threadIdx.x][0] = codes, places[threadIdx.x][1] = scale;
    }
    __syncthreads();
    const int chunks = c.dim >> 4, across = c.heads * chunks;  // sixteen values each
    const uint8_t* from = blockIdx.z ? c.v : c.k;
    const uint8_t* scales = blockIdx.z ? c.v_scales : c.k_scales;
    T* to = static_cast<T*>(blockIdx.z ? x.v : x.k);
    const int64_t row_step = blockIdx.z ? x.v_row : x.k_row, head_step = blockIdx.z ? x.v_head : x.k_head;
    for (int i = threadIdx.x + blockIdx.y * kThreads; i < kReadRows * across; i += kThreads * gridDim.y) {
        const int r = i / across, head = i % across / chunks, col = i % chunks * 16;
        const int64_t place = places[r][0];
        if (place == -2) continue;
        uint4 w = make_uint4(0u, 0u, 0u, 0u);
        float scale = 0.0f;
        if (place >= 0) {
            w = __ldg(reinterpret_cast<const uint4*>(from + place + head * c.head_step + col));
            scale = scale_of(__ldg(scales + places[r][1] + head));
        }
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
        float v[16];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 a = values_of(u[j] & 0xffffu), b = values_of(u[j] >> 16);
            v[4 * j] = a.x * scale, v[4 * j + 1] = a.y * scale, v[4 * j + 2] = b.x * scale, v[4 * j + 3] = b.y * scale;
        }
        T* at = to + (row0 + r) * row_step + head * head_step + col;
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
                reinterpret_cast<uint4*>(at)[j] = make_uint4(bf16x2_of(v[8 * j], v[8 * j + 1]), bf16x2_of(v[8 * j + 2], v[8 * j + 3]),
                                                             bf16x2_of(v[8 * j + 4], v[8 * j + 5]), bf16x2_of(v[8 * j + 6], v[8 * j + 7]));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) reinterpret_cast<float4*>(at)[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        }
    }
}

}  // namespace

int cache_write(const Cache& c, const Step& p, const Rows& x, bool bf16, uint32_t* status, cudaStream_t s) {
    const int64_t places = p.starts ? (int64_t(p.rows) >> c.page_shift) + 2ll * p.seqs : p.seqs, units = places * 2 * c.heads;
    const int64_t blocks = (units * (1 << c.page_shift) / 16 + kThreads / 32 - 1) / (kThreads / 32);
    if (blocks >= int64_t(1) << 31) return PVQ_ERR_UNSUPPORTED;
    void (*const kernel)(Cache, Step, Rows, int64_t, uint32_t*) = bf16 ? cache_write_kernel<__nv_bfloat16> : cache_write_kernel<float>;
    return launch_early(kernel, dim3(static_cast<unsigned>(blocks)), kThreads, 0, 0, s, c, p, x, units, status);
}

int cache_read(const Cache& c, const Step& p, const Rows& x, bool bf16, uint32_t* status, cudaStream_t s) {
    void (*const kernel)(Cache, Step, Rows, uint32_t*) = bf16 ? cache_read_kernel<__nv_bfloat16> : cache_read_kernel<float>;
    return launch_early(kernel, dim3(static_cast<unsigned>((p.rows + kReadRows - 1) / kReadRows), 1, 2), kThreads, 0, 0, s, c, p, x, status);
}

}  // namespace fp8
}  // namespace pvq
