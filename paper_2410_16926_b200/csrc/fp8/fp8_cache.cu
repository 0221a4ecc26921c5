// The 8-bit key and value cache: new tokens quantised into their sequences' pages, and read back.
#include "fp8_cache.cuh"

namespace pvq {
namespace fp8 {
namespace {

constexpr int kThreads = 256;
constexpr int kFewTokens = 8;  // of a sequence, on average, up to which 16 threads take a page

// Eight values of a thread, as they were loaded.
template <class T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
    uint4 w;
    __device__ __forceinline__ void load(const void* p) { w = __ldg(static_cast<const uint4*>(p)); }
    __device__ __forceinline__ void values(float (&x)[8]) const {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(u[i] << 16), x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
    __device__ __forceinline__ uint32_t largest() const {  // bits of the largest magnitude, as fp32, NaN above all
        uint32_t m = w.x & 0x7fff7fffu;
        asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(w.y & 0x7fff7fffu));
        asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(w.z & 0x7fff7fffu));
        asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(w.w & 0x7fff7fffu));
        return max(m << 16, m & 0x7fff0000u);
    }
};
template <>
struct Eight<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const void* p) { a = __ldg(static_cast<const float4*>(p)), b = __ldg(static_cast<const float4*>(p) + 1); }
    __device__ __forceinline__ void values(float (&x)[8]) const { x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w; }
    __device__ __forceinline__ uint32_t largest() const {
        const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        uint32_t m = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
        return m;
    }
};
// The largest finite magnitude's bits, where some are not.
template <class T>
__device__ __forceinline__ uint32_t largest_finite(const Eight<T>& v) {
    float x[8];
    v.values(x);
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t u = __float_as_uint(x[i]) & 0x7fffffffu;
        m = max(m, u < kFiniteEnd ? u : 0u);
    }
    return m;
}

// Eight codes of values times `inverse`, a power of two; beyond the largest code that one.  ODD: what is not finite becomes NaN.
template <bool ODD>
__device__ __forceinline__ uint2 eight_codes(const float (&x)[8], float inverse) {
    uint32_t two[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = x[2 * i] * inverse, b = x[2 * i + 1] * inverse;
        if (ODD && (__float_as_uint(x[2 * i]) & 0x7fffffffu) >= kFiniteEnd) a = __uint_as_float(0x7fffffffu);
        if (ODD && (__float_as_uint(x[2 * i + 1]) & 0x7fffffffu) >= kFiniteEnd) b = __uint_as_float(0x7fffffffu);
        two[i] = codes_of(a, b);
    }
    return make_uint2(two[0] | two[1] << 16, two[2] | two[3] << 16);
}

// The last of `count` sequences for which at(s) <= what, or 0: at is ascending.  A warp looks at 32 of them at a time.
template <class F>
__device__ __forceinline__ int last_at_most(int count, int64_t what, F&& at) {
    const int lane = threadIdx.x & 31;
    int lo = 0, n = count;  // it is among lo .. lo + n - 1, or 0
    while (n > 1) {
        const int step = (n + 31) / 32, s = lo + lane * step;
        const uint32_t below = __ballot_sync(0xffffffffu, lane * step < n && at(s) <= what);
        const int nth = below ? 31 - __clz(below) : 0;
        n = min(step, n - nth * step);
        lo += nth * step;
    }
    return lo;
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
//
// What bounds it: what has to be known one after the other (starts, lengths, the page's number, values) with four blocks an SM, and issue (69 %): 18400
// rows of 8 heads of 128, bf16, 27.1 us from a graph (fp32 39.0), of which the bytes take 17.9 at the copy rate.  (Comparing values one by one, and holding them as fp32: 78 us.)
template <class T>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 2) cache_write_kernel(const Cache c, const Step p, const Rows x, int64_t units, uint32_t* status) {
    __shared__ uint32_t most[kThreads / 32];
    dependency_wait();
    launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, page = 1 << c.page_shift, warps = page >> 4;  // (of a unit)
    const int64_t unit = (int64_t(blockIdx.x) * (kThreads / 32) + warp) >> (c.page_shift - 4);
    bool mine = unit < units;
    const uint32_t per_place = 2 * c.heads, place = static_cast<uint32_t>(unit) / per_place;  // (units are fewer than 2^31)
    const int head = (static_cast<uint32_t>(unit) - place * per_place) >> 1, which = unit & 1;
    int s = static_cast<int>(place), nth = 0;
    if (p.starts) {
        const auto start = [&](int i) { return min(max(__ldg(p.starts + i), 0), p.rows) >> c.page_shift; };
        s = last_at_most(p.seqs, place, [&](int i) { return start(i) + 2ll * i; });
        nth = static_cast<int>(place - start(s) - 2ll * s);  // (negative: rows in front of the first sequence)
    }
    int begin = 0, end = 0, row = 0, id = -1;  // tokens of the page that are written, the first one's row, the page's number
    if (mine) {
        const Sequence q = sequence_of(p, s, c.page_shift);
        const int from = max(q.first, 0), all = q.first + q.n, to = min(all, q.held);
        if (status && lane == 0 && nth == 0 && which == 0 && head == 0 && q.n > 0 && (q.first < 0 || to < all)) atomicOr(status, PVQ_STATUS_BAD_PAGE);
        const int nth_page = (from >> c.page_shift) + nth;  // of the sequence
        mine = q.n > 0 && nth >= 0 && from < to && nth_page <= (to - 1) >> c.page_shift;
        if (mine) {
            const int at = nth_page << c.page_shift;  // the page's first position
            begin = max(from, at) - at, end = min(to - at, page);
            row = q.row + (at + begin - q.first);
            id = __ldg(p.table + s * p.ld + nth_page);
        }
    }
    const int chunks = c.dim >> 3, within = (warp & (warps - 1)) * 16;  // eight values each; the warp's first token
    const T* values = static_cast<const T*>(which ? x.v : x.k) + head * (which ? x.v_head : x.k_head);
    const int64_t step = which ? x.v_row : x.k_row;
    const uint32_t by_chunks = (65536u + chunks - 1) / chunks;  // at / chunks for at < 256: exact, since chunks <= 16
    const auto token_of = [&](int at) { return within + static_cast<int>(at * by_chunks >> 16); };
    Eight<T> v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = i * 32 + lane, token = token_of(at);
        if (mine && at < 16 * chunks && token >= begin && token < end) v[i].load(values + (row + token - begin) * step + (at - (token - within) * chunks) * 8);
    }
    uint8_t *codes = nullptr, *scale = nullptr;
    uint32_t had = 0u;
    if (mine) {
        if (id < 0 || id >= c.pages) {
            mine = false;
            if (status && lane == 0) atomicOr(status, PVQ_STATUS_BAD_PAGE);
        } else {
            codes = (which ? c.v : c.k) + id * c.page_step + head * c.head_step;
            scale = (which ? c.v_scales : c.k_scales) + id * c.scale_step + head;
            if (begin > 0) had = *scale;
        }
    }
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = i * 32 + lane, token = token_of(at);
        if (mine && at < 16 * chunks && token >= begin && token < end) top = max(top, v[i].largest());
    }
    const bool finite = top < kFiniteEnd;
    if (!finite) {
        top = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int at = i * 32 + lane, token = token_of(at);
            if (mine && at < 16 * chunks && token >= begin && token < end) top = max(top, largest_finite(v[i]));
        }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (warps > 1) {
        if (lane == 0) most[warp] = top;
        __syncthreads();  // (and the scale was read by all warps)
        for (int i = 0; i < warps; ++i) top = max(top, most[(warp & ~(warps - 1)) + i]);
    }
    if (!mine) return;
    int byte = page_scale_byte(top);
    if (begin > 0) {
        const int before = min(max(static_cast<int>(had), kLeastScale), kMostScale);
        byte = max(byte, before);
        if (byte > before) {  // what the page holds, in the new scale
            const float factor = __uint_as_float(static_cast<uint32_t>(127 - (byte - before)) << 23);
#pragma unroll 4
            for (int i = 0; i < 8; ++i) {
                const int at = i * 32 + lane, token = token_of(at);
                if (at < 16 * chunks && token < begin) {
                    uint2* to = reinterpret_cast<uint2*>(codes + token * c.token_step + (at - (token - within) * chunks) * 8);
                    *to = rescaled(*to, factor);
                }
            }
        }
    }
    if (lane == 0 && within == 0) *scale = static_cast<uint8_t>(byte);
    const float inverse = inverse_of(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = i * 32 + lane, token = token_of(at);
        if (at < 16 * chunks && token >= begin && token < end) {
            float y[8];
            v[i].values(y);
            *reinterpret_cast<uint2*>(codes + token * c.token_step + (at - (token - within) * chunks) * 8) =
                finite ? eight_codes<false>(y, inverse) : eight_codes<true>(y, inverse);
        }
    }
}

// The same for few tokens a sequence: 16 threads a unit, eight dims each, which go through its tokens four at a time; up to four stay in registers.
// One token of 256 sequences 2.7 us (by 16 tokens a warp: 4.6 in pages of 16, 22 in pages of 128); 64 sequences of 8 tokens, pages of 64, 5.5 and 8.9; of 16
// tokens 8.7 and 9.3, in pages of 16 6.2 and 5.8.
template <class T>
__global__ void __launch_bounds__(kThreads) cache_write_few_kernel(const Cache c, const Step p, const Rows x, int64_t units, uint32_t* status) {
    dependency_wait();
    launch_dependents();
    const int64_t unit = (int64_t(blockIdx.x) * kThreads + threadIdx.x) >> 4;
    const int col = (threadIdx.x & 15) * 8;
    const bool leads = col == 0, there = unit < units;
    const uint32_t per_place = 2 * c.heads, place = static_cast<uint32_t>(there ? unit : 0) / per_place;
    const int head = (static_cast<uint32_t>(there ? unit : 0) - place * per_place) >> 1, which = unit & 1;
    int s = static_cast<int>(place), nth = 0;
    if (p.starts) {
        const auto start = [&](int i) { return min(max(__ldg(p.starts + i), 0), p.rows) >> c.page_shift; };
        int lo = 0, hi = p.seqs;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (start(mid) + 2ll * mid <= place) lo = mid;
            else hi = mid;
        }
        s = lo;
        nth = static_cast<int>(place - start(s) - 2ll * s);
    }
    const Sequence q = sequence_of(p, s, c.page_shift);
    const int from = max(q.first, 0), all = q.first + q.n, to = min(all, q.held), nth_page = (from >> c.page_shift) + nth;
    if (there && status && leads && nth == 0 && which == 0 && head == 0 && q.n > 0 && (q.first < 0 || to < all)) atomicOr(status, PVQ_STATUS_BAD_PAGE);
    bool mine = there && q.n > 0 && nth >= 0 && from < to && nth_page <= (to - 1) >> c.page_shift;
    int begin = 0, n = 0, id = -1;
    const T* values = nullptr;
    if (mine) {
        const int at = nth_page << c.page_shift;
        begin = max(from, at) - at, n = min(to - at, 1 << c.page_shift) - begin;
        id = __ldg(p.table + s * p.ld + nth_page);
        values = static_cast<const T*>(which ? x.v : x.k) + (q.row + (at + begin - q.first)) * (which ? x.v_row : x.k_row) + head * (which ? x.v_head : x.k_head) + col;
    }
    const int64_t step = which ? x.v_row : x.k_row;
    if (col >= c.dim) n = 0;  // (of no dims)
    Eight<T> v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) v[i].load(values + i * step);
    if (mine && (id < 0 || id >= c.pages)) {
        mine = false;
        n = 0;
        if (status && leads) atomicOr(status, PVQ_STATUS_BAD_PAGE);
    }
    uint8_t* codes = (which ? c.v : c.k) + (mine ? id * c.page_step + head * c.head_step : 0) + col;
    uint8_t* scale = (which ? c.v_scales : c.k_scales) + (mine ? id * c.scale_step + head : 0);
    const uint32_t had = mine && begin > 0 ? *scale : 0u;
    uint32_t top = 0u;
    for (int t = 0; t < n; t += 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (t + i < n) {
                if (t > 0) v[i].load(values + (t + i) * step);
                const uint32_t m = v[i].largest();
                top = max(top, m < kFiniteEnd ? m : largest_finite(v[i]));
            }
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));  // (and the scale was read by all)
    if (!mine) return;
    int byte = page_scale_byte(top);
    if (begin > 0) {
        const int before = min(max(static_cast<int>(had), kLeastScale), kMostScale);
        byte = max(byte, before);
        if (byte > before && col < c.dim) {  // what the page holds, in the new scale
            const float factor = __uint_as_float(static_cast<uint32_t>(127 - (byte - before)) << 23);
#pragma unroll 8
            for (int t = 0; t < begin; ++t) {
                uint2* at = reinterpret_cast<uint2*>(codes + t * c.token_step);
                *at = rescaled(*at, factor);
            }
        }
    }
    if (leads) *scale = static_cast<uint8_t>(byte);
    const float inverse = inverse_of(byte);
    for (int t = 0; t < n; t += 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (t + i < n) {
                if (n > 4) v[i].load(values + (t + i) * step);
                float y[8];
                v[i].values(y);
                *reinterpret_cast<uint2*>(codes + (begin + t + i) * c.token_step) = eight_codes<true>(y, inverse);
            }
    }
}

constexpr int kMostRows = 32;  // of a reading block

// 32 bytes of result a thread, of two rows at once.  A warp of the block finds its rows' places first.  Bound by memory: 43500 tokens of 8 heads of
// 128 to bf16 89.3 us from a graph, of which the bytes take 81.7 at the copy rate.
template <class T>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const Cache c, const Step p, const Rows x, int rows, uint32_t* status) {
    constexpr int kEach = 32 / sizeof(T);
    __shared__ int64_t places[kMostRows][2];  // of codes and scales; -1: none, -2: a row of no sequence
    dependency_wait();
    launch_dependents();
    const int64_t row0 = int64_t(blockIdx.x) * rows;
    if (threadIdx.x < 32) {
        const int64_t row = row0 + threadIdx.x;
        int64_t codes = -2, scale = -2;
        int s = static_cast<int>(min(row, int64_t(p.seqs) - 1));
        if (p.starts) {  // the first row's sequence, or one behind it
            s = last_at_most(p.seqs, row0, [&](int i) { return __ldg(p.starts + i); });
            if (s + 1 < p.seqs && __ldg(p.starts + s + 1) <= row) {
                int lo = s + 1, hi = p.seqs;
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (__ldg(p.starts + mid) <= row) lo = mid;
                    else hi = mid;
                }
                s = lo;
            }
        }
        if (threadIdx.x < rows && row < p.rows) {
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
        if (threadIdx.x < rows) places[threadIdx.x][0] = codes, places[threadIdx.x][1] = scale;
    }
    const uint32_t chunks = c.dim / kEach, across = c.heads * chunks;  // of a row
    const uint8_t* from = blockIdx.z ? c.v : c.k;
    const uint8_t* scales = blockIdx.z ? c.v_scales : c.k_scales;
    T* to = static_cast<T*>(blockIdx.z ? x.v : x.k) + row0 * (blockIdx.z ? x.v_row : x.k_row);
    const int64_t row_step = blockIdx.z ? x.v_row : x.k_row, head_step = blockIdx.z ? x.v_head : x.k_head;
    const uint32_t groups = across < kThreads ? kThreads / across : 1, group = across < kThreads ? threadIdx.x / across : 0;  // of threads, a row each
    __syncthreads();
    if (group >= groups) return;
    for (uint32_t i = threadIdx.x - group * across; i < across; i += kThreads) {
        const uint32_t head = i / chunks, col = (i - head * chunks) * kEach;
        const int64_t code_at = head * c.head_step + col, value_at = head * head_step + col;
        for (uint32_t r0 = group; r0 < rows; r0 += 2 * groups) {
            uint4 w[2];
            uint32_t byte[2];
            bool any[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t r = r0 + j * groups;
                const int64_t place = r < rows ? places[r][0] : -2;
                any[j] = place != -2;
                w[j] = make_uint4(0u, 0u, 0u, 0u);
                byte[j] = 127u;
                if (place < 0) continue;
                if constexpr (kEach == 16) {
                    w[j] = __ldg(reinterpret_cast<const uint4*>(from + place + code_at));
                } else {
                    const uint2 two = __ldg(reinterpret_cast<const uint2*>(from + place + code_at));
                    w[j].x = two.x, w[j].y = two.y;
                }
                byte[j] = __ldg(scales + places[r][1] + head);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (!any[j]) continue;
                T* at = to + (r0 + j * groups) * row_step + value_at;
                const float scale = scale_of(byte[j]);
                const uint32_t u[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
                float v[kEach];
#pragma unroll
                for (int k = 0; k < kEach / 4; ++k) {
                    const float2 a = values_of(u[k] & 0xffffu), b = values_of(u[k] >> 16);
                    v[4 * k] = a.x * scale, v[4 * k + 1] = a.y * scale, v[4 * k + 2] = b.x * scale, v[4 * k + 3] = b.y * scale;
                }
                if constexpr (sizeof(T) == 2) {
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        reinterpret_cast<uint4*>(at)[k] = make_uint4(bf16x2_of(v[8 * k], v[8 * k + 1]), bf16x2_of(v[8 * k + 2], v[8 * k + 3]),
                                                                     bf16x2_of(v[8 * k + 4], v[8 * k + 5]), bf16x2_of(v[8 * k + 6], v[8 * k + 7]));
                } else {
#pragma unroll
                    for (int k = 0; k < 2; ++k) reinterpret_cast<float4*>(at)[k] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
                }
            }
        }
    }
}

}  // namespace

int cache_write(const Cache& c, const Step& p, const Rows& x, bool bf16, uint32_t* status, cudaStream_t s) {
    const int64_t places = p.starts ? (int64_t(p.rows) >> c.page_shift) + 2ll * p.seqs : p.seqs, units = places * 2 * c.heads;
    const bool few = p.rows <= kFewTokens * int64_t(p.seqs);
    const int64_t blocks = few ? (units * 16 + kThreads - 1) / kThreads : (units * (1 << c.page_shift) / 16 + kThreads / 32 - 1) / (kThreads / 32);
    if (blocks >= int64_t(1) << 27) return PVQ_ERR_UNSUPPORTED;
    void (*const kernel)(Cache, Step, Rows, int64_t, uint32_t*) = few ? (bf16 ? cache_write_few_kernel<__nv_bfloat16> : cache_write_few_kernel<float>)
                                                                      : (bf16 ? cache_write_kernel<__nv_bfloat16> : cache_write_kernel<float>);
    return launch_early(kernel, dim3(static_cast<unsigned>(blocks)), kThreads, 0, 0, s, c, p, x, units, status);
}

int cache_read(const Cache& c, const Step& p, const Rows& x, bool bf16, uint32_t* status, cudaStream_t s) {
    void (*const kernel)(Cache, Step, Rows, int, uint32_t*) = bf16 ? cache_read_kernel<__nv_bfloat16> : cache_read_kernel<float>;
    int rows = kMostRows;  // fewer where the blocks would not fill the SMs
    while (rows > 4 && int64_t(p.rows) < int64_t(rows) * kSms * 4) rows /= 2;
    return launch_early(kernel, dim3(static_cast<unsigned>((p.rows + rows - 1) / rows), 1, 2), kThreads, 0, 0, s, c, p, x, rows, status);
}

}  // namespace fp8
}  // namespace pvq
