// Attention of many query rows over the 8-bit cache: bound by the tensor cores and the exponentials.
//
// A block takes 256 query rows, as two tiles of 128 with four warps each, a thread a row, which compute weights while the tensor cores
// multiply: for each tile of rows there are scores of 64 tokens in two places of tensor memory, so that those of the next 64 are there when the
// weights of these are done.  S = Q K^T from the codes of K as they lie, Q split into two codes (2^-17 of the row's largest),
// which costs what a product of 16-bit operands would, and K needs no conversion.  The weights go back into tensor memory as fp16, over
// the scores, and O += P V takes V as fp16, which four warps make of its codes (exact) for both tiles.
//
// As in the kernel for few rows, exponents of the pages' scales of V are added to the scores, so that weights are relative to the largest of
// w * scale; 16 tokens, of one page, share both scales, which are applied to their largest score and inside the exponent, at no cost
// a score.  Sums of V in tensor memory are rescaled only when a row's largest has grown by 2^8 since.  The largest gets a weight of 2^7, so that fp16 is used up
// to 2^15: a weight is off by 2^-11 of itself, or by 2^-32 of the row's largest, where fp16 ends.
//
// Warps: eight for the weights, four convert V, one issues the copies, one for each tile of rows the products.
//
// What bounds it: the weights' warps, one of each tile of rows in a quarter of the SM.  256 rows by 128 tokens of 128 dims take 2.16 us, about 4000 cycles, two
// steps of 64 tokens of each row; the exponentials' unit needs 2080 of them, the tensor cores 2200.  128 scores a step: 2.8; one thread for both tiles'
// products: 2.46, since an answer from a barrier takes it 200 cycles; scores not loaded ahead: 2.32.
#include "fp8_attention.cuh"

namespace pvq {
namespace fp8 {
namespace {

constexpr int kThreads = 512, kRows = 256;
constexpr int kBytes = kTile * 128;     // a tile's codes, rows of 128 bytes
constexpr int kKeys = 3, kCodes = 2, kValues = 2;  // stages
constexpr int kQueryAt = 0, kKeyAt = 4 * kBytes, kCodeAt = kKeyAt + kKeys * kBytes, kValueAt = kCodeAt + kCodes * kBytes,
              kBarAt = kValueAt + kValues * 2 * kBytes;
constexpr size_t kShared = 1024 + kBarAt + 512;
constexpr float kRoom = 8.0f;           // exponent by which a row's largest may be behind
constexpr float kShift = 7.0f;          // ... and of the weight that it gets: up to 2^15 in all

constexpr int kRegisters = 128, kMany = 168, kFew = 88;
static_assert(2 * kMany + 2 * kFew <= 4 * kRegisters, "a share beyond these would be waited for without end");
static_assert(kShared + 2048 <= 232448, "shared memory");

// D += A B with A in tensor memory, both fp16.
__device__ __forceinline__ void multiply_f16(uint32_t d, uint32_t a, uint64_t b, uint32_t product, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b),
                 "r"(product), "r"(static_cast<uint32_t>(add))
                 : "memory");
}
__device__ __forceinline__ uint32_t f16x2_of(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// 32 of a lane's words to as many columns.
__device__ __forceinline__ void tensor_store32(uint32_t at, const uint32_t (&w)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,"
        "%29,%30,%31,%32};" ::"r"(at),
        "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "r"(w[8]), "r"(w[9]), "r"(w[10]), "r"(w[11]), "r"(w[12]),
        "r"(w[13]), "r"(w[14]), "r"(w[15]), "r"(w[16]), "r"(w[17]), "r"(w[18]), "r"(w[19]), "r"(w[20]), "r"(w[21]), "r"(w[22]), "r"(w[23]), "r"(w[24]),
        "r"(w[25]), "r"(w[26]), "r"(w[27]), "r"(w[28]), "r"(w[29]), "r"(w[30]), "r"(w[31])
        : "memory");
}

// Waits for the loads, of which v's values are not to be looked at before.
__device__ __forceinline__ void tensor_wait(float (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]),
                   "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]),
                   "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29])
                 :
                 : "memory");
    asm volatile("" : "+f"(v[30]), "+f"(v[31]));
}
// Two values at a time.
__device__ __forceinline__ float2 two_fma(float2 a, float2 b, float2 c) {
    float2 r;
    asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 a, a, b, c;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}
__device__ __forceinline__ float2 two_add(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// The largest of 16.
__device__ __forceinline__ float most_of(const float* v) {
    const float a = max3(v[0], v[1], v[2]), b = max3(v[3], v[4], v[5]), c = max3(v[6], v[7], v[8]), d = max3(v[9], v[10], v[11]), e = max3(v[12], v[13], v[14]);
    return max3(max3(a, b, c), max3(d, e, v[15]), a);
}
__device__ __forceinline__ void hide(float (&v)[32], int begin, int end) {
#pragma unroll
    for (int i = 0; i < 32; ++i)
        if (i < begin || i >= end) v[i] = kNone;
}

__global__ void __launch_bounds__(kThreads, 1) attention_many_kernel(const __grid_constant__ CacheMaps maps, const __grid_constant__ AttentionArgs p) {
    extern __shared__ uint8_t raw[];
    const uint32_t base = (shared_address(raw) + 1023u) & ~1023u;
    const uint32_t keys_full = base + kBarAt, keys_empty = keys_full + 8 * kKeys, codes_full = keys_empty + 8 * kKeys, codes_empty = codes_full + 8 * kCodes,
                   values_full = codes_empty + 8 * kCodes, values_empty = values_full + 8 * kValues, scores_full = values_empty + 8 * kValues,
                   weights_full = scores_full + 32, queries_full = weights_full + 32, scales_full = queries_full + 16,
                   drained = scales_full + 8 * kScaleSlots;  // (scores, weights: [tile of rows][half of the tokens]; drained: [tile of rows])
    __shared__ uint32_t tensor_base, issued[2];
    __shared__ int over;
    __shared__ PlanShared plan;
    __shared__ __align__(16) float page_scales[kScaleSlots][3][8];  // of 16 tokens each: keys', values' exponent, 1 / values'
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp == 0) {
        constexpr int kCodesEmpty = 2 * kKeys + kCodes, kValuesFull = kCodesEmpty + kCodes, kScores = kValuesFull + 2 * kValues, kAll = kScores + 10 + kScaleSlots + 2;
        for (int i = lane; i < kAll; i += 32) {
            const bool by_warps = (i >= kCodesEmpty && i < kValuesFull + kValues) || (i >= kScores + 4 && i < kScores + 10);  // codes empty, values full, weights, queries
            const bool by_both = (i >= kKeys && i < 2 * kKeys) || (i >= kValuesFull + kValues && i < kScores);  // keys empty, values empty
            barrier_init(keys_full + 8 * i, by_warps ? 4 : (by_both ? 2 : 1));
        }
        barrier_init_fence();
        if (lane == 0) {
            over = 0;
            issued[0] = issued[1] = 0;
            prefetch_map(&maps.k), prefetch_map(&maps.v);
        }
    } else if (warp == 13) {
        tensor_alloc<false>(shared_address(&tensor_base), 512);
    }
    tensor_fence_before();
    __syncthreads();
    tensor_fence_after();
    launch_dependents();
    dependency_wait();
    const uint32_t tensor = tensor_base;
    Bounds bounds{&over, p.status};
    const Withheld withheld = withheld_in(bounds);
    const Share share = find_share<kThreads, kRows>(p, plan, 0);
    Walk<kRows> walk(p, share, plan);

    if (warp < 8) {
        more_registers<kMany>();
        const int which = warp >> 2, row = (warp & 3) * 32 + lane;  // tile of rows, row in it
        const uint32_t mine = (warp & 3) << 21, scores = tensor + mine + which * 128, sums = tensor + mine + 256 + which * 128;
        PartHead* head = part_heads<kRows>(p) + blockIdx.x;
        if (threadIdx.x == 0 && gridDim.x > 1) head->parts = 0;
        const uint32_t scores_bar = scores_full + 16 * which, weights_bar = weights_full + 16 * which;
        uint32_t tile = 0, phase = 0;  // tiles of this block; phases of each half's scores
        int passed = 0;                // tiles of items without rows here since the last that had some
        bool ok = true;
        for (; walk.there(); walk.next()) {
            const Item& it = walk.it;
            const int count = walk.count();
            if (it.rows <= 128 * which) {  // no rows here
                tile += count;
                passed += count;
                continue;
            }
            const RowPlace place = place_of(p, it.q, it.head, it.q0 + min(which * 128 + row, it.rows - 1));
            const int position = it.q.first + place.row - it.q.row;
            const int to = p.causal ? min(it.q.held, position + 1) : it.q.held, from = first_seen(p, position);
            uint32_t byte = 127u;
            // The warp's 32 rows of queries: 16 lanes a row, eight dims each.  None where the item has no tiles in this share: nothing would hold the warps
            // together then, so that one could put its results where another's queries are on their way, and a phase of queries_full pass unseen.
#pragma unroll 1
            for (int i0 = count > 0 ? 0 : 16; i0 < 16; i0 += 8) {
                uint4 w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int r = 2 * (i0 + i) + (lane >> 4);
                    const int64_t at = __shfl_sync(0xffffffffu, place.row * p.q_row + place.head * p.q_head, r);
                    w[i] = make_uint4(0u, 0u, 0u, 0u);
                    if (8 * (lane & 15) < p.cache.dim) w[i] = __ldg(reinterpret_cast<const uint4*>(p.q + at) + (lane & 15));
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int r = (warp & 3) * 32 + 2 * (i0 + i) + (lane >> 4);
                    const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
                    uint32_t most = 0u, hi[4], lo[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) most = max(most, max((u[j] << 16) & 0x7fffffffu, u[j] & 0x7fff0000u));
#pragma unroll
                    for (int o = 1; o < 16; o <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
                    const uint32_t its = most < kFiniteEnd ? scale_byte(most) : 255u;
                    const uint32_t own = __shfl_sync(0xffffffffu, its, (lane & 1) * 16);
                    if ((lane >> 1) == i0 + i) byte = own;
                    const float inverse = inverse_of(its == 255u ? 127u : its);
#pragma unroll
                    for (int j = 0; j < 4; ++j) two_codes(__uint_as_float(u[j] << 16) * inverse, __uint_as_float(u[j] & 0xffff0000u) * inverse, hi[j], lo[j]);
                    const uint32_t at = base + kQueryAt + which * 2 * kBytes + r * 128 + ((((lane & 15) >> 1) ^ (r & 7)) << 4) + (lane & 1) * 8;
                    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(hi[0] | hi[1] << 16), "r"(hi[2] | hi[3] << 16) : "memory");
                    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at + kBytes), "r"(lo[0] | lo[1] << 16), "r"(lo[2] | lo[3] << 16) : "memory");
                }
            }
            async_fence();
            __syncwarp();
            if (lane == 0 && count > 0) barrier_arrive(queries_full + 8 * which);
            const bool finite = byte != 255u;
            // (At least 2^-86, so that no page's scale, 2^-40 at least, makes it 0, times -inf: a score is off by 2^-21 at most, under 2^40.)
            const float factor = fmaxf(finite ? row_factor(byte, p.scale) : p.scale, 0x1p-86f);
            // what every row of the warp sees
            const int all_to = __reduce_min_sync(0xffffffffu, to), all_from = __reduce_max_sync(0xffffffffu, from);
            float top = kNone, weight = 0.0f;
            float s[2][32];
            if (count > 0) {
                // Scores first: when they are there, the slot's scales of eight tiles ago are long past, so that the parity can only mean these.  (Warps
                // that had no rows in the items before did not wait for those items' scales.)
                // The other tile of rows may have all those items before it: a poll more for each of their tiles, of 2.2 us.
                Bounds longer = bounds;
                longer.polls += min(passed, 1 << 24) << 6;
                passed = 0;
                ok = ok && warp_waits(scores_bar, phase & 1, longer) && warp_waits(scales_full + 8 * (tile % kScaleSlots), (tile / kScaleSlots) & 1, bounds);
                tensor_fence_after();
                tensor_load(scores, s[0]);
                tensor_load(scores + 32, s[1]);
            }
            for (int t = 0; t < count; ++t, ++tile, ++phase) {
                const uint32_t slot = tile % kScaleSlots;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int first = (walk.begin() + t) * kTile + 64 * half;
                    const float4 keys = *reinterpret_cast<const float4*>(&page_scales[slot][0][4 * half]), value = *reinterpret_cast<const float4*>(&page_scales[slot][1][4 * half]),
                                 out_of = *reinterpret_cast<const float4*>(&page_scales[slot][2][4 * half]);
                    const float key[4] = {fminf(factor * keys.x, kLargest), fminf(factor * keys.y, kLargest), fminf(factor * keys.z, kLargest),
                                          fminf(factor * keys.w, kLargest)};  // (never inf: times 0)
                    tensor_wait(s[0]);
                    tensor_wait(s[1]);
                    if (first < all_from || first + 64 > all_to) {
                        hide(s[0], from - first, to - first);
                        hide(s[1], from - first - 32, to - first - 32);
                    }
                    const float high = fmaxf(max3(fmaf(most_of(&s[0][0]), key[0], value.x), fmaf(most_of(&s[0][16]), key[1], value.y), fmaf(most_of(&s[1][0]), key[2], value.z)),
                                             fmaf(most_of(&s[1][16]), key[3], value.w));
                    if (t == 0 && half == 0) {
                        top = high;
                    } else if (__any_sync(0xffffffffu, high > top + kRoom)) {
                        // (the products with the weights before are done when the scores behind them are)
                        ok = ok && warp_waits(scores_bar + 8 * (half ^ 1), half ? (phase + 1) & 1 : phase & 1, bounds);
                        tensor_fence_after();
                        const float next = fmaxf(top, high), less = next == kNone ? 1.0f : exp2_of(top - next);
                        weight *= less;
                        top = next;
#pragma unroll 1
                        for (int c = 0; c < 128; c += 16) {
                            float v[16];
                            uint32_t w[16];
                            tensor_load(sums + c, v);
                            tensor_wait_loads();
#pragma unroll
                            for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(v[i] * less);
                            tensor_store(sums + c, w);
                        }
                    }
                    const float against = top == kNone ? 0.0f : top - kShift;
                    const float rest[4] = {value.x - against, value.y - against, value.z - against, value.w - against}, back[4] = {out_of.x, out_of.y, out_of.z, out_of.w};
                    const bool more = half == 0 || t + 1 < count;
                    uint32_t w[32];
                    bool there = false;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const float (&v)[32] = s[c >> 1];
                        const float2 k = make_float2(key[c], key[c]), r = make_float2(rest[c], rest[c]);
                        float2 sum = make_float2(0.0f, 0.0f);
                        // (asked before there is nothing else to do: an answer takes 150 to 200 cycles, also where it is yes)
                        if (c == 2 && more)
                            there = barrier_over(scores_bar + 8 * (half ^ 1), (phase + half) & 1) &&
                                    (half == 0 || barrier_over(scales_full + 8 * ((tile + 1) % kScaleSlots), ((tile + 1) / kScaleSlots) & 1));
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            const float2 x = two_fma(make_float2(v[16 * (c & 1) + i], v[16 * (c & 1) + i + 1]), k, r);
                            const float2 e = make_float2(exp2_of(x.x), exp2_of(x.y));
                            sum = two_add(sum, e);
                            w[8 * c + i / 2] = f16x2_of(e.x, e.y);
                        }
                        weight = fmaf(sum.x + sum.y, back[c], weight);
                    }
                    tensor_store32(scores + 64 * half, w);  // (over the scores that have been read)
                    const bool early = __all_sync(0xffffffffu, there);
                    if (early) {  // the next scores, while the weights are on their way
                        tensor_fence_after();
                        tensor_load(scores + 64 * (half ^ 1), s[0]);
                        tensor_load(scores + 64 * (half ^ 1) + 32, s[1]);
                    }
                    tensor_wait_stores();
                    tensor_fence_before();
                    __syncwarp();
                    if (lane == 0) barrier_arrive(weights_bar + 8 * half);
                    if (more && !early) {
                        ok = ok && (half == 0 || warp_waits(scales_full + 8 * ((tile + 1) % kScaleSlots), ((tile + 1) / kScaleSlots) & 1, bounds)) &&
                             warp_waits(scores_bar + 8 * (half ^ 1), (phase + half) & 1, bounds);
                        tensor_fence_after();
                        tensor_load(scores + 64 * (half ^ 1), s[0]);
                        tensor_load(scores + 64 * (half ^ 1) + 32, s[1]);
                    }
                }
            }
            if (count > 0) {  // the last phases: the products with the last weights
                ok = ok && warp_waits(scores_bar, phase & 1, bounds) && warp_waits(scores_bar + 8, phase & 1, bounds);
                ++phase;
                tensor_fence_after();
            }
            const bool whole = walk.first() && walk.last();
            const int rows = it.rows - which * 128 - (warp & 3) * 32;  // of the warp, those that there are
            if (!ok || over) weight = top = __uint_as_float(0x7fffffffu);
            top -= kShift;  // what the weights are relative to
            if (!finite && to > from) weight = __uint_as_float(0x7fffffffu);  // (where the row sees something)
            if (!whole && walk.first() && threadIdx.x == 0) *head = {walk.parts(plan), it.q.row, it.q0, it.rows, it.head};
            float* part = p.workspace + (2 * int64_t(blockIdx.x) + (walk.first() ? 1 : 0)) * part_floats<kRows>();
            const float one = whole ? (weight == 0.0f ? 0.0f : 1.0f / weight) : 1.0f;
            // The rows' results go through the place of their queries, from where 16 lanes store 256 bytes of a row: all of it in bf16, or, of a part,
            // 64 columns of fp32 at a time.
            const uint32_t stage = base + kQueryAt + which * 2 * kBytes + (warp & 3) * 32 * 256;
#pragma unroll 1
            for (int turn = 0; turn < (whole || p.cache.dim <= 64 ? 1 : 2); ++turn) {
                __syncwarp();
#pragma unroll 1
                for (int c = 0; c < (whole ? (p.cache.dim + 31) / 32 : 2); ++c) {
                    float v[32];
                    if (count > 0) {
                        tensor_load(sums + 64 * turn + 32 * c, v);
                        tensor_wait(v);
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = 0.0f;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {  // 16 bytes a store, in places turned by the row
                        if (whole) {
                            const uint32_t at = stage + lane * 256 + (((4 * c + i) ^ (lane & 15)) << 4);
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(bf16x2_of(v[8 * i] * one, v[8 * i + 1] * one)),
                                         "r"(bf16x2_of(v[8 * i + 2] * one, v[8 * i + 3] * one)), "r"(bf16x2_of(v[8 * i + 4] * one, v[8 * i + 5] * one)),
                                         "r"(bf16x2_of(v[8 * i + 6] * one, v[8 * i + 7] * one))
                                         : "memory");
                        } else {
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                const uint32_t at = stage + lane * 256 + (((8 * c + 2 * i + j) ^ (lane & 15)) << 4);
                                asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(v[8 * i + 4 * j]), "f"(v[8 * i + 4 * j + 1]),
                                             "f"(v[8 * i + 4 * j + 2]), "f"(v[8 * i + 4 * j + 3])
                                             : "memory");
                            }
                        }
                    }
                }
                __syncwarp();
#pragma unroll 4
                for (int i = 0; i < 16; ++i) {
                    const int r = 2 * i + (lane >> 4);
                    const int64_t at = __shfl_sync(0xffffffffu, place.row * p.out_row + place.head * p.out_head, r);
                    uint4 w;
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w)
                                 : "r"(stage + r * 256 + (((lane & 15) ^ (r & 15)) << 4)));
                    if (r >= rows) continue;
                    if (!whole) *reinterpret_cast<uint4*>(part + (which * 128 + (warp & 3) * 32 + r) * 128 + 64 * turn + 4 * (lane & 15)) = w;
                    else if (8 * (lane & 15) < p.cache.dim) *reinterpret_cast<uint4*>(p.out + at + 8 * (lane & 15)) = w;
                }
            }
            if (lane < rows) {
                if (!whole) part[kRows * 128 + which * 128 + row] = top, part[kRows * 129 + which * 128 + row] = weight;
                else if (p.lse) p.lse[int64_t(place.row) * p.heads + place.head] = row_lse(top, weight);
            }
            asm volatile("bar.sync %0, 128;" ::"r"(1 + which) : "memory");  // (the next item's queries come to the same place)
            tensor_fence_before();  // (the sums are read before the next item's queries are there)
        }
    } else if (warp < 12) {
        fewer_registers<kFew>();
        const int token = (warp & 3) * 32 + lane;
        const int chunks = (p.cache.dim + 15) / 16;  // of 16 codes
        uint32_t tile = 0;
        bool ok = true;
        for (; walk.there() && ok; walk.next())
            for (int t = 0; t < walk.count(); ++t, ++tile) {
                const uint32_t from = tile % kCodes, to = tile % kValues;
                ok = warp_waits(codes_full + 8 * from, (tile / kCodes) & 1, bounds) && warp_waits(values_empty + 8 * to, ((tile / kValues) & 1) ^ 1, bounds);
                if (!ok) break;
                // What no row sees may be anything, NaN too, which a weight of zero would not take out.
                const int position = (walk.begin() + t) * kTile + token;
                const bool seen = position >= walk.it.lo && position < walk.it.hi;
                const uint32_t codes = base + kCodeAt + from * kBytes + token * 128, values = base + kValueAt + to * 2 * kBytes + token * 128;
#pragma unroll 2
                for (int j = 0; j < chunks; ++j) {
                    uint32_t w[4], v[8];
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                                 : "r"(codes + ((j ^ (token & 7)) << 4)));
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(v[2 * i]) : "h"(static_cast<uint16_t>(w[i])));
                        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(v[2 * i + 1]) : "h"(static_cast<uint16_t>(w[i] >> 16)));
                    }
                    if (!seen) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = 0u;
                    }
                    const uint32_t at = values + (j >> 2) * kBytes;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + (((2 * (j & 3) + i) ^ (token & 7)) << 4)), "r"(v[4 * i]), "r"(v[4 * i + 1]),
                                     "r"(v[4 * i + 2]), "r"(v[4 * i + 3])
                                     : "memory");
                }
                async_fence();
                __syncwarp();
                if (lane == 0) {
                    barrier_arrive(codes_empty + 8 * from);
                    barrier_arrive(values_full + 8 * to);
                }
            }
    } else {
        fewer_registers<kFew>();
        if (warp == 12) {
            const int pages = kTile >> p.cache.page_shift, page_bytes = 128 << p.cache.page_shift;  // of a tile
            uint32_t tile = 0, loaded[2] = {0, 0};
            bool ok = true;
            for (; walk.there() && ok; walk.next()) {
                if (walk.count() == 0) continue;
                Pages list(p, walk.it, walk.begin() * pages);
                int within = 0;
                for (int t = 0; t < walk.count() && ok; ++t, ++tile) {
                    if (within == 32) list.next(), within = 0;
                    const uint32_t slot = tile % kScaleSlots;
                    const int page = __shfl_sync(0xffffffffu, list.id, within + (lane & (pages - 1)));
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t stages = half ? kCodes : kKeys, at = tile % stages, parity = ((tile / stages) & 1) ^ 1;
                        const uint32_t bar = (half ? codes_full : keys_full) + 8 * at;
                        ok = !(withheld.copies && tile >= kKeys + kWithheldFrom) &&
                             (tile < stages || warp_waits((half ? codes_empty : keys_empty) + 8 * at, parity, bounds));
                        if (!ok) break;
                        if (lane == 0) barrier_expect(bar, kBytes);
                        __syncwarp();
                        if (lane < pages) load_page(base + (half ? kCodeAt : kKeyAt) + at * kBytes + lane * page_bytes, half ? &maps.v : &maps.k, walk.it.head, page, bar);
                        __syncwarp();
                        ++loaded[half];
                    }
                    if (withheld.scales) __nanosleep(kLate);
                    if (t == 0) list.first_scales();
                    const uint32_t word = __shfl_sync(0xffffffffu, list.scales, within + ((lane & 7) * pages >> 3));
                    within += pages;
                    if (!ok) break;
                    if (lane < 8) {
                        page_scales[slot][0][lane] = __uint_as_float((word & 0xffu) << 23);
                        page_scales[slot][1][lane] = static_cast<float>(static_cast<int>(word >> 8) - 127);
                        page_scales[slot][2][lane] = __uint_as_float((254u - (word >> 8)) << 23);
                    }
                    __syncwarp();
                    if (lane == 0) barrier_arrive(scales_full + 8 * slot);
                }
            }
            if (lane == 0) issued[0] = loaded[0], issued[1] = loaded[1];
        } else if (warp < 15 && elected()) {  // a tile of rows each: neither waits for what the other waits for
            const int which = warp - 13;
            constexpr uint32_t to_scores = product_codes(128, 64, false, false);
            const uint32_t to_sums = product_codes(128, p.cache.dim, false, true);  // (fp16 has the code of e4m3)
            const uint64_t queries0 = operand(base + kQueryAt + which * 2 * kBytes), keys0 = operand(base + kKeyAt), values0 = operand(base + kValueAt, kBytes);
            const uint32_t scores0 = tensor + which * 128, sums = tensor + 256 + which * 128, scores_bar = scores_full + 16 * which,
                           weights_bar = weights_full + 16 * which;
            const int steps = (p.cache.dim + 31) / 32;
            uint32_t tile = 0, weighted = 0, items = 0;
            bool ok = true;
            const auto score = [&](int half, uint32_t t) {
                const uint64_t k = keys0 + (t % kKeys) * (kBytes >> 4) + half * (kBytes >> 5);
                const uint32_t d = scores0 + half * 64;
                for (int i = 0; i < steps; ++i) {
                    multiply_codes(d, queries0 + 2 * i, k + 2 * i, to_scores, i > 0);
                    multiply_codes(d, queries0 + (kBytes >> 4) + 2 * i, k + 2 * i, to_scores, true);
                }
            };
            const auto add = [&](int half, uint32_t t, bool first) {
                const uint64_t v = values0 + (t % kValues) * (2 * kBytes >> 4) + half * (kBytes >> 5);
#pragma unroll
                for (int i = 0; i < 4; ++i) multiply_f16(sums, scores0 + half * 64 + 8 * i, v + 128 * i, to_sums, !first || i > 0);
            };
            const auto keys_there = [&](uint32_t t) { return barrier_over(keys_full + 8 * (t % kKeys), (t / kKeys) & 1); };
            const auto keys_wait = [&](uint32_t t) { return thread_waits(keys_full + 8 * (t % kKeys), (t / kKeys) & 1, bounds); };
            const auto values_there = [&](uint32_t t) { return barrier_over(values_full + 8 * (t % kValues), (t / kValues) & 1); };
            const auto values_wait = [&](uint32_t t) { return thread_waits(values_full + 8 * (t % kValues), (t / kValues) & 1, bounds); };
            for (; walk.there() && ok; walk.next()) {
                const int count = walk.count();
                if (walk.it.rows <= 128 * which) {  // no rows here: the other's tiles pass
                    for (int t = 0; t < count && ok; ++t, ++tile) {
                        ok = keys_wait(tile) && values_wait(tile);
                        if (!ok) break;
                        barrier_arrive(keys_empty + 8 * (tile % kKeys));
                        barrier_arrive(values_empty + 8 * (tile % kValues));
                    }
                    continue;
                }
                if (count == 0) continue;
                ok = thread_waits(queries_full + 8 * which, items++ & 1, bounds) && keys_wait(tile);
                if (!ok) break;
                tensor_fence_after();
                for (int half = 0; half < 2; ++half) {
                    score(half, tile);
                    products_done<false>(scores_bar + 8 * half);
                }
                products_done<false>(keys_empty + 8 * (tile % kKeys));
                // (what the next step waits for is asked before this one's products: an answer takes 150 to 200 cycles, also where it is yes)
                bool values = false, keys = false, weights = false;
                for (int t = 0; t < count; ++t, ++tile, ++weighted) {
                    const bool more = t + 1 < count;
                    ok = (values || values_wait(tile)) && (!more || keys || keys_wait(tile + 1));
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        ok = ok && (weights || thread_waits(weights_bar + 8 * half, weighted & 1, bounds));
                        if (!ok) break;
                        tensor_fence_after();
                        add(half, tile, t == 0 && half == 0);
                        weights = (half == 0 || more) && barrier_over(weights_bar + 8 * (half ^ 1), (weighted + half) & 1);
                        if (half == 1) {
                            values = more && values_there(tile + 1);
                            keys = t + 2 < count && keys_there(tile + 2);
                        }
                        if (more) score(half, tile + 1);  // (over these weights, behind the products with them)
                        products_done<false>(scores_bar + 8 * half);
                    }
                    if (!ok) break;
                    products_done<false>(values_empty + 8 * (tile % kValues));
                    if (more) products_done<false>(keys_empty + 8 * ((tile + 1) % kKeys));
                }
            }
            if (!ok) {
                products_done<false>(drained + 8 * which);
                for (int polls = 0; polls < kLandings && !barrier_passed(drained + 8 * which, 0); ++polls) {}
            }
        }
    }
    __syncwarp();
    tensor_fence_before();
    __syncthreads();
    if (__builtin_expect(over, 0) && warp == 12) {  // copies in flight have to land before the block ends
        land<kKeys>(keys_full, issued[0]);
        land<kCodes>(codes_full, issued[1]);
    }
    if (warp == 13) {
        tensor_fence_after();
        tensor_free<false>(tensor, 512);
    }
}

}  // namespace

int attention_many(const AttentionArgs& a, int blocks, cudaStream_t s) {
    CacheMaps maps;
    int st = cache_maps(a.cache, &maps);
    if (st == PVQ_OK) st = allow_shared(reinterpret_cast<const void*>(attention_many_kernel), kShared);
    int registers = 0;
    if (st == PVQ_OK) st = registers_of(reinterpret_cast<const void*>(attention_many_kernel), &registers);
    if (st != PVQ_OK) return st;
    if (registers < kRegisters) return PVQ_ERR_UNSUPPORTED;  // (a build that gives it fewer: the warps' shares would be waited for without end)
    return launch_early(attention_many_kernel, dim3(static_cast<unsigned>(blocks)), kThreads, kShared, 0, s, maps, a);
}

}  // namespace fp8
}  // namespace pvq
