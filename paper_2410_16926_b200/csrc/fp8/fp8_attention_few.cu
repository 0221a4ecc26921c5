// Attention of few query rows over the 8-bit cache: bound by reading the cache.
//
// For each tile of 128 tokens the tokens are the products' 128 lanes and the query rows their columns: S^T = K Q^T, then, with
// a thread a token, the weights w = 2^(s - m) and P^T, and O^T = V^T P^T with the dims as lanes, added to sums in registers.  Both
// products take the cache's codes as they lie in memory, the keys along k and the values across it.  What they are multiplied
// by is split into two codes each (queries to 2^-17 of the row's largest).
//
// A page's scales are powers of two: that of the keys multiplies a token's scores, that of the values is added to their exponents, so that
// what is weighed is w * scale; the weights' sum takes the scale out again.
//
// The weights' codes are relative to the tile's own largest (to a power of two of the row's largest so far, so that a tile's sums join the row's
// by an exact factor): a token that leads by far costs the other tiles nothing, and what many small weights hold together stays.  The
// second codes, of what the first ones leave, are 2^5 times as large, in columns of their own behind the first ones': one product of twice the columns.
// Within a tile a weight is off by 2^-8 of itself or 2^-22 of the tile's largest.
//
// Warps: one issues the copies, one the products, four hold the tokens (then the dims).
//
// What bounds it: memory, up to 16 rows.  A tile of 32 KB in each of 296 blocks takes 1.46 to 1.53 us (1.48 at the copy rate); with 32 rows 2.4, the
// tokens' warps.  That takes the 4, 8 or 16 columns that there are rows for: computing on all 16 for 4 rows cost 1.7 us a tile of latency, and short
// calls 2.5 us.  Before the first copy pass 3.5 us (lengths, a scan of the sequences' work, the table), 1.2 less without the scan.
#include "fp8_attention.cuh"

namespace pvq {
namespace fp8 {
namespace {

constexpr int kThreads = 192;
constexpr int kHalf = kTile * 128;       // bytes of a tile's keys or values, rows of 128 bytes
constexpr float kShift = 8.0f;           // weights are up to 2^8: the first codes are off by 8 at most
constexpr float kApart = 32.0f;          // ... and the second ones up to 2^8, too

// ROWS query rows of an item: a product has 16 or 32 columns, of which 4, 8 or all are used.
template <int ROWS>
struct Few {
    static constexpr int kWide = ROWS <= 16 ? 16 : 32;  // columns of a product
    static constexpr int kHalves = kWide == 16 ? 6 : 5;
    static constexpr int kQueries = kHalves * kHalf, kQueryBytes = kWide * 128;  // two codes each
    static constexpr int kWeights = kQueries + 2 * kQueryBytes, kWeightBytes = kWide * kTile;
    static constexpr int kBars = kWeights + 2 * kWeightBytes;
    static constexpr size_t kShared = 1024 + kBars + 256;
    static constexpr int kColumns = kWide == 16 ? 64 : 128;  // of tensor memory: scores twice, sums of first and of second codes
    static_assert(kWeightBytes == kWide / 16 * kTile * 16, "the second codes are the next columns");
    static_assert(2 * (kShared + 1024 + 1200 + 200 * ROWS) <= 233472, "two blocks an SM, with the system's kilobyte each and what else they share");
};

// Operand across k whose 16 columns of one k lie together: eight k's are 128 bytes, the next 16 columns are `further`.
__device__ __forceinline__ uint64_t operand_plain(uint32_t at, uint32_t further) {
    return static_cast<uint64_t>((at & 0x3ffffu) >> 4) | static_cast<uint64_t>(128u >> 4) << 16 | static_cast<uint64_t>(further >> 4) << 32 | uint64_t(1) << 46;
}

__device__ __forceinline__ float warp_max(float x) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ void tokens_meet() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

// A lane's values of 4, 8, 16 or 32 columns.
template <int N>
__device__ __forceinline__ void load_columns(uint32_t at, float (&v)[N]) {
    if constexpr (N == 4) {
        uint32_t r[4];
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
    } else if constexpr (N == 8) {
        uint32_t r[8];
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                     : "r"(at));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
    } else {
        tensor_load(at, v);
    }
}

// CLUSTER: an item for each cluster (of a.split blocks; one block alone is one too) instead of a share of all items' work for each block.
template <int ROWS, bool CLUSTER>
__global__ void __launch_bounds__(kThreads, 2) attention_few_kernel(const __grid_constant__ CacheMaps maps, const __grid_constant__ AttentionArgs p) {
    using S = Few<ROWS>;
    constexpr int kHalves = S::kHalves, kWide = S::kWide;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (shared_address(raw) + 1023u) & ~1023u;
    const uint32_t full = base + S::kBars, empty = full + 8 * kHalves, scales_full = empty + 8 * kHalves, scores_full = scales_full + 8 * kScaleSlots,
                   weights_full = scores_full + 16, sums_full = weights_full + 8, queries_full = sums_full + 8, drained = queries_full + 8;
    __shared__ uint32_t tensor_base, issued_halves;
    __shared__ int over;
    __shared__ PlanShared plan;
    __shared__ float page_scales[kScaleSlots][3][8];  // of 16 tokens each: keys', values' exponent, 1 / values'
    __shared__ __align__(16) float factor[ROWS], highs[2][4][ROWS];  // rows' factors; their largest scores, of each warp
    __shared__ float4 tops[2][4][ROWS];         // of each warp: what a tile's weights are relative to, what joins them to the row's, what the row's lose
    __shared__ float ends[4][ROWS], ones[ROWS];  // the weights' sums, and 1 over them
    __shared__ int64_t places[ROWS];      // of their results
    __shared__ int from[ROWS], to[ROWS];  // positions that a row sees
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp == 0) {  // a barrier a lane
        constexpr int kAll = 2 * kHalves + kScaleSlots + 6;
        static_assert(kAll <= 32, "one lane each");
        const int i = lane - (2 * kHalves + kScaleSlots);  // scores twice, weights, sums, queries, drained
        if (lane < kAll) barrier_init(full + 8 * lane, i == 2 || i == 4 ? 4 : 1);
        barrier_init_fence();
        if (lane == 0) {
            over = 0;
            issued_halves = 0;
            prefetch_map(&maps.k), prefetch_map(&maps.v);
        }
    } else if (warp == 1) {
        tensor_alloc<false>(shared_address(&tensor_base), S::kColumns);
    }
    tensor_fence_before();
    __syncthreads();
    tensor_fence_after();
    launch_dependents();
    dependency_wait();
    const uint32_t tensor = tensor_base, sums = tensor + 2 * kWide;
    Bounds bounds{&over, p.status};
    const Withheld withheld = withheld_in(bounds);
    const int rank = CLUSTER && p.split > 1 ? static_cast<int>(cluster_rank()) : 0;
    Walk<ROWS> walk = [&] {
        if constexpr (CLUSTER) return Walk<ROWS>(p, blockIdx.x / p.split, rank, p.split);
        else return Walk<ROWS>(p, find_share<kThreads, ROWS>(p, plan, 128), plan);
    }();
    if (CLUSTER && p.status && threadIdx.x == 0 && rank == 0) {
        const Sequence& q = walk.it.q;
        if (q.first < 0 || q.held < q.first + q.n) atomicOr(p.status, PVQ_STATUS_BAD_PAGE);
    }

    if (warp == 0) {
        const int pages = kTile >> p.cache.page_shift, page_bytes = 128 << p.cache.page_shift;  // of a tile
        Turn<kHalves> turn;
        uint32_t issued = 0, tile = 0;
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
                    ok = !(withheld.copies && issued >= kHalves + kWithheldFrom) &&
                         (issued < kHalves || warp_wait(empty + 8 * turn.at, turn.parity ^ 1, bounds));
                    if (!ok) break;
                    const uint32_t bar = full + 8 * turn.at;
                    if (lane == 0) barrier_expect(bar, kHalf);
                    __syncwarp();
                    if (lane < pages) load_page(base + turn.at * kHalf + lane * page_bytes, half ? &maps.v : &maps.k, walk.it.head, page, bar);
                    __syncwarp();
                    turn.next();
                    ++issued;
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
        if (lane == 0) issued_halves = issued;
    } else if (warp == 1) {
        if (elected()) {
            constexpr uint32_t scores = product_codes(128, kWide, false, false), results = product_codes(128, 2 * kWide, true, true);
            const uint64_t tiles0 = operand(base), queries0 = operand(base + S::kQueries), weights0 = operand_plain(base + S::kWeights, kTile * 16);
            const int steps = (p.cache.dim + 31) / 32;
            uint32_t tile = 0, items = 0;
            bool ok = true;
            const auto half_at = [&](uint32_t h) { return tiles0 + (h % kHalves) * (kHalf >> 4); };
            const auto arrived = [&](uint32_t h) { return barrier_wait(full + 8 * (h % kHalves), (h / kHalves) & 1, bounds); };
            const auto score = [&](uint32_t t) {
                ok = arrived(2 * t);
                if (!ok) return;
                tensor_fence_after();
                const uint64_t k = half_at(2 * t);
                const uint32_t d = tensor + (t & 1) * kWide;
                for (int i = 0; i < steps; ++i) {
                    multiply_codes(d, k + 2 * i, queries0 + 2 * i, scores, i > 0);
                    multiply_codes(d, k + 2 * i, queries0 + (S::kQueryBytes >> 4) + 2 * i, scores, true);
                }
                products_done<false>(empty + 8 * (2 * t % kHalves));
                products_done<false>(scores_full + 8 * (t & 1));
            };
            for (; walk.there() && ok; walk.next()) {
                const int count = walk.count();
                if (count == 0) continue;
                ok = barrier_wait(queries_full, items++ & 1, bounds);
                if (!ok) break;
                tensor_fence_after();
                score(tile);
                for (int t = 0; t < count && ok; ++t, ++tile) {
                    if (t + 1 < count) score(tile + 1);
                    ok = ok && barrier_wait(weights_full, tile & 1, bounds) && arrived(2 * tile + 1);
                    if (!ok) break;
                    tensor_fence_after();
                    const uint64_t v = half_at(2 * tile + 1);
#pragma unroll
                    for (int i = 0; i < 4; ++i) multiply_codes(sums, v + 256 * i, weights0 + 32 * i, results, i > 0);
                    products_done<false>(empty + 8 * ((2 * tile + 1) % kHalves));
                    products_done<false>(sums_full);
                }
            }
            if (!ok) {
                products_done<false>(drained);
                for (int polls = 0; polls < kLandings && !barrier_passed(drained, 0); ++polls) {}
            }
        }
    } else {
        const int quarter = warp & 3, thread = quarter * 32 + lane;  // token, then dim
        const uint32_t mine = quarter << 21;
        PartHead* head = part_heads<ROWS>(p) + blockIdx.x;
        if (!CLUSTER && thread == 0) head->parts = 0;
        if (ROWS < S::kWide) {  // columns that are not used: zeros
            for (int i = thread; i < (2 * S::kQueryBytes + 2 * S::kWeightBytes) / 16; i += 128)
                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(base + S::kQueries + 16 * i), "r"(0u) : "memory");
            tokens_meet();
        }
        uint32_t tile = 0;
        bool ok = true;
        for (; walk.there(); walk.next()) {
            const Item& it = walk.it;
            const int count = walk.count();
            {  // queries, 8 threads a row (4 of 32 rows); rows that are not used were zeros from the start
                constexpr int kAcross = ROWS <= 16 ? 8 : 4, kEach = 128 / kAcross;  // dims of a thread
                const int r = thread / kAcross, col = thread % kAcross * kEach;
                if (r < ROWS) {  // (whole warps)
                    float x[kEach];
                    uint32_t most = 0u;
                    const RowPlace place = place_of(p, it.q, it.head, it.q0 + min(r, it.rows - 1));
                    const __nv_bfloat16* q = p.q + place.row * p.q_row + place.head * p.q_head + col;
#pragma unroll
                    for (int j = 0; j < kEach / 8; ++j) {
                        uint4 w = make_uint4(0u, 0u, 0u, 0u);
                        if (col + 8 * j < p.cache.dim) w = __ldg(reinterpret_cast<const uint4*>(q + 8 * j));
                        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[8 * j + 2 * i] = __uint_as_float(u[i] << 16), x[8 * j + 2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
                    }
#pragma unroll
                    for (int j = 0; j < kEach; ++j) most = max(most, __float_as_uint(x[j]) & 0x7fffffffu);
#pragma unroll
                    for (int o = 1; o < kAcross; o <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
                    const uint32_t byte = most < kFiniteEnd ? scale_byte(most) : 127u;
                    const float inverse = inverse_of(byte);
                    const uint32_t at = base + S::kQueries + r * 128;
#pragma unroll
                    for (int j = 0; j < kEach / 16; ++j) {
                        uint32_t hi[4], lo[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t h0, l0, h1, l1;
                            const float* y = x + 16 * j + 4 * i;
                            two_codes(y[0] * inverse, y[1] * inverse, h0, l0);
                            two_codes(y[2] * inverse, y[3] * inverse, h1, l1);
                            hi[i] = h0 | h1 << 16, lo[i] = l0 | l1 << 16;
                        }
                        const uint32_t chunk = at + (((col / 16 + j) ^ (r & 7)) << 4);
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(chunk), "r"(hi[0]), "r"(hi[1]), "r"(hi[2]), "r"(hi[3]) : "memory");
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(chunk + S::kQueryBytes), "r"(lo[0]), "r"(lo[1]), "r"(lo[2]), "r"(lo[3])
                                     : "memory");
                    }
                    if (thread % kAcross == 0) {
                        const int position = it.q.first + divide(it.q0 + r, p.by_group);
                        factor[r] = most < kFiniteEnd ? row_factor(byte, p.scale) : __uint_as_float(0x7fffffffu);
                        to[r] = r < it.rows ? (p.causal ? min(it.q.held, position + 1) : it.q.held) : 0;
                        from[r] = first_seen(p, position);
                    }
                }
                async_fence();
                __syncwarp();
                if (lane == 0 && count > 0) barrier_arrive(queries_full);  // (without tiles nothing would hold the next item's back)
            }
            tokens_meet();
            // positions that every row sees, and that any does (a later query sees from later on, and farther)
            const int all_from = from[it.rows - 1], all_to = to[0], any_from = from[0], any_to = to[it.rows - 1];
            float weight[ROWS], sum[ROWS];
#pragma unroll
            for (int n = 0; n < ROWS; ++n) weight[n] = 0.0f, sum[n] = 0.0f;
            float top = kNone;  // of row `lane`, over all tiles so far
            const auto add_sums = [&](uint32_t t) {
                ok = ok && warp_wait(sums_full, t & 1, bounds);
                tensor_fence_after();
#pragma unroll
                for (int c = 0; c < ROWS; c += 16) {
                    constexpr int kHere = ROWS < 16 ? ROWS : 16;
                    float v[kHere], w[kHere];
                    load_columns(sums + mine + c, v);
                    load_columns(sums + mine + kWide + c, w);
                    tensor_wait_loads();
#pragma unroll
                    for (int n = 0; n < kHere; ++n) sum[c + n] = fmaf(fmaf(w[n], 1.0f / kApart, v[n]), tops[t & 1][quarter][c + n].y, sum[c + n]);
                }
            };
            for (int t = 0; t < count; ++t, ++tile) {
                const int tile_at = (walk.begin() + t) * kTile, position = tile_at + thread;
                const uint32_t slot = tile % kScaleSlots;
                ok = ok && warp_wait(scales_full + 8 * slot, (tile / kScaleSlots) & 1, bounds) &&
                     warp_wait(scores_full + 8 * (tile & 1), (tile >> 1) & 1, bounds);
                tensor_fence_after();
                float s[ROWS];
                load_columns(tensor + mine + (tile & 1) * kWide, s);
                const float key = page_scales[slot][0][thread >> 4], value = page_scales[slot][1][thread >> 4], out_of = page_scales[slot][2][thread >> 4];
                tensor_wait_loads();
#pragma unroll
                for (int n = 0; n < ROWS; ++n) s[n] = fmaf(s[n] * factor[n], key, value);
                if (tile_at < all_from || tile_at + kTile > all_to) {
#pragma unroll
                    for (int n = 0; n < ROWS; ++n)
                        if (position < from[n] || position >= to[n]) s[n] = kNone;
                }
                float (&high)[4][ROWS] = highs[tile & 1];
                float4 (&relative)[ROWS] = tops[tile & 1][quarter];
#pragma unroll
                for (int n = 0; n < ROWS; n += 4) {
                    const float4 h = make_float4(warp_max(s[n]), warp_max(s[n + 1]), warp_max(s[n + 2]), warp_max(s[n + 3]));
                    if (lane == 0) *reinterpret_cast<float4*>(&high[quarter][n]) = h;
                }
                tokens_meet();
                bool grown = false;
                if (lane < ROWS) {  // a row each: the tile's weights are relative to 2^-below of the row's largest, which is 1 to 2 times the tile's
                    const float h = fmaxf(fmaxf(high[0][lane], high[1][lane]), fmaxf(high[2][lane], high[3][lane])), now = fmaxf(top, h);
                    const int below = __float2int_rd(fminf(now - h, 120.0f));  // (120: nothing seen, or nothing left of it)
                    grown = now > top;
                    relative[lane] = make_float4(now == kNone ? 0.0f : now - static_cast<float>(below) - kShift, __uint_as_float(static_cast<uint32_t>(127 - below) << 23),
                                                 grown ? exp2_of(top - now) : 1.0f, 0.0f);
                    top = now;
                }
                grown = __any_sync(0xffffffffu, grown);
                __syncwarp();
                if (t > 0) add_sums(tile - 1);
                if (grown) {
#pragma unroll
                    for (int n = 0; n < ROWS; ++n) {
                        const float less = relative[n].z;
                        sum[n] *= less, weight[n] *= less;
                    }
                }
                uint32_t hi[ROWS / 4], lo[ROWS / 4];
#pragma unroll
                for (int n = 0; n < ROWS; n += 4) {
                    float w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 r = *reinterpret_cast<const float2*>(&relative[n + i]);
                        w[i] = exp2_of(s[n + i] - r.x);
                        weight[n + i] = fmaf(w[i] * out_of, r.y, weight[n + i]);
                    }
                    uint32_t h0, l0, h1, l1;
                    two_codes(w[0], w[1], h0, l0, kApart);
                    two_codes(w[2], w[3], h1, l1, kApart);
                    hi[n / 4] = h0 | h1 << 16, lo[n / 4] = l0 | l1 << 16;
                }
                const uint32_t place = base + S::kWeights + thread * 16;
                if constexpr (ROWS == 4) {
                    asm volatile("st.shared.b32 [%0], %1;" ::"r"(place), "r"(hi[0]) : "memory");
                    asm volatile("st.shared.b32 [%0], %1;" ::"r"(place + S::kWeightBytes), "r"(lo[0]) : "memory");
                } else if constexpr (ROWS == 8) {
                    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(place), "r"(hi[0]), "r"(hi[1]) : "memory");
                    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(place + S::kWeightBytes), "r"(lo[0]), "r"(lo[1]) : "memory");
                } else {
#pragma unroll
                    for (int n = 0; n < ROWS / 4; n += 4) {
                        const uint32_t at = place + n * 4 * kTile;
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(hi[n]), "r"(hi[n + 1]), "r"(hi[n + 2]), "r"(hi[n + 3]) : "memory");
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + S::kWeightBytes), "r"(lo[n]), "r"(lo[n + 1]), "r"(lo[n + 2]), "r"(lo[n + 3])
                                     : "memory");
                    }
                }
                // What no row sees may be anything, NaN too, which a weight of zero would not take out.
                if (tile_at < any_from || tile_at + kTile > any_to) {
                    const uint32_t h = 2 * tile + 1, row = base + (h % kHalves) * kHalf + thread * 128;
                    ok = ok && warp_wait(full + 8 * (h % kHalves), (h / kHalves) & 1, bounds);
                    if (position < any_from || position >= any_to) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(row + 16 * j), "r"(0u) : "memory");
                    }
                }
                async_fence();
                tensor_fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive(weights_full);
            }
            if (count > 0) add_sums(tile - 1);
            tensor_fence_before();
            // The weights' sums over the warp's tokens, in a fixed order: of halves of the columns by halves of the lanes, until lane n has column n.
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                if (o >= ROWS) {
#pragma unroll
                    for (int n = 0; n < ROWS; ++n) weight[n] += __shfl_xor_sync(0xffffffffu, weight[n], o);
                } else {
#pragma unroll
                    for (int n = 0; n < o; ++n) {
                        const bool upper = (lane & o) != 0;
                        const float keep = upper ? weight[n + o] : weight[n], send = upper ? weight[n] : weight[n + o];
                        weight[n] = keep + __shfl_xor_sync(0xffffffffu, send, o);
                    }
                }
            }
            if (lane < ROWS) ends[quarter][lane] = weight[0];
            tokens_meet();
            if (CLUSTER && p.split > 1) {
                // The parts of the cluster's blocks, in the stages' place, which is free once all are here: those of a share of the dims go to the
                // block that adds them up, in the order of the ranks: [rank][row][dim of the share], then [rank][largest, weights][row].  (Copies of a block whose
                // wait ran out may still come over them: its dims are NaN then, as its part makes the others'.)
                const int split = p.split, share = 128 / split;
                const uint32_t stats = base + ROWS * 512;
                float all = 0.0f, relative = kNone;
                if (thread < ROWS) {
                    all = (ends[0][thread] + ends[1][thread]) + (ends[2][thread] + ends[3][thread]), relative = top - kShift;
                    if (over) all = relative = __uint_as_float(0x7fffffffu);
                }
                cluster_barrier();
#pragma unroll
                for (int n = 0; n < ROWS; ++n)
                    if (n < it.rows) store_in(address_in(base + ((rank * ROWS + n) * share + thread % share) * 4, thread / share), __float_as_uint(sum[n]));
                if (thread < it.rows)
                    for (int r = 0; r < split; ++r) {
                        store_in(address_in(stats + (rank * 2 * ROWS + thread) * 4, r), __float_as_uint(relative));
                        store_in(address_in(stats + (rank * 2 * ROWS + ROWS + thread) * 4, r), __float_as_uint(all));
                    }
                cluster_barrier();
                for (int i = thread; i < it.rows * share; i += 128) {
                    const int n = i / share, d = i - n * share;
                    float m[8], top = over ? __uint_as_float(0x7fffffffu) : kNone;
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        m[r] = kNone;
                        if (r < split) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(m[r]) : "r"(stats + (r * 2 * ROWS + n) * 4));
                        top = m[r] != m[r] ? m[r] : (top != top ? top : fmaxf(top, m[r]));
                    }
                    float v = 0.0f, weights = 0.0f;
#pragma unroll
                    for (int r = 0; r < 8; ++r)
                        if (r < split) {
                            const float less = exp2_of(m[r] - (top == kNone ? 0.0f : top));
                            float x, w;
                            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(base + ((r * ROWS + n) * share + d) * 4));
                            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(w) : "r"(stats + (r * 2 * ROWS + ROWS + n) * 4));
                            v = fmaf(x, less, v), weights = fmaf(w, less, weights);
                        }
                    const RowPlace place = place_of(p, it.q, it.head, it.q0 + n);
                    const int dim = rank * share + d;
                    if (dim < p.cache.dim) p.out[place.row * p.out_row + place.head * p.out_head + dim] = __float2bfloat16(weights == 0.0f ? 0.0f : v / weights);
                    if (p.lse && dim == 0) p.lse[int64_t(place.row) * p.heads + place.head] = row_lse(top, weights);
                }
                continue;
            }
            const bool whole = walk.first() && walk.last();
            float* part = p.workspace + (2 * int64_t(blockIdx.x) + (walk.first() ? 1 : 0)) * part_floats<ROWS>();
            if (thread < it.rows) {
                float all = (ends[0][thread] + ends[1][thread]) + (ends[2][thread] + ends[3][thread]), relative = top - kShift;
                if (over) all = relative = __uint_as_float(0x7fffffffu);
                if (whole) {
                    const RowPlace place = place_of(p, it.q, it.head, it.q0 + thread);
                    places[thread] = place.row * p.out_row + place.head * p.out_head;
                    ones[thread] = all == 0.0f ? 0.0f : 1.0f / all;
                    if (p.lse) p.lse[int64_t(place.row) * p.heads + place.head] = row_lse(relative, all);
                } else {
                    part[ROWS * 128 + thread] = relative, part[ROWS * 129 + thread] = all;
                }
            }
            if (!whole && walk.first() && thread == 0) *head = {walk.parts(plan), it.q.row, it.q0, it.rows, it.head};
            if (whole) {
                tokens_meet();
                if (thread < p.cache.dim) {
#pragma unroll
                    for (int n = 0; n < ROWS; ++n)
                        if (n < it.rows) p.out[places[n] + thread] = __float2bfloat16(sum[n] * ones[n]);
                }
            } else {
#pragma unroll
                for (int n = 0; n < ROWS; ++n)
                    if (n < it.rows) part[n * 128 + thread] = sum[n];
            }
            tokens_meet();  // (what the block knows of this item is read)
        }
    }
    __syncwarp();
    if (CLUSTER && p.split > 1 && warp < 2) {  // (the others have met twice)
        cluster_barrier();
        cluster_barrier();
    }
    tensor_fence_before();
    __syncthreads();
    if (__builtin_expect(over, 0) && warp == 0) land<kHalves>(full, issued_halves);  // copies in flight have to land before the block ends
    if (warp == 1) {
        tensor_fence_after();
        tensor_free<false>(tensor, S::kColumns);
    }
}

template <int ROWS, bool CLUSTER>
int launch(const AttentionArgs& a, int blocks, cudaStream_t s) {
    CacheMaps maps;
    int st = cache_maps(a.cache, &maps);
    void (*const kernel)(CacheMaps, AttentionArgs) = attention_few_kernel<ROWS, CLUSTER>;
    if (st == PVQ_OK) st = allow_shared(reinterpret_cast<const void*>(kernel), Few<ROWS>::kShared);
    if (st != PVQ_OK) return st;
    return launch_early(kernel, dim3(static_cast<unsigned>(blocks)), kThreads, Few<ROWS>::kShared, CLUSTER && a.split > 1 ? a.split : 0, s, maps, a);
}
}  // namespace

int attention_few(const AttentionArgs& a, int rows, int blocks, cudaStream_t s) {
    if (rows == 4) return a.split ? launch<4, true>(a, blocks, s) : launch<4, false>(a, blocks, s);
    if (rows == 8) return a.split ? launch<8, true>(a, blocks, s) : launch<8, false>(a, blocks, s);
    if (rows == 16) return a.split ? launch<16, true>(a, blocks, s) : launch<16, false>(a, blocks, s);
    return launch<32, false>(a, blocks, s);
}

}  // namespace fp8
}  // namespace pvq
