// The 8-bit product of few rows, or of little work: out[i][j] = sum_k a(i,k) b(j,k), bound by reading b.
//
// The operands change places: 128 columns of the result (rows of b, the weight) are the product's 128 lanes, ROWS rows of a
// (16 to 128) its columns, so that a token costs 1/16 of a tile's width and not 1/128 of its height.  k is split over the
// blocks of a cluster where there are few tiles: each sums its part in tensor memory and puts it into the shared memory of the
// blocks that its columns fall to, each of which adds the parts of its share of the columns in the order of the ranks (no
// atomics: the same bits every time).
//
// Warps: one issues the copies, one the products, one allocates tensor memory, four bring the scales there (four blocks along k
// at a time, in four sets of columns) and then read the result.
//
// What bounds it: memory, behind a start and an end.  One row, 4096 to 14336: 13.3 us, of which the weight's 58.7 MB take 9.1 at
// the copy rate, which it runs at once the first tiles are there (after 2 to 4 us); the parts are added and stored in the last 1.5.
// 33 rows, 14336 to 4096: 14.9 to 15.3 us (a microsecond more when each block read the others' shared memory, which needs a second
// meeting of the cluster), 64 rows 4096 to 14336 14.7, 128 rows 17.7; with the transposed weight 15.7, 16.1 and 18.4.
#include <atomic>

#include "fp8_matmul.cuh"

namespace pvq {
namespace fp8 {
namespace {

constexpr int kThreads = 256;
// fp32 results: what a block sums in tensor memory, whose sums are cut off and not rounded, is at most about 64 blocks along k, as in
// matmul_many_kernel.  Where a part of a cluster of eight has more, it goes where it is added in runs of so many sets of scales, of
// four blocks each.  (200000 values: 2.2e-6 of the result off in eight parts alone, 4.9e-7 so; 128 rows,
// 128256 to 4096, 175 us and 185.)
constexpr int kRunSets = 16;

template <int ROWS, int SPLIT>
struct Shape {
    static constexpr int kStageBytes = (128 + ROWS) * kBlock;
    // two blocks an SM up to 32 rows, then one
    static constexpr int kStages = ROWS == 16 || (ROWS == 32 && SPLIT == 1) ? 5 : (ROWS == 32 ? 4 : (ROWS == 64 ? 8 : (SPLIT == 1 ? 6 : 5)));
    // The parts of a block's share of the columns: in the stages' place where they are the block's own, otherwise in one of
    // their own, since the others' arrive while it still loads.
    static constexpr int kPartsAt = SPLIT == 1 ? 0 : kStages * kStageBytes, kPartsBytes = ROWS * 512;
    static constexpr int kBarsAt = kStages * kStageBytes + (SPLIT == 1 ? 0 : kPartsBytes);
    static constexpr int kWordsB = ROWS <= 32 ? 1 : ROWS / 32;             // of scales, a lane
    static constexpr int kScales = ROWS < 32 ? 32 : ROWS;                  // columns before them
    static constexpr int kScaleSets = 4;
    static constexpr int kColumns = ROWS == 128 ? 256 : (ROWS == 64 ? 128 : 64);  // of tensor memory, a power of two
    static constexpr size_t kShared = 1024 + kBarsAt + 256;
    static_assert(kStages * kStageBytes >= kPartsBytes, "the result takes the stages' place");
    static_assert(kScales + 8 * kScaleSets <= kColumns, "tensor memory");
    static_assert(kShared <= 232448 - 64, "shared memory");
};

struct Maps {
    CUtensorMap a, b;
};

// Adds the parts of this block's share of the columns, 128 / SPLIT, in the order of the ranks, and stores them: four columns a
// thread, eight reads at a time.  parts: [rank][row][column of the share].
template <int ROWS, int SPLIT, class T>
__device__ __forceinline__ void add_parts(uint32_t parts, int rank, const MatmulArgs& p, int64_t row0, int64_t col0) {
    constexpr int kShare = 128 / SPLIT, kAcross = kShare / 4, kStep = kThreads / kAcross, kAtOnce = 8 / SPLIT;
    const int within = threadIdx.x % kAcross * 4;
    const int64_t col = col0 + rank * kShare + within, left = p.outs - col;
    const int rows = static_cast<int>(min(int64_t(ROWS), p.rows - row0));
    if (left <= 0) return;
    T* out = static_cast<T*>(p.out) + row0 * p.ld + col;
    for (int r0 = threadIdx.x / kAcross; r0 < rows; r0 += kStep * kAtOnce) {
        float4 part[kAtOnce][SPLIT];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
            for (int s = 0; s < SPLIT; ++s)
                if (r0 + i * kStep < rows)
                    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                                 : "=f"(part[i][s].x), "=f"(part[i][s].y), "=f"(part[i][s].z), "=f"(part[i][s].w)
                                 : "r"(parts + ((s * ROWS + r0 + i * kStep) * kShare + within) * 4));
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            if (r0 + i * kStep >= rows) break;
            float4 v = part[i][0];
#pragma unroll
            for (int s = 1; s < SPLIT; ++s) v.x += part[i][s].x, v.y += part[i][s].y, v.z += part[i][s].z, v.w += part[i][s].w;
            T* to = out + (r0 + i * kStep) * p.ld;
            if (left >= 4) {
                if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(to) = make_uint2(bf16x2_of(v.x, v.y), bf16x2_of(v.z, v.w));
                else *reinterpret_cast<float4*>(to) = v;
            } else {
                to[0] = T(v.x);
                if (left > 1) to[1] = T(v.y);
                if (left > 2) to[2] = T(v.z);
            }
        }
    }
}

template <int ROWS, int SPLIT, bool ACROSS, class T>
__global__ void __launch_bounds__(kThreads) matmul_few_kernel(const __grid_constant__ Maps maps, const __grid_constant__ MatmulArgs p) {
    using S = Shape<ROWS, SPLIT>;
    constexpr bool kRuns = SPLIT == 8 && sizeof(T) == 4;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (shared_address(raw) + 1023u) & ~1023u;
    const uint32_t parts = base + S::kPartsAt, full = base + S::kBarsAt, empty = full + 8 * S::kStages, scales_full = empty + 8 * S::kStages,
                   scales_empty = scales_full + 8 * S::kScaleSets, sum_full = scales_empty + 8 * S::kScaleSets, drained = sum_full + 8, sum_empty = drained + 8;
    __shared__ uint32_t tensor_base, issued_stages;
    __shared__ int over;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = blockIdx.x % SPLIT;  // in the cluster
    if (SPLIT > 1) cluster_arrive();      // (every block runs before another writes to its shared memory)
    const int64_t col0 = int64_t(blockIdx.x / SPLIT) * 128, row0 = int64_t(blockIdx.y) * ROWS;
    const int blocks = static_cast<int>((p.inner + kBlock - 1) / kBlock);
    const int first = static_cast<int>(int64_t(blocks) * rank / SPLIT), last = static_cast<int>(int64_t(blocks) * (rank + 1) / SPLIT);  // (SPLIT <= blocks)
    Bounds bounds{&over, p.status};

    const auto load = [&](int kb, uint32_t stage) {
        const uint32_t at = base + stage * S::kStageBytes, bar = full + 8 * stage;
        barrier_expect(bar, S::kStageBytes);
        if (ACROSS) load_tile<false>(at, &maps.b, static_cast<int>(col0), kb * kBlock, bar);
        else load_tile<false>(at, &maps.b, kb * kBlock, static_cast<int>(col0), bar);
        load_tile<false>(at + 128 * kBlock, &maps.a, kb * kBlock, static_cast<int>(row0), bar);
    };
    // the first copies and scales are asked for before the block meets
    uint32_t w[S::kScaleSets][4], x[S::kScaleSets][S::kWordsB];
    const auto scales_of = [&](int f0) {
#pragma unroll
        for (int i = 0; i < S::kScaleSets; ++i) {
            if (f0 + i > (last - 1) / 4) break;
            scale_words<ACROSS>(p.b, col0, f0 + i, w[i]);
            scale_words<false>(p.a, row0, f0 + i, x[i]);  // (row0: a multiple of 128, or 0)
        }
    };
    if (warp == 0) {
        // a barrier a lane: stages' full and empty, the scales' sets full and empty, the sum's full, drained, the sum's empty
        constexpr int kBars = 2 * S::kStages + 2 * S::kScaleSets + (kRuns ? 3 : 2);
        static_assert(kBars <= 32, "one lane each");
        if (lane < kBars) barrier_init(full + 8 * lane, (lane >= 2 * S::kStages && lane < 2 * S::kStages + S::kScaleSets) || (kRuns && lane == kBars - 1) ? 4 : 1);
        barrier_init_fence();
        if (lane == 0) over = 0;
        __syncwarp();
        if (elected()) {
            prefetch_map(&maps.a), prefetch_map(&maps.b);
            dependency_wait();
            for (int i = 0; i < S::kStages && first + i < last; ++i) load(first + i, i);
        }
        __syncwarp();
    } else if (warp == 2) {
        tensor_alloc<false>(shared_address(&tensor_base), S::kColumns);
    }
    if (warp != 2) dependency_wait();
    if (warp >= 4) scales_of(first / 4);
    tensor_fence_before();
    __syncthreads();
    tensor_fence_after();
    launch_dependents();
    if (warp == 2) dependency_wait();
    const uint32_t tensor = tensor_base;
    const Withheld withheld = withheld_of(bounds, rank);

    if (warp == 0) {
        if (elected()) {
            Turn<S::kStages> turn;  // the second time round, and so on
            uint32_t issued = min(S::kStages, last - first);
            for (int kb = first + S::kStages; kb < last; ++kb) {
                if (withheld.copies && issued >= S::kStages + kWithheldFrom) break;
                if (!barrier_wait(empty + 8 * turn.at, turn.parity, bounds)) break;
                load(kb, turn.at);
                turn.next();
                ++issued;
            }
            issued_stages = issued;
        }
    } else if (warp == 1) {
        if (elected()) {
            constexpr uint32_t product = product_e4m3(128, ROWS, ACROSS, false);
            constexpr uint32_t kAlongW = (ACROSS ? 32 * kBlock : 32) >> 4;
            const uint64_t w0 = operand(base, ACROSS ? 128 * kBlock : 16), x0 = operand(base + 128 * kBlock);
            Turn<S::kStages> turn;
            Turn<S::kScaleSets> scales;
            bool ok = true, there = false, starts = true;
            uint32_t run = 0;
            for (int kb = first; kb < last; ++kb) {
                const uint32_t part = kb & 3;
                if (part == 0 || kb == first) ok = barrier_wait(scales_full + 8 * scales.at, scales.parity, bounds);
                ok = ok && (there || barrier_wait(full + 8 * turn.at, turn.parity, bounds));
                if (!ok) break;
                const Turn<S::kStages> now = turn;
                turn.next();
                there = kb + 1 < last && barrier_over(full + 8 * turn.at, turn.parity);
                tensor_fence_after();
                const uint64_t w = w0 + now.at * (S::kStageBytes >> 4), x = x0 + now.at * (S::kStageBytes >> 4);
                const uint32_t sw = tensor + S::kScales + 8 * scales.at, with = with_part(product, part);
#pragma unroll
                for (int k = 0; k < 4; ++k) multiply_e4m3<false>(tensor, w + kAlongW * k, x + 2 * k, with, sw, sw + 4, (kRuns ? !starts : kb > first) || k > 0);
                starts = false;
                products_done<false>(empty + 8 * now.at);
                if (part == 3) {
                    products_done<false>(scales_empty + 8 * scales.at);
                    scales.next();
                }
                if (kRuns && part == 3 && kb + 1 < last && ((kb + 1) / 4 - first / 4) % kRunSets == 0) {
                    products_done<false>(sum_full);
                    ok = barrier_wait(sum_empty, run & 1, bounds);
                    if (!ok) break;
                    ++run;
                    starts = true;
                }
            }
            products_done<false>(ok ? sum_full : drained);
            for (int polls = 0; !ok && polls < kLandings && !barrier_passed(drained, 0); ++polls) {}
        }
    } else if (warp >= 4) {
        const uint32_t mine = tensor + ((warp & 3) << 21);
        constexpr int kShare = 128 / SPLIT;
        const int column = (warp & 3) * 32 + lane;
        // A lane's column of the part goes to the block whose share it is in; kRuns: is added to what is there.
        const auto place = [&]() -> uint32_t {
            const uint32_t at = parts + (rank * ROWS * kShare + column % kShare) * 4;
            return SPLIT > 1 ? address_in(at, column / kShare) : at;
        };
        const auto put_sum = [&](uint32_t to, int rows, bool add) {
            tensor_fence_after();
#pragma unroll
            for (int c = 0; c < ROWS; c += 16) {
                if (c >= rows) break;
                float v[16];
                tensor_load(mine + c, v);
                tensor_wait_loads();
                if (kRuns && add) {
                    float before[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (c + i < rows) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(before[i]) : "r"(to + (c + i) * kShare * 4) : "memory");
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (c + i < rows) v[i] += before[i];
                }
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (c + i < rows) {
                        if (SPLIT > 1) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + (c + i) * kShare * 4), "f"(v[i]) : "memory");
                        else asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + (c + i) * kShare * 4), "f"(v[i]) : "memory");
                    }
            }
        };
        uint32_t run = 0;
        bool met = false;
        Turn<S::kScaleSets> turn;
        bool ok = true;
        // asked for as many steps at once as there are sets of columns: to wait for one before the next is a microsecond each
        for (int f0 = first / 4; f0 <= (last - 1) / 4 && ok; f0 += S::kScaleSets) {
            if (f0 > first / 4) scales_of(f0);
            if (kRuns && f0 > first / 4 && (f0 - first / 4) % kRunSets == 0) {
                ok = warp_wait(sum_full, run & 1, bounds);
                if (!met) cluster_wait();
                met = true;
                if (!ok) break;
                put_sum(place(), static_cast<int>(min(int64_t(ROWS), p.rows - row0)), run > 0);
                ++run;
                tensor_fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive(sum_empty);
            }
#pragma unroll
            for (int i = 0; i < S::kScaleSets; ++i) {
                if (f0 + i > (last - 1) / 4) break;
                if (withheld.scales && f0 + i >= first / 4 + kWithheldFrom) break;
                ok = warp_wait(scales_empty + 8 * turn.at, turn.parity ^ 1, bounds);
                if (!ok) break;
                tensor_fence_after();
                tensor_store(mine + S::kScales + 8 * turn.at, w[i]);
                tensor_store(mine + S::kScales + 8 * turn.at + 4, x[i]);
                tensor_wait_stores();
                tensor_fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive(scales_full + 8 * turn.at);
                turn.next();
            }
        }
        ok = ok && warp_wait(sum_full, kRuns ? run & 1 : 0, bounds);
        if (SPLIT > 1 && !(kRuns && met)) cluster_wait();
        const uint32_t to = place();
        const int rows = static_cast<int>(min(int64_t(ROWS), p.rows - row0));
        if (__builtin_expect(ok, 1)) {
            put_sum(to, rows, kRuns && run > 0);
        } else if (SPLIT > 1) {  // a part that is missing is NaN
#pragma unroll 1
            for (int r = 0; r < rows; ++r) store_in(to + r * kShare * 4, 0x7fffffffu);
        }
        tensor_fence_before();
    }
    __syncwarp();
    if (SPLIT > 1 && warp < 4) cluster_wait();
    if (SPLIT > 1) cluster_barrier();
    else __syncthreads();
    add_parts<ROWS, SPLIT, T>(parts, rank, p, row0, col0);
    if (__builtin_expect(over, 0)) {
        if (SPLIT == 1) {
            __syncthreads();
            if (32 * warp < ROWS) spoil(static_cast<T*>(p.out), p.ld, row0 + 32 * warp, min(p.rows, row0 + ROWS), col0, p.outs, 128);
        }
        if (warp == 0) land<S::kStages>(full, issued_stages);  // copies in flight have to land before the block ends
    }
    if (warp == 2) {
        tensor_fence_after();
        tensor_free<false>(tensor, S::kColumns);
    }
}

template <int ROWS, int SPLIT, bool ACROSS, class T>
int launch(const MatmulArgs& p, cudaStream_t s) {
    Maps maps;
    int st = tile_map(&maps.a, p.a.codes, Element::kByte, p.a.rows, p.a.cols, p.a.ld_codes, kBlock, ROWS);
    if (st == PVQ_OK) st = tile_map(&maps.b, p.b.codes, Element::kByte, p.b.rows, p.b.cols, p.b.ld_codes, kBlock, 128);
    void (*const kernel)(Maps, MatmulArgs) = matmul_few_kernel<ROWS, SPLIT, ACROSS, T>;
    if (st == PVQ_OK) st = allow_shared(reinterpret_cast<const void*>(kernel), Shape<ROWS, SPLIT>::kShared);
    if (st != PVQ_OK) return st;
    const dim3 grid(static_cast<unsigned>((p.outs + 127) / 128 * SPLIT), static_cast<unsigned>((p.rows + ROWS - 1) / ROWS));
    return launch_early(kernel, grid, kThreads, Shape<ROWS, SPLIT>::kShared, SPLIT, s, maps, p);
}

template <int ROWS, int SPLIT>
int launch_split(const MatmulArgs& p, bool transposed, bool bf16, cudaStream_t s) {
    if (transposed) return bf16 ? launch<ROWS, SPLIT, true, __nv_bfloat16>(p, s) : launch<ROWS, SPLIT, true, float>(p, s);
    return bf16 ? launch<ROWS, SPLIT, false, __nv_bfloat16>(p, s) : launch<ROWS, SPLIT, false, float>(p, s);
}
template <int ROWS>
int launch_rows(const MatmulArgs& p, bool transposed, bool bf16, int split, cudaStream_t s) {
    if (split == 1) return launch_split<ROWS, 1>(p, transposed, bf16, s);
    if (split == 2) return launch_split<ROWS, 2>(p, transposed, bf16, s);
    if (split == 4) return launch_split<ROWS, 4>(p, transposed, bf16, s);
    return launch_split<ROWS, 8>(p, transposed, bf16, s);
}

template <int ROWS, int SPLIT>
int clusters(int* n) {
    static std::atomic<int> known[16];  // of the first devices; every call of few rows asks for it
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return set_cuda_error(e);
    if (dev < 16 && (*n = known[dev].load(std::memory_order_relaxed)) > 0) return PVQ_OK;
    const void* kernel = reinterpret_cast<const void*>(matmul_few_kernel<ROWS, SPLIT, false, __nv_bfloat16>);  // (the others take the same)
    int st = allow_shared(kernel, Shape<ROWS, SPLIT>::kShared);
    if (st == PVQ_OK) st = clusters_of(kernel, kThreads, Shape<ROWS, SPLIT>::kShared, SPLIT, n);
    if (st == PVQ_OK && dev < 16) known[dev].store(*n, std::memory_order_relaxed);
    return st;
}
template <int ROWS>
int clusters_split(int split, int* n) {
    return split == 2 ? clusters<ROWS, 2>(n) : (split == 4 ? clusters<ROWS, 4>(n) : clusters<ROWS, 8>(n));
}

}  // namespace

int matmul_few_clusters(int high, int split, int* n) {
    if (high == 16) return clusters_split<16>(split, n);
    if (high == 32) return clusters_split<32>(split, n);
    return high == 64 ? clusters_split<64>(split, n) : clusters_split<128>(split, n);
}

int matmul_few(const MatmulArgs& p, bool transposed, bool bf16, int split, cudaStream_t s) {
    if (p.rows <= 16) return launch_rows<16>(p, transposed, bf16, split, s);
    if (p.rows <= 32) return launch_rows<32>(p, transposed, bf16, split, s);
    if (p.rows <= 64) return launch_rows<64>(p, transposed, bf16, split, s);
    return launch_rows<128>(p, transposed, bf16, split, s);
}

}  // namespace fp8
}  // namespace pvq
