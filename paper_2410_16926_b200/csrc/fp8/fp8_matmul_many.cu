// The 8-bit product where there is enough of it to fill the GPU: out[i][j] = sum_k a(i,k) b(j,k).
//
// A pair of thread blocks on two neighbouring SMs makes tiles of 256 x 256, each block 128 of the rows; each loads its 128
// rows of a and half of the 256 of b (32 KB a block of 128 along k), and the product reads both halves.  The scales are
// powers of two, which the tensor cores apply to the products of a step (32 values of k) before they add them, so that a
// tile's sum stays in tensor memory from the first to the last k, and is read once.
//
// Warps of a block: one issues the copies, one (of the pair's first block) the products, four bring the scales to tensor
// memory - four blocks along k at a time, double-buffered, a lane the words of its rows, the same in each quarter of the
// lanes as the product wants it -, eight read the result, round it and store it by tiled copies, a warp its own 32 rows.
// Tensor memory has 512 columns, too few for two results of 256 and the scales: the results of successive tiles overlap in 32
// columns, which are read first, so that the next tile's products wait for those alone (875 us for 16384 x 4096 by 14336 when
// they waited for all, 829 so).
//
// What bounds it: the power limit.  16384 x 4096 by 14336 takes 790 to 840 us (2.3 to 2.4 PFLOP/s), at 1000 W and 1.15 GHz, with
// the tensor cores at work nine cycles in ten; for a few milliseconds, at a full clock, 690 us.  Multicast copies, which would spare
// the L2 cache half of its reads, are not used: they must never read another GPU's memory, and a kernel cannot see whose its
// operands are.
#include "fp8_matmul.cuh"

namespace pvq {
namespace fp8 {
namespace {

constexpr int kStages = 5, kStageBytes = 2 * 128 * kBlock, kThreads = 512;
constexpr int kStoreBytes = 4096;  // 32 rows of 128 bytes
constexpr int kSecond = 224;                   // first column of odd tiles' results; the first 32 of them are even tiles' last
constexpr int kScalesA = 480, kScalesB = 488;  // columns, two buffers of 4 and of 8
constexpr int kGroup = 8;  // tiles down that are taken together across
// fp32 results of more than kRun blocks along k are summed in parts of about as many: sums in tensor memory are cut off, not
// rounded, and come out 8e-8 of themselves too small for every 1024 values (14336 values: 1.1e-6).  The parts are added in
// registers, for which the warpgroups share those of the block out anew.
constexpr int kRun = 64, kRegisters = 128, kFew = 48, kSome = 64, kMany = 200;
static_assert(kFew + kSome + 2 * kMany <= 4 * kRegisters, "a share beyond these would be waited for without end");
constexpr size_t kShared = 1024 + kStages * kStageBytes + 8 * 2 * kStoreBytes + 256;

struct Maps {
    CUtensorMap a, b, out;
};

struct Tiles {
    int down, across;
    __device__ __forceinline__ int count() const { return down * across; }
    // Tiles of kGroup rows of tiles go down first, so that those of one moment share what they read.
    __device__ __forceinline__ void at(int t, int* m, int* n) const {
        const int group = t / (kGroup * across), first = group * kGroup, rest = t - group * kGroup * across;
        const int high = min(kGroup, down - first);
        *m = first + rest % high;
        *n = rest / high;
    }
};

template <bool ACROSS, class T>
__global__ void __launch_bounds__(kThreads, 1) matmul_many_kernel(const __grid_constant__ Maps maps, const __grid_constant__ MatmulArgs p) {
    extern __shared__ uint8_t raw[];
    const uint32_t base = (shared_address(raw) + 1023u) & ~1023u;
    const uint32_t stores = base + kStages * kStageBytes, bars = stores + 8 * 2 * kStoreBytes;
    const uint32_t full = bars, empty = full + 8 * kStages, scales_full = empty + 8 * kStages, scales_empty = scales_full + 16, sum_full = scales_empty + 16,
                   sum_empty = sum_full + 16, shared_empty = sum_empty + 16, drained = shared_empty + 8;
    __shared__ uint32_t tensor_base, issued_stages[2];  // (issued: this block's stages, and the other's once a wait has run out)
    __shared__ int lost_from[8];  // a warp's first tile without a result
    __shared__ int over;  // a wait has run out in either block
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    if (warp == 0) {  // a barrier a lane, in the order of their places
        constexpr int kBars = 2 * kStages + 10;
        static_assert(kBars <= 32, "one lane each");
        const int i = lane - 2 * kStages;  // scales' full and empty, sum's full and empty, two each; shared, drained
        if (lane < kBars) barrier_init(full + 8 * lane, i == 0 || i == 1 || i == 8 ? 8 : (i == 6 || i == 7 ? 16 : 1));
        barrier_init_fence();
        if (lane == 0) {
            over = 0;
            prefetch_map(&maps.a), prefetch_map(&maps.b), prefetch_map(&maps.out);
        }
    }
    if (warp == 2) tensor_alloc<true>(shared_address(&tensor_base), 512);
    tensor_fence_before();
    __syncthreads();
    cluster_barrier();
    tensor_fence_after();
    launch_dependents();
    dependency_wait();
    const uint32_t tensor = tensor_base;
    Bounds bounds{&over, p.status, 2};
    const Withheld withheld = withheld_of(bounds, rank);
    const Tiles tiles{static_cast<int>((p.rows + 255) / 256), static_cast<int>((p.outs + 255) / 256)};
    const int blocks = static_cast<int>((p.inner + kBlock - 1) / kBlock), first = blockIdx.x / 2, step = gridDim.x / 2;
    constexpr bool kParts = sizeof(T) == 4;
    const int about = kParts ? (blocks + kRun - 1) / kRun : 1, part_blocks = (blocks + about - 1) / about, parts = (blocks + part_blocks - 1) / part_blocks;

    const uint32_t full_there = address_in(full, 0);
    const auto load = [&](uint32_t stage, int row, int col, int kb) {
        const uint32_t at = base + stage * kStageBytes;
        if (rank == 0) barrier_expect(full + 8 * stage, 2 * kStageBytes);  // both blocks' tiles
        load_tile<true>(at, &maps.a, kb * kBlock, row, full_there + 8 * stage);
        if (ACROSS) load_tile<true>(at + kStageBytes / 2, &maps.b, col, kb * kBlock, full_there + 8 * stage);
        else load_tile<true>(at + kStageBytes / 2, &maps.b, kb * kBlock, col, full_there + 8 * stage);
    };

    if (warp < 4) {
        if constexpr (kParts) fewer_registers<kFew>();
    }
    if (warp == 0) {
        if (elected()) {
            Turn<kStages> turn;
            uint32_t issued = 0;
            bool ok = true;
            for (int t = first; t < tiles.count() && ok; t += step) {
                int m, n;
                tiles.at(t, &m, &n);
                const int row = m * 256 + rank * 128, col = n * 256 + rank * 128;
                for (int kb = 0; kb < blocks; ++kb) {
                    ok = !(withheld.copies && issued >= kStages + kWithheldFrom) && barrier_wait<true>(empty + 8 * turn.at, turn.parity ^ 1, bounds);
                    if (!ok) break;
                    load(turn.at, row, col, kb);
                    turn.next();
                    ++issued;
                }
            }
            issued_stages[rank] = issued;
        }
    } else if (warp == 1) {
        if (rank == 0 && elected()) {
            constexpr uint32_t product = product_e4m3(256, 256, false, ACROSS);
            constexpr uint32_t kAlongB = (ACROSS ? 32 * kBlock : 32) >> 4;
            const uint64_t a0 = operand(base), b0 = operand(base + kStageBytes / 2, ACROSS ? kStageBytes / 2 : 16);
            Turn<kStages> turn;
            Turn<2> scales;
            Turn<2> sums;           // the two places of the result
            uint32_t shared = 1;    // the parity of the columns that they share
            bool ok = true, there = false;
            for (int t = first; t < tiles.count() && ok; t += step) {
                int left = 0;  // of the part
                for (int kb = 0; kb < blocks; ++kb, --left) {
                    const uint32_t part = kb & 3;
                    const bool starts = left == 0;
                    if (starts) {
                        ok = barrier_wait<true>(sum_empty + 8 * sums.at, sums.parity ^ 1, bounds) && barrier_wait<true>(shared_empty, shared, bounds);
                        left = part_blocks;
                    }
                    if (part == 0) ok = ok && barrier_wait<true>(scales_full + 8 * scales.at, scales.parity, bounds);
                    ok = ok && (there || barrier_wait<true>(full + 8 * turn.at, turn.parity, bounds));
                    if (!ok) break;
                    const uint32_t now = turn.at;
                    turn.next();
                    there = barrier_over<true>(full + 8 * turn.at, turn.parity);
                    tensor_fence_after();
                    const uint64_t a = a0 + now * (kStageBytes >> 4), b = b0 + now * (kStageBytes >> 4);
                    const uint32_t sum = tensor + kSecond * sums.at, sa = tensor + kScalesA + 4 * scales.at, sb = tensor + kScalesB + 8 * scales.at,
                                   with = with_part(product, part);
#pragma unroll
                    for (int k = 0; k < 4; ++k) multiply_e4m3<true>(sum, a + 2 * k, b + kAlongB * k, with, sa, sb, !starts || k > 0);
                    products_done<true>(empty + 8 * now);
                    if (part == 3 || kb == blocks - 1) {
                        products_done<true>(scales_empty + 8 * scales.at);
                        scales.next();
                    }
                    if (left == 1 || kb == blocks - 1) {
                        products_done<true>(sum_full + 8 * sums.at);
                        sums.next();
                        shared ^= 1;
                    }
                }
            }
            if (!ok) {
                products_done<true>(drained);
                for (int polls = 0; polls < kLandings && !barrier_passed<true>(drained, 0); ++polls) {}
            }
        }
    } else if (warp >= 4 && warp < 8) {
        if constexpr (kParts) fewer_registers<kSome>();
        const uint32_t mine = tensor + ((warp & 3) << 21);
        const uint32_t full_there = address_in(scales_full, 0);
        // The words of four blocks along k are asked for two such steps before they are needed, in two sets of registers that
        // take turns (to hand a loaded word on is to wait for it): one step at a time took 350 ns a block.
        struct Step {
            int t, kb;
        } next{first, 0};
        uint32_t a[2][4], b[2][8], four = 0;
        const auto load = [&](uint32_t (&a)[4], uint32_t (&b)[8]) {
            if (next.t < tiles.count()) {
                int m, n;
                tiles.at(next.t, &m, &n);
                scale_words<false>(p.a, int64_t(m) * 256 + rank * 128, next.kb / 4, a);
                scale_words<ACROSS>(p.b, int64_t(n) * 256, next.kb / 4, b);
                next.kb += 4;
                if (next.kb >= blocks) next.kb = 0, next.t += step;
            }
        };
        const auto put = [&](const uint32_t (&a)[4], const uint32_t (&b)[8]) -> bool {
            const uint32_t buffer = four & 1;
            if (four >= 2) {
                if (!warp_wait<true>(scales_empty + 8 * buffer, ((four >> 1) - 1) & 1, bounds)) return false;
                tensor_fence_after();
            }
            tensor_store(mine + kScalesA + 4 * buffer, a);
            tensor_store(mine + kScalesB + 8 * buffer, b);
            tensor_wait_stores();
            tensor_fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive_in(full_there + 8 * buffer);
            ++four;
            return true;
        };
        load(a[0], b[0]);
        load(a[1], b[1]);
        const int64_t steps = int64_t((tiles.count() - first + step - 1) / step) * ((blocks + 3) / 4);
        for (int64_t i = 0; i < steps; i += 2) {
            if (withheld.scales && i >= kWithheldFrom) break;
            if (!put(a[0], b[0])) break;
            load(a[0], b[0]);
            if (i + 1 >= steps || !put(a[1], b[1])) break;
            load(a[1], b[1]);
        }
    } else if (warp >= 8) {
        constexpr int kColumns = 128 / sizeof(T);  // of a stored tile
        const int quarter = warp & 3, half = (warp - 8) >> 2;
        constexpr int kChunks = 128 / kColumns;
        const uint32_t buffers = stores + (warp - 8) * 2 * kStoreBytes, empty_there = address_in(sum_empty, 0), shared_there = address_in(shared_empty, 0);
        if constexpr (kParts) more_registers<kMany>();
        // A chunk of 32 words a lane (bf16: 64 columns, fp32: 32) to memory.
        uint32_t buffer = 0;
        const auto put = [&](const uint32_t (&w)[32], int64_t row, int64_t col) {
            // A tiled store ends at a multiple of 16 bytes behind the last column: where that is not the row's end, and
            // might be another matrix's, the last tile is stored by values.
            if (col + kColumns > p.outs && p.outs * sizeof(T) % 16 != 0) {
                if (row + lane < p.rows) {
                    T* to_row = static_cast<T*>(p.out) + (row + lane) * p.ld + col;
#pragma unroll
                    for (int i = 0; i < kColumns; ++i)
                        if (col + i < p.outs) {
                            if constexpr (sizeof(T) == 2) reinterpret_cast<uint16_t*>(to_row)[i] = static_cast<uint16_t>(w[i / 2] >> (16 * (i & 1)));
                            else reinterpret_cast<uint32_t*>(to_row)[i] = w[i];
                        }
                }
                return;
            }
            const uint32_t to = buffers + buffer * kStoreBytes;
            buffer ^= 1;
            if (lane == 0) store_wait_read<1>();
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 8; ++j)
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + lane * 128 + ((j ^ (lane & 7)) << 4)), "r"(w[4 * j]), "r"(w[4 * j + 1]),
                             "r"(w[4 * j + 2]), "r"(w[4 * j + 3])
                             : "memory");
            async_fence();
            __syncwarp();
            if (lane == 0) {
                if (row < p.rows && col < p.outs) store_tile(&maps.out, static_cast<int>(col), static_cast<int>(row), to);
                store_commit();
            }
        };
        // Parts of tiles: even ones share their last columns with the next, odd ones their first.  Each half begins with what it
        // may share: the right one goes backwards.
        uint32_t item = 0;
        const auto chunk = [&](int i) { return half ? kChunks - 1 - i : i; };
        int t = first;
        for (; t < tiles.count(); t += step) {
            int m, n;
            tiles.at(t, &m, &n);
            const int64_t row = int64_t(m) * 256 + rank * 128 + quarter * 32, col = int64_t(n) * 256 + half * 128;
            bool ok = true;
            const auto read = [&](int i) {  // has read chunk i of four or two
                if ((i == 0 && half == ((item & 1) ^ 1)) || i == kChunks - 1) {
                    tensor_fence_before();
                    __syncwarp();
                    if (lane == 0 && i == 0 && half == ((item & 1) ^ 1)) barrier_arrive_in(shared_there);
                    if (lane == 0 && i == kChunks - 1) barrier_arrive_in(empty_there + 8 * (item & 1));
                }
            };
            if constexpr (kParts) {
                float sum[128];
#pragma unroll
                for (int k = 0; k < 128; ++k) sum[k] = 0.0f;
#pragma unroll 1
                for (int part = 0; part < parts; ++part, ++item) {
                    ok = warp_wait<true>(sum_full + 8 * (item & 1), (item >> 1) & 1, bounds);
                    if (!ok) break;
                    tensor_fence_after();
                    const uint32_t mine = tensor + (quarter << 21) + (item & 1) * kSecond + half * 128;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float v[32];
                        tensor_load(mine + chunk(i) * 32, v);
                        tensor_wait_loads();
                        read(i);
#pragma unroll
                        for (int k = 0; k < 32; ++k) sum[i * 32 + k] += v[k];
                    }
                }
                if (!ok) break;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t w[32];
#pragma unroll
                    for (int k = 0; k < 32; ++k) w[k] = __float_as_uint(sum[i * 32 + k]);
                    put(w, row, col + chunk(i) * 32);
                }
            } else {
                ok = warp_wait<true>(sum_full + 8 * (item & 1), (item >> 1) & 1, bounds);
                if (!ok) break;
                tensor_fence_after();
                const uint32_t mine = tensor + (quarter << 21) + (item & 1) * kSecond + half * 128;
#pragma unroll 1
                for (int i = 0; i < kChunks; ++i) {
                    const int c = chunk(i);
                    float v[kColumns];
#pragma unroll
                    for (int k = 0; k < kColumns; k += 32) tensor_load(mine + c * kColumns + k, reinterpret_cast<float(&)[32]>(v[k]));
                    tensor_wait_loads();
                    read(i);
                    uint32_t w[32];
#pragma unroll
                    for (int k = 0; k < 32; ++k) w[k] = bf16x2_of(v[2 * k], v[2 * k + 1]);
                    put(w, row, col + c * kColumns);
                }
                ++item;
            }
        }
        if (lane == 0) lost_from[warp - 8] = t;
        if (lane == 0) store_wait_all();
    }
    __syncwarp();
    tensor_fence_before();
    __syncthreads();
    cluster_barrier();
    if (__builtin_expect(over, 0)) {
        // Copies in flight have to land before their block ends, and both blocks' report to the first's barriers.  Stages that one of
        // them did not ask for any more are filled up, so that each report is complete.
        if (threadIdx.x == 0) store_in(address_in(shared_address(&issued_stages[rank]), rank ^ 1), issued_stages[rank]);
        __syncwarp();
        cluster_barrier();
        if (threadIdx.x == 0) {
            const uint32_t all = max(issued_stages[0], issued_stages[1]);
#pragma unroll 1
            for (uint32_t i = issued_stages[rank]; i < all; ++i) load(i % kStages, 0, 0, 0);
            if (rank == 0) land<kStages, true>(full, all);
        }
        if (warp >= 8)
#pragma unroll 1
            for (int t = lost_from[warp - 8]; t < tiles.count(); t += step) {
                int m, n;
                tiles.at(t, &m, &n);
                spoil(static_cast<T*>(p.out), p.ld, int64_t(m) * 256 + rank * 128 + (warp & 3) * 32, p.rows, int64_t(n) * 256 + (warp - 8) / 4 * 128, p.outs, 128);
            }
        __syncwarp();
        cluster_barrier();
    }
    if (warp == 2) tensor_free<true>(tensor, 512);
}

template <bool ACROSS, class T>
int launch(const MatmulArgs& p, cudaStream_t s) {
    Maps maps;
    const Element out = sizeof(T) == 2 ? Element::kBf16 : Element::kF32;
    int st = tile_map(&maps.a, p.a.codes, Element::kByte, p.a.rows, p.a.cols, p.a.ld_codes, kBlock, 128);
    if (st == PVQ_OK) st = tile_map(&maps.b, p.b.codes, Element::kByte, p.b.rows, p.b.cols, p.b.ld_codes, kBlock, 128);
    if (st == PVQ_OK) st = tile_map(&maps.out, p.out, out, p.rows, p.outs, p.ld, 128 / sizeof(T), 32);
    void (*const kernel)(Maps, MatmulArgs) = matmul_many_kernel<ACROSS, T>;
    if (st == PVQ_OK && sizeof(T) == 4) {
        int registers = 0;
        st = registers_of(reinterpret_cast<const void*>(kernel), &registers);
        if (st == PVQ_OK && registers < kRegisters) st = PVQ_ERR_UNSUPPORTED;
    }
    if (st == PVQ_OK) st = allow_shared(reinterpret_cast<const void*>(kernel), kShared);
    if (st != PVQ_OK) return st;
    const int64_t tiles = ((p.rows + 255) / 256) * ((p.outs + 255) / 256);
    if (tiles >= int64_t(1) << 30) return PVQ_ERR_UNSUPPORTED;
    const unsigned pairs = static_cast<unsigned>(tiles < kSms / 2 ? tiles : kSms / 2);
    return launch_early(kernel, dim3(2 * pairs), kThreads, kShared, 2, s, maps, p);
}

}  // namespace

int matmul_many(const MatmulArgs& p, bool transposed, bool bf16, cudaStream_t s) {
    if (transposed) return bf16 ? launch<true, __nv_bfloat16>(p, s) : launch<true, float>(p, s);
    return bf16 ? launch<false, __nv_bfloat16>(p, s) : launch<false, float>(p, s);
}

}  // namespace fp8
}  // namespace pvq
