// The gradient of a weight from the 8-bit input that was kept: out[o][i] = sum_t dy[t][o] x[t][i].
//
// The scales of x lie along t, inside the sum, so x is made bf16 (a code times a power of two: exact) on its way to the
// tensor cores: tiles of codes arrive by tiled copies, eight warps convert them into the operand's layout, and the product
// takes both operands across k, as they lie in memory.  The tensor cores cut off what an addition to a running sum loses
// instead of rounding it: over 16384 values of t a sum in tensor memory ends 1.9e-5 of itself too small.  So after every
// 512 values of t the sum is read and added to one in registers (fp32, rounded to nearest), while the products go on in
// a second buffer.
//
// PAIR: two blocks on neighbouring SMs make 256 x 256 of the result, each 128 rows of it and half of the other operand.
// Otherwise a block makes 128 x 128, and where there are few tiles the blocks of a cluster split t, and add their sums
// through one another's shared memory in the order of the ranks.
//
// READY: x lies in the caller's workspace as bf16, converted once and not for every 256 rows of the result, and is copied like
// dy: 16384 tokens, 14336 x 4096, 1480 us instead of 1730, the conversion in front included.  What bounds it there is the power
// limit (1000 W): work saved is clock gained.  Short products are bound by what comes before the first and after the last
// step: 1001 tokens, 1024 x 4096, 13.4 us, of which the operations take 5.
//
// Warps of a block: one issues the copies, one the products, eight convert, eight hold and store the sums.
#include "fp8_mma.cuh"

namespace pvq {
namespace fp8 {
namespace {

constexpr int kDepth = 64;                    // values of t a stage
constexpr int kAtom = kDepth * 128;           // bytes from 64 bf16 columns to the next 64
// A stage: 128 columns of dy (bf16) and 128 of x, as codes, or READY: as bf16.
template <bool READY>
struct Shape {
    static constexpr int kConverters = READY ? 0 : 8;  // warps
    static constexpr int kThreads = 32 * (4 + kConverters + 8);
    static constexpr int kStages = READY ? 6 : 5, kStageBytes = (READY ? 4 : 3) * kAtom;
    static constexpr int kConverted = READY ? 0 : 4;
    static constexpr size_t kShared = 1024 + kStages * kStageBytes + kConverted * 2 * kAtom + 8 * 4096 + 256;
};
constexpr int kRun = 512 / kDepth;            // stages that are added in tensor memory
constexpr int kStoreBytes = 4096;             // 32 rows of 128 bytes
constexpr int kGroup = 8;                     // tiles down that are taken together across

struct Maps {
    CUtensorMap dy, x, out;
};
struct Args {
    Matrix x;
    void* out;
    int64_t outer, ld;
    uint32_t* status;
    int split;
    int tiles;  // of this launch
    int after;  // without PAIR: tiles are quarters of pairs' tiles from this one on (-1: tiles of their own)
};

// Registers a thread of the five warpgroups of a pair's block: what all are launched with, shared out anew.  A sum of 128
// columns takes 128 of them.
constexpr int kRegisters = 96, kFew = 32, kSome = 56, kMany = 168;
static_assert(kFew + 2 * kSome + 2 * kMany <= 5 * kRegisters, "a share beyond these would be waited for without end");

// Column j of four neighbouring ones lies in place turned(j) of the converted operand, and so of the sums: two codes of a word
// are made two values where they are, bytes 0 and 2, 1 and 3.
__host__ __device__ constexpr int turned(int j) { return (j & ~3) | (j & 1) << 1 | (j & 2) >> 1; }

// 64 codes of a row to bf16, by integer instructions (16384 tokens, 14336 x 4096, without a workspace: 1727 us, by conversion
// instructions 1861): a code's exponent and mantissa, in the places of bf16's, are its value times 2^-120, subnormal ones too,
// and a product with 2^120 times the scale is exact.  False where that is not enough: a NaN among the
// codes (magnitude 0x7f), a scale above 2^7, or NaN.
__device__ __forceinline__ bool convert_row(uint32_t from, uint32_t to, int half, int row, uint32_t byte) {
    const uint32_t one = (byte + 120u) << 7, factor = one | one << 16;
    uint32_t most = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t w[4], v[8];
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                     : "r"(from + (((half * 4 + j) ^ (row & 7)) << 4)));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t even = (w[i] << 4) & 0x07f007f0u, odd = (w[i] >> 4) & 0x07f007f0u;
            asm("max.u16x2 %0, %0, %1;" : "+r"(most) : "r"(even));
            asm("max.u16x2 %0, %0, %1;" : "+r"(most) : "r"(odd));
            asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(v[2 * i]) : "r"(((w[i] << 8) & 0x80008000u) | even), "r"(factor));
            asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(v[2 * i + 1]) : "r"((w[i] & 0x80008000u) | odd), "r"(factor));
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (((2 * j + i) ^ (row & 7)) << 4)), "r"(v[4 * i]), "r"(v[4 * i + 1]),
                         "r"(v[4 * i + 2]), "r"(v[4 * i + 3])
                         : "memory");
    }
    return byte <= 134u && (most & 0xffffu) != 0x07f0u && (most >> 16) != 0x07f0u;
}
// ... any codes and scale, by fp32.
__device__ __forceinline__ void convert_row_any(uint32_t from, uint32_t to, int half, int row, uint32_t byte) {
    const float scale = scale_of(byte);
#pragma unroll 1
    for (int j = 0; j < 8; ++j) {  // eight codes
        uint32_t w[2], v[4];
        asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(from + (((half * 4 + j / 2) ^ (row & 7)) << 4) + j % 2 * 8));
        for (int i = 0; i < 2; ++i) {
            const float2 lo = values_of(w[i] & 0xffffu), hi = values_of(w[i] >> 16);
            v[2 * i] = bf16x2_of(lo.x * scale, hi.x * scale);
            v[2 * i + 1] = bf16x2_of(lo.y * scale, hi.y * scale);
        }
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + ((j ^ (row & 7)) << 4)), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
    }
}

template <bool PAIR, bool READY, class T>
__global__ void __launch_bounds__(Shape<READY>::kThreads, 1) weight_grad_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Args p) {
    using S = Shape<READY>;
    constexpr int kStages = S::kStages, kStageBytes = S::kStageBytes, kConverted = S::kConverted, kConvertedBytes = 2 * kAtom;
    constexpr int kFirstHolder = 4 + S::kConverters;  // warp
    constexpr int kSide = PAIR ? 256 : 128;   // of a tile
    constexpr int kHeld = kSide / 2;          // columns of the sum a warp holds
    constexpr uint32_t kBlocks = PAIR ? 2 : 1;
    static_assert(8 * (kHeld * sizeof(T) / 128 - 1) * kStoreBytes <= kStages * kStageBytes, "the last tile is stored from the stages' place");
    extern __shared__ uint8_t raw[];
    const uint32_t base = (shared_address(raw) + 1023u) & ~1023u;
    const uint32_t converted = base + kStages * kStageBytes, stores = converted + kConverted * kConvertedBytes, bars = stores + 8 * kStoreBytes;
    const uint32_t full_dy = bars, full_x = full_dy + 8 * kStages, empty = full_x + 8 * kStages, converted_full = empty + 8 * kStages,
                   converted_empty = converted_full + 8 * kConverted, sum_full = converted_empty + 8 * kConverted, sum_empty = sum_full + 16,
                   drained = sum_empty + 16;
    __shared__ uint32_t tensor_base, issued_stages[2];  // (issued: this block's stages, and the pair's other's once a wait has run out)
    __shared__ int lost_from[8];  // a warp's first tile without a result
    __shared__ int over;          // a wait has run out in any block of the cluster
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_rank() : 0;              // in the pair
    const int part = PAIR ? 0 : static_cast<int>(cluster_rank());  // of t
    if (warp == 0) {  // a barrier a lane, in the order of their places
        constexpr int kBars = 3 * kStages + 2 * kConverted + 5;
        static_assert(kBars <= 32, "one lane each");
        const int i = lane - 3 * kStages, j = i - 2 * kConverted;  // converted full and empty; sum's full and empty, two each; drained
        if (lane < kBars) barrier_init(full_dy + 8 * lane, i >= 0 && i < kConverted ? 4 * kBlocks : (j == 2 || j == 3 ? 8 * kBlocks : 1));
        barrier_init_fence();
        if (lane == 0) {
            over = 0;
            prefetch_map(&maps.dy), prefetch_map(&maps.x), prefetch_map(&maps.out);
        }
    }
    if (warp == 2) tensor_alloc<PAIR>(shared_address(&tensor_base), 2 * kSide);
    tensor_fence_before();
    __syncthreads();
    cluster_barrier();
    tensor_fence_after();
    launch_dependents();
    dependency_wait();
    const uint32_t tensor = tensor_base;
    Bounds bounds{&over, p.status, static_cast<uint32_t>(PAIR ? 2 : p.split)};
    const Withheld withheld = withheld_of(bounds, PAIR ? rank : part);
    const bool quarters = !PAIR && p.after >= 0;
    const int side = quarters ? 256 : kSide, tiles = p.tiles;
    const int down = static_cast<int>((p.outer + side - 1) / side), across = static_cast<int>((p.x.cols + side - 1) / side);
    const int team = PAIR ? 2 : p.split, step = gridDim.x / team;
    const int stages = static_cast<int>((p.x.rows + kDepth - 1) / kDepth);
    const int begin = static_cast<int>(int64_t(stages) * part / p.split), end = static_cast<int>(int64_t(stages) * (part + 1) / p.split);

    // Tiles of kGroup rows of tiles go down first, so that those of one moment share what they read.
    const auto tile_at = [&](int t, int* m, int* n) {
        const int i = quarters ? p.after + t / 4 : t;
        const int group = i / (kGroup * across), first = group * kGroup, rest = i - group * kGroup * across, high = min(kGroup, down - first);
        *m = first + rest % high;
        *n = rest / high;
        if (quarters) *m = 2 * *m + (t & 1), *n = 2 * *n + (t >> 1 & 1);
    };

    const uint32_t dy_there = PAIR ? address_in(full_dy, 0) : full_dy;
    const auto load = [&](uint32_t stage, int row, int col, int kb) {
        const uint32_t at = base + stage * kStageBytes, bar = dy_there + 8 * stage;
        if (rank == 0) barrier_expect(full_dy + 8 * stage, kBlocks * (READY ? 4 : 2) * kAtom);
        if constexpr (READY) {
            load_tile<PAIR>(at + 2 * kAtom, &maps.x, col, kb * kDepth, bar);
            load_tile<PAIR>(at + 3 * kAtom, &maps.x, col + 64, kb * kDepth, bar);
        } else {
            barrier_expect(full_x + 8 * stage, kAtom);
            load_tile<false>(at + 2 * kAtom, &maps.x, col, kb * kDepth, full_x + 8 * stage);
        }
        load_tile<PAIR>(at, &maps.dy, row, kb * kDepth, bar);
        load_tile<PAIR>(at + kAtom, &maps.dy, row + 64, kb * kDepth, bar);
    };

    if (warp < 4) {
        if constexpr (!READY) fewer_registers<kFew>();
        if (warp == 0 && elected()) {
            Turn<kStages> turn;
            uint32_t issued = 0;
            bool ok = true;
            for (int t = blockIdx.x / team; t < tiles && ok; t += step) {
                int m, n;
                tile_at(t, &m, &n);
                const int row = m * kSide + rank * 128, col = n * kSide + rank * 128;
                for (int kb = begin; kb < end; ++kb) {
                    ok = !(withheld.copies && issued >= kStages + kWithheldFrom) && barrier_wait<PAIR>(empty + 8 * turn.at, turn.parity ^ 1, bounds);
                    if (!ok) break;
                    load(turn.at, row, col, kb);
                    turn.next();
                    ++issued;
                }
            }
            issued_stages[rank] = issued;
        } else if (warp == 1 && rank == 0 && elected()) {
            constexpr uint32_t product = product_bf16(kSide, kSide, true, true);
            const uint64_t a0 = operand(base, kAtom), b0 = operand(READY ? base + 2 * kAtom : converted, kAtom);
            Turn<kStages> turn;
            Turn<kConverted> ready;
            Turn<2> sums;
            bool ok = true;
            for (int t = blockIdx.x / team; t < tiles && ok; t += step) {
                int within = 0;
                for (int kb = begin; kb < end; ++kb) {
                    if (within == 0) ok = barrier_wait<PAIR>(sum_empty + 8 * sums.at, sums.parity ^ 1, bounds);
                    ok = ok && barrier_wait<PAIR>(full_dy + 8 * turn.at, turn.parity, bounds);
                    if constexpr (!READY) ok = ok && barrier_wait<PAIR>(converted_full + 8 * ready.at, ready.parity, bounds);
                    if (!ok) break;
                    tensor_fence_after();
                    const uint64_t a = a0 + turn.at * (kStageBytes >> 4), b = b0 + (READY ? turn.at * (kStageBytes >> 4) : ready.at * (kConvertedBytes >> 4));
#pragma unroll
                    for (int k = 0; k < kDepth / 16; ++k) multiply_bf16<PAIR>(tensor + sums.at * kSide, a + 128 * k, b + 128 * k, product, within > 0 || k > 0);
                    products_done<PAIR>(empty + 8 * turn.at);
                    if constexpr (!READY) {
                        products_done<PAIR>(converted_empty + 8 * ready.at);
                        ready.next();
                    }
                    turn.next();
                    if (++within == kRun || kb == end - 1) {
                        products_done<PAIR>(sum_full + 8 * sums.at);
                        sums.next();
                        within = 0;
                    }
                }
            }
            if (!ok) {
                products_done<PAIR>(drained);
                for (int polls = 0; polls < kLandings && !barrier_passed<PAIR>(drained, 0); ++polls) {}
            }
        }
    } else if (warp < kFirstHolder) {
        if constexpr (!READY) {
        fewer_registers<kSome>();
        // a thread takes 64 codes of one t: a row of the tile, eight neighbouring rows in eight different places
        const int row = lane + 32 * (warp & 1), half = (warp >> 1) & 1;
        const uint32_t full_there = PAIR ? address_in(converted_full, 0) : converted_full;
        const int turn = (warp - 4) >> 2;  // four warps take a tile's even stages, four the odd ones
        uint32_t it0 = 0;
        bool ok = true;
        for (int t = blockIdx.x / team; t < tiles && ok; t += step, it0 += end - begin) {
            int m, n;
            tile_at(t, &m, &n);
            const int block = n * (kSide / kBlock) + rank;
            const uint8_t* scales = p.x.scales + block;
            const auto scale_at = [&](int kb) -> uint32_t {  // (rows behind the end: codes of zero)
                const uint32_t r = uint32_t(kb) * kDepth + row;
                return kb < end && r < uint32_t(p.x.rows) && block < p.x.blocks ? __ldg(scales + (r >> p.x.shift) * p.x.ld_scales) : 127u;
            };
            // (loaded for four stages at a time, those of the next four meanwhile: to hand a loaded value on is to wait for it)
            uint32_t bytes, next[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) next[i] = scale_at(begin + turn + 2 * i);
            for (int kb0 = begin + turn; kb0 < end && ok; kb0 += 8) {
                bytes = next[0] | next[1] << 8 | next[2] << 16 | next[3] << 24;
#pragma unroll
                for (int i = 0; i < 4; ++i) next[i] = scale_at(kb0 + 8 + 2 * i);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (kb0 + 2 * i >= end) break;
                    ok = !(withheld.scales && it0 + (kb0 + 2 * i - begin) >= kStages + kWithheldFrom);
                    if (!ok) break;
                    const uint32_t it = it0 + (kb0 + 2 * i - begin), s = it % kStages, c = it % kConverted;
                    ok = warp_wait(full_x + 8 * s, (it / kStages) & 1, bounds) && warp_wait<PAIR>(converted_empty + 8 * c, ((it / kConverted) & 1) ^ 1, bounds);
                    if (!ok) break;
                    const uint32_t from = base + s * kStageBytes + 2 * kAtom + row * 128, to = converted + c * kConvertedBytes + half * kAtom + row * 128;
                    const uint32_t byte = (bytes >> (8 * i)) & 0xffu;
                    if (!convert_row(from, to, half, row, byte)) convert_row_any(from, to, half, row, byte);
                    async_fence();
                    __syncwarp();
                    if (lane == 0) {
                        if (PAIR) {
                            release_shared();
                            barrier_arrive_in(full_there + 8 * c);
                        } else {
                            barrier_arrive(full_there + 8 * c);
                        }
                    }
                }
            }
        }
        }
    } else {
        if constexpr (!READY) more_registers<kMany>();
        constexpr int kColumns = 128 / sizeof(T);  // of a stored tile
        const int quarter = warp & 3, half = (warp - kFirstHolder) >> 2;
        const uint32_t buffer_at = stores + (warp - kFirstHolder) * kStoreBytes, empty_there = PAIR ? address_in(sum_empty, 0) : sum_empty;
        const uint32_t mine = tensor + (quarter << 21) + half * kHeld;
        const auto place = [](int j) { return READY ? j : turned(j); };
        uint32_t run = 0;
        int t = blockIdx.x / team;
        for (; t < tiles; t += step) {
            int m, n;
            tile_at(t, &m, &n);
            bool ok = true;
            float sum[kHeld];
#pragma unroll
            for (int i = 0; i < kHeld; ++i) sum[i] = 0.0f;
            for (int kb = begin; kb < end; kb += kRun, ++run) {
                const uint32_t buffer = run & 1;
                ok = warp_wait<PAIR>(sum_full + 8 * buffer, (run >> 1) & 1, bounds);
                if (!ok) break;
                tensor_fence_after();
#pragma unroll
                for (int c = 0; c < kHeld; c += 16) {
                    float v[16];
                    tensor_load(mine + buffer * kSide + c, v);
                    tensor_wait_loads();
#pragma unroll
                    for (int i = 0; i < 16; ++i) sum[c + i] += v[i];
                }
                tensor_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR) barrier_arrive_in(empty_there + 8 * buffer);
                    else barrier_arrive(empty_there + 8 * buffer);
                }
            }
            if (!ok) break;
            if (!PAIR && p.split > 1) {  // the part of the sum, in shared memory: [row][128], in places turned by the row
                const uint32_t to = base + (quarter * 32 + lane) * 512;
#pragma unroll
                for (int c = 0; c < kHeld / 4; ++c)
                    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to + (((half * (kHeld / 4) + c) ^ (lane & 7)) << 4)), "f"(sum[4 * c]),
                                 "f"(sum[place(4 * c + 1)]), "f"(sum[place(4 * c + 2)]), "f"(sum[4 * c + 3])
                                 : "memory");
                continue;  // (the only tile)
            }
            const int64_t row = int64_t(m) * kSide + rank * 128 + quarter * 32;
#pragma unroll
            for (int c = 0; c < kHeld / kColumns; ++c) {
                const int64_t col = int64_t(n) * kSide + half * kHeld + c * kColumns;
                uint32_t w[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    if constexpr (sizeof(T) == 2) w[i] = bf16x2_of(sum[c * kColumns + place(2 * i)], sum[c * kColumns + place(2 * i + 1)]);
                    else w[i] = __float_as_uint(sum[c * kColumns + place(i)]);
                }
                // A tiled store ends at a multiple of 16 bytes behind the last column: where that is not the row's end, and
                // might be another matrix's, the last tile is stored by values.
                if (col + kColumns > p.x.cols && p.x.cols * sizeof(T) % 16 != 0) {
                    if (row + lane < p.outer) {
                        T* to_row = static_cast<T*>(p.out) + (row + lane) * p.ld + col;
#pragma unroll
                        for (int i = 0; i < kColumns; ++i)
                            if (col + i < p.x.cols) {
                                if constexpr (sizeof(T) == 2) reinterpret_cast<uint16_t*>(to_row)[i] = static_cast<uint16_t>(w[i / 2] >> (16 * (i & 1)));
                                else reinterpret_cast<uint32_t*>(to_row)[i] = w[i];
                            }
                    }
                    continue;
                }
                // behind the last tile the stages are free: a place of its own for each stored tile (one after another through
                // one place they took 1.6 us)
                uint32_t at = buffer_at;
                if (c > 0 && t + step >= tiles) {
                    at = base + ((warp - kFirstHolder) * (kHeld / kColumns - 1) + c - 1) * kStoreBytes;
                } else {
                    if (lane == 0) store_wait_read<0>();
                    __syncwarp();
                }
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + lane * 128 + ((j ^ (lane & 7)) << 4)), "r"(w[4 * j]),
                                 "r"(w[4 * j + 1]), "r"(w[4 * j + 2]), "r"(w[4 * j + 3])
                                 : "memory");
                async_fence();
                __syncwarp();
                if (lane == 0) {
                    if (row < p.outer && col < p.x.cols) store_tile(&maps.out, static_cast<int>(col), static_cast<int>(row), at);
                    store_commit();
                }
            }
        }
        if (lane == 0) lost_from[warp - kFirstHolder] = t;
        if (lane == 0) store_wait_all();
    }
    __syncwarp();
    tensor_fence_before();
    __syncthreads();
    cluster_barrier();
    if (__builtin_expect(over, 0)) {
        if (PAIR) {
            // As in matmul_many_kernel: stages that one block did not ask for any more are filled up, and all copies land before
            // either block ends.
            if (threadIdx.x == 0) store_in(address_in(shared_address(&issued_stages[rank]), rank ^ 1), issued_stages[rank]);
            __syncwarp();
            cluster_barrier();
            if (threadIdx.x == 0) {
                const uint32_t all = max(issued_stages[0], issued_stages[1]);
#pragma unroll 1
                for (uint32_t i = issued_stages[rank]; i < all; ++i) load(i % kStages, 0, 0, 0);
                if (rank == 0) land<kStages, PAIR>(full_dy, all);
                if (!READY) land<kStages>(full_x, all);
            }
        } else if (warp == 0) {
            land<kStages>(full_dy, issued_stages[0]);
            if (!READY) land<kStages>(full_x, issued_stages[0]);
        }
        if (warp >= kFirstHolder && (PAIR || p.split == 1))
#pragma unroll 1
            for (int t = lost_from[warp - kFirstHolder]; t < tiles; t += step) {
                int m, n;
                tile_at(t, &m, &n);
                spoil(static_cast<T*>(p.out), p.ld, int64_t(m) * kSide + rank * 128 + (warp & 3) * 32, p.outer,
                      int64_t(n) * kSide + (warp - kFirstHolder) / 4 * kHeld, p.x.cols, kHeld);
            }
        __syncwarp();
        if (PAIR) cluster_barrier();
    }
    if (!PAIR && p.split > 1) {
        const bool lost = over;
        if (warp >= kFirstHolder) {  // this block's share of the rows, eight columns a thread
            int m, n;
            tile_at(blockIdx.x / team, &m, &n);
            const int thread = threadIdx.x - 32 * kFirstHolder, share = 128 / p.split, col = thread % 16 * 8;
            const int64_t left = p.x.cols - int64_t(n) * 128 - col;
            for (int r = part * share + thread / 16; r < (part + 1) * share; r += 16) {
                const int64_t row = int64_t(m) * 128 + r;
                if (row >= p.outer || left <= 0) break;
                float v[8] = {};
                for (int s = 0; s < p.split; ++s) {
                    float4 lo, hi;
                    const uint32_t lo_at = address_in(base + r * 512 + (((col / 4) ^ (r & 7)) << 4), s);
                    const uint32_t hi_at = address_in(base + r * 512 + (((col / 4 + 1) ^ (r & 7)) << 4), s);
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(lo.x), "=f"(lo.y), "=f"(lo.z), "=f"(lo.w) : "r"(lo_at));
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(hi.x), "=f"(hi.y), "=f"(hi.z), "=f"(hi.w) : "r"(hi_at));
                    v[0] += lo.x, v[1] += lo.y, v[2] += lo.z, v[3] += lo.w, v[4] += hi.x, v[5] += hi.y, v[6] += hi.z, v[7] += hi.w;
                }
                if (lost)
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(0x7fffffffu);
                T* to = static_cast<T*>(p.out) + row * p.ld + int64_t(n) * 128 + col;
                if (left >= 8) {
                    if constexpr (sizeof(T) == 2) {
                        *reinterpret_cast<uint4*>(to) = make_uint4(bf16x2_of(v[0], v[1]), bf16x2_of(v[2], v[3]), bf16x2_of(v[4], v[5]), bf16x2_of(v[6], v[7]));
                    } else {
                        reinterpret_cast<float4*>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
                        reinterpret_cast<float4*>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i < left) to[i] = T(v[i]);
                }
            }
        }
        __syncwarp();
        cluster_barrier();  // the others have read this block's part
    }
    if (warp == 2) {
        tensor_fence_after();
        tensor_free<PAIR>(tensor, 2 * kSide);
    }
}

template <bool PAIR, bool READY, class T>
int launch(const Args& p, const Maps& maps, cudaStream_t s) {
    using S = Shape<READY>;
    constexpr size_t kShared = S::kShared;
    constexpr unsigned kThreads = S::kThreads;
    void (*const kernel)(Maps, Args) = weight_grad_kernel<PAIR, READY, T>;
    int st = allow_shared(reinterpret_cast<const void*>(kernel), kShared), registers = 0;
    if (st == PVQ_OK && !READY) {
        st = registers_of(reinterpret_cast<const void*>(kernel), &registers);
        if (st == PVQ_OK && registers < kRegisters) st = PVQ_ERR_UNSUPPORTED;
    }
    if (st != PVQ_OK) return st;
    const int team = PAIR ? 2 : p.split, teams = p.split > 1 || p.tiles < kSms / team ? p.tiles : kSms / team;
    return launch_early(kernel, dim3(static_cast<unsigned>(teams * team)), kThreads, kShared, team, s, maps, p);
}

// Tiles of 128 x 128 where one round of them does it, else pairs of thread blocks with 256 x 256.  1024 x 2304 over 4096 tokens (144
// tiles) 33.0 us and 32.9 in pairs, 1024 x 1152 (72 tiles in two parts) 24.4 and 32.7, 1024 x 2560 (160 tiles) 58.2 and 34.6.
int64_t small_tiles(int64_t inner, int64_t outer) { return ((outer + 127) / 128) * ((inner + 127) / 128); }
bool one_round(int64_t inner, int64_t outer) { return small_tiles(inner, outer) <= kSms; }

// x as bf16 in the caller's workspace.
int64_t workspace_ld(int64_t cols) { return (cols + 7) / 8 * 8; }
// Converting first, or in the kernel, tokens x inputs to outputs: 512 x 4096 to 4096 24.5 and 26.1 us, 1024 x 4096 to 14336 107 and 134,
// 4096 x 4096 to 1024 34.0 and 37.3; 2048 x 4096 to 1024 21.1 and 22.8; 4096 x 1024 to 2560 28.5 and 34.0; but
// 1001 x 4096 to 1024 14.6 and 13.4 (with the second launch), 4096 x 8192 to 512 44.4 and 39.0.
bool worth_a_workspace(int64_t rows, int64_t inner, int64_t outer) {
    return outer >= 1024 && !one_round(inner, outer) && static_cast<double>(rows) * inner * outer >= 8.0e9;
}

// Parts of t for as many tiles of 128 x 128: as many as run at once in clusters, with two runs each.  (512 x 512 over 16384 tokens,
// 16 tiles: 36 us in four parts, 49 in eight, of which 15 clusters run at once, 109 in one.)
template <class T>
int parts(int64_t tiles, int64_t stages, int* split) {
    const void* kernel = reinterpret_cast<const void*>(weight_grad_kernel<false, false, T>);
    *split = 1;
    for (int next = 2; next <= 8 && stages >= 2 * kRun * next; next *= 2) {
        int clusters = 0, st = allow_shared(kernel, Shape<false>::kShared);
        if (st == PVQ_OK) st = clusters_of(kernel, Shape<false>::kThreads, Shape<false>::kShared, next, &clusters);
        if (st != PVQ_OK) return st;
        if (tiles > clusters) break;
        *split = next;
    }
    return PVQ_OK;
}

template <class T>
int weight_grad_of(Args p, const void* dy, int64_t ld_dy, void* workspace, cudaStream_t s) {
    const int64_t pairs = ((p.outer + 255) / 256) * ((p.x.cols + 255) / 256), tiles = small_tiles(p.x.cols, p.outer);
    const int64_t stages = (p.x.rows + kDepth - 1) / kDepth;
    if (tiles >= int64_t(1) << 30) return PVQ_ERR_UNSUPPORTED;
    Maps maps;
    const Element out = sizeof(T) == 2 ? Element::kBf16 : Element::kF32;
    int st = tile_map(&maps.dy, dy, Element::kBf16, p.x.rows, p.outer, ld_dy, 64, kDepth);
    if (st == PVQ_OK) st = tile_map(&maps.x, p.x.codes, Element::kByte, p.x.rows, p.x.cols, p.x.ld_codes, 128, kDepth);
    if (st == PVQ_OK) st = tile_map(&maps.out, p.out, out, p.outer, p.x.cols, p.ld, 128 / sizeof(T), 32);
    if (st != PVQ_OK) return st;
    p.split = 1, p.after = -1;
    if (one_round(p.x.cols, p.outer)) {
        p.tiles = static_cast<int>(tiles);
        st = parts<T>(tiles, stages, &p.split);
        return st != PVQ_OK ? st : launch<false, false, T>(p, maps, s);
    }
    // The last round of tiles, where it is a small one, is shared by all SMs, in quarters and with t in parts, where a round is
    // long or one of two: 16384 values of t, 896 tiles (8 in the last round) 1446 us instead of 1500, 80 tiles 171 instead of 192, 4096
    // values and 80 tiles 50 instead of 54; but 4096 values and 448 tiles (4 in the last) 211 instead of 198: the launch behind
    // the others, while a few tiles alone run at a higher clock.
    constexpr int kPairs = kSms / 2;
    const int last = static_cast<int>(pairs % kPairs);
    int split = 1;
    if (last > 0) st = parts<T>(4 * last, stages, &split);
    if (st != PVQ_OK) return st;
    const bool shared = pairs > last && last > 0 && split > 1 && (stages >= 128 || pairs < 2 * kPairs);
    p.tiles = static_cast<int>(shared ? pairs - last : pairs);
    if (workspace) {
        const int64_t ld = workspace_ld(p.x.cols);
        Maps ready = maps;
        st = dequantize(p.x, workspace, true, ld, s);
        if (st == PVQ_OK) st = tile_map(&ready.x, workspace, Element::kBf16, p.x.rows, p.x.cols, ld, 64, kDepth);
        if (st == PVQ_OK) st = launch<true, true, T>(p, ready, s);
    } else {
        st = launch<true, false, T>(p, maps, s);
    }
    if (st != PVQ_OK || !shared) return st;
    p.after = p.tiles;
    p.tiles = 4 * last;
    p.split = split;
    return launch<false, false, T>(p, maps, s);
}

}  // namespace

size_t weight_grad_workspace(int64_t rows, int64_t inner, int64_t outer) {
    return worth_a_workspace(rows, inner, outer) ? static_cast<size_t>(rows) * workspace_ld(inner) * 2 : 0;
}

int weight_grad(const void* dy, int64_t outer, int64_t ld_dy, const Matrix& x, void* out, bool bf16, int64_t ld, void* workspace, uint32_t* status,
                cudaStream_t s) {
    const Args p{x, out, outer, ld, status, 1, 0, -1};
    if (!worth_a_workspace(x.rows, x.cols, outer)) workspace = nullptr;
    return bf16 ? weight_grad_of<__nv_bfloat16>(p, dy, ld_dy, workspace, s) : weight_grad_of<float>(p, dy, ld_dy, workspace, s);
}

}  // namespace fp8
}  // namespace pvq
