// The instructions of the tensor-core kernels: barriers, tiled copies, tensor memory, matrix products.
#pragma once
#include <cuda.h>

#include "fp8_internal.cuh"

namespace pvq {
namespace fp8 {

__device__ __forceinline__ uint32_t shared_address(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// ---- barriers in shared memory

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void barrier_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// The address of `a` in the shared memory of the cluster's thread block `rank`.
__device__ __forceinline__ uint32_t address_in(uint32_t a, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
    return r;
}
// An arrival at another block's barrier, whose threads wait for it with the cluster's scope.  It orders no memory by
// itself.  Reads and writes of tensor memory are ordered by tensor_fence_before in front of it and tensor_fence_after behind the
// wait; writes to the block's own shared memory by release_shared in front of it.  (A release of all memory to the cluster waits for
// every access of the SM's, a thousand cycles with global loads in flight, whichever thread asks for it: training product 957 us and
// 804 so, weight gradient of 512 tokens, 8192 x 4096, 72 us and 40.)
__device__ __forceinline__ void barrier_arrive_in(uint32_t cluster_address) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_address) : "memory");
}
__device__ __forceinline__ void release_shared() { asm volatile("fence.release.sync_restrict::shared::cta.cluster;" ::: "memory"); }

__device__ __forceinline__ void store_in(uint32_t cluster_address, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_address), "r"(v) : "memory");
}

constexpr int kPolls = 1 << 20;     // of a wait; a poll itself may wait for some time
constexpr int kLandings = 1 << 14;  // of a wait for what is in flight, once another wait has run out

// What a block, or a cluster whose blocks wait for one another, shares about waits that ran out: one that does ends all others, and
// sets the status word.
struct Bounds {
    volatile int* over;
    uint32_t* status;
    uint32_t blocks = 1;  // that are told
    int polls = kPolls;
};
__device__ __forceinline__ void ran_out(volatile int* over, uint32_t* status, uint32_t blocks) {
    if (blocks == 1) {
        *over = 1;
    } else {
#pragma unroll 1
        for (uint32_t r = 0; r < blocks; ++r) store_in(address_in(shared_address(const_cast<const int*>(over)), r), 1);
    }
    if (status) atomicOr(status, PVQ_STATUS_STAGING_TIMEOUT);
}
// The bounds-checked build leaves copies or scales out where the caller's status word says so, and then waits for a short while only.
struct Withheld {
    bool copies = false, scales = false;  // from the block's stage `kWithheldFrom` behind the ring's first turn on
};
constexpr uint32_t kWithheldFrom = 2;
__device__ __forceinline__ Withheld withheld_of(Bounds& b, uint32_t rank) {
    Withheld w;
#ifdef PVQ_DEBUG
    const uint32_t bits = b.status ? *const_cast<const volatile uint32_t*>(b.status) : 0u;
    w.copies = (bits & PVQ_DEBUG_WITHHOLD) != 0u || ((bits & PVQ_DEBUG_WITHHOLD_SECOND) != 0u && (rank & 1u));
    w.scales = (bits & PVQ_DEBUG_WITHHOLD_SCALES) != 0u;
    if (bits & (PVQ_DEBUG_WITHHOLD | PVQ_DEBUG_WITHHOLD_SECOND | PVQ_DEBUG_WITHHOLD_SCALES)) b.polls = 1 << 10;
#endif
    return w;
}
// Whether the phase `parity` is over, after a short wait.  CLUSTER: what another block of the cluster did to shared memory before it
// arrived (or its copies and products, which do so themselves) is seen from here on.  (Acquiring all memory would empty the L1 cache
// at each poll, from which the scales are read: a product of 1999 x 4096 by 4096 39.9 us and 34.4 so.)
template <bool CLUSTER = false>
__device__ __forceinline__ bool barrier_passed(uint32_t bar, uint32_t parity) {
    uint32_t done;
    if (CLUSTER)
        asm volatile(
            "{\n\t"
            ".reg .pred p;\n\t"
            "mbarrier.try_wait.parity.relaxed.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "fence.acquire.sync_restrict::shared::cluster.cluster;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t"
            "}"
            : "=r"(done)
            : "r"(bar), "r"(parity)
            : "memory");
    else
        asm volatile(
            "{\n\t"
            ".reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t"
            "}"
            : "=r"(done)
            : "r"(bar), "r"(parity)
            : "memory");
    return done;
}
// Waits for the phase `parity` (a new barrier counts as past the phase before its first, of parity 1); false when that took too
// long here or in another thread.
template <bool CLUSTER = false>
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, const Bounds& b) {
#pragma unroll 1
    for (int i = 0; i < b.polls; ++i) {
        if (barrier_passed<CLUSTER>(bar, parity)) return true;
        if ((i & 63) == 63 && *b.over) return false;
    }
    ran_out(b.over, b.status, b.blocks);
    return false;
}

// Whether the phase is over, without waiting.  (The thread that issues the products asks this of the next stage before it issues
// this one's: an answer takes 150 to 200 cycles, also where it is yes.  1999 x 4096 by 4096 31.4 us without, 29.7 with.)
template <bool CLUSTER = false>
__device__ __forceinline__ bool barrier_over(uint32_t bar, uint32_t parity) {
    uint32_t done;
    if (CLUSTER)
        asm volatile(
            "{\n\t"
            ".reg .pred p;\n\t"
            "mbarrier.test_wait.parity.relaxed.cluster.shared::cta.b64 p, [%1], %2;\n\t"
            "fence.acquire.sync_restrict::shared::cluster.cluster;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t"
            "}"
            : "=r"(done)
            : "r"(bar), "r"(parity)
            : "memory");
    else
        asm volatile(
            "{\n\t"
            ".reg .pred p;\n\t"
            "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t"
            "}"
            : "=r"(done)
            : "r"(bar), "r"(parity)
            : "memory");
    return done;
}

// The same for a whole warp, which has time: it sleeps between its polls (8 or 12 warps that poll without a pause cost the weight
// gradient 6%).
template <bool CLUSTER = false>
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, const Bounds& b) {
#pragma unroll 1
    for (int i = 0; i < b.polls; ++i) {
        if (__all_sync(0xffffffffu, barrier_passed<CLUSTER>(bar, parity))) return true;
        if ((i & 63) == 63 && __any_sync(0xffffffffu, *b.over)) return false;
        __nanosleep(40);
    }
    if ((threadIdx.x & 31) == 0) ran_out(b.over, b.status, b.blocks);
    __syncwarp();
    return false;
}

// One thread of the warp, all of which call it.  What it does alone has to be under this, not under a comparison of lanes: the
// products' operands are then known to be the same for all threads that are there (256 x 256 x 128 of a product: 368 ns, under a
// comparison 465).
__device__ __forceinline__ bool elected() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0u;
}

// A ring's place and the parity of its turn.
template <int SIZE>
struct Turn {
    uint32_t at = 0, parity = 0;
    __device__ __forceinline__ void next() {
        if (++at == SIZE) at = 0, parity ^= 1;
    }
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// Every thread of every block of the cluster.
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

// Its two halves; the first may be long before the second.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

// ---- copies of tiles

// Box at (x, y) of a matrix to shared memory; PAIR: the barrier may be that of the pair's other block.
template <bool PAIR>
__device__ __forceinline__ void load_tile(uint32_t to, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if (PAIR)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(to),
                     "l"(map), "r"(x), "r"(y), "r"(bar)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(to), "l"(map),
                     "r"(x), "r"(y), "r"(bar)
                     : "memory");
}
__device__ __forceinline__ void store_tile(const CUtensorMap* map, int x, int y, uint32_t from) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(from) : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int PENDING>
__device__ __forceinline__ void store_wait_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PENDING) : "memory");
}
__device__ __forceinline__ void store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// Writes to shared memory, before a copy or a product reads them.
__device__ __forceinline__ void async_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

// ---- tensor memory (an address: the lane in the upper half, the column in the lower one)

template <bool PAIR>
__device__ __forceinline__ void tensor_alloc(uint32_t to, uint32_t columns) {  // one warp (of each block of a pair)
    if (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}
template <bool PAIR>
__device__ __forceinline__ void tensor_free(uint32_t at, uint32_t columns) {
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
__device__ __forceinline__ void tensor_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tensor_wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// A lane's values of 16 or 32 columns; `at` is at the warp's own quarter of the lanes.
__device__ __forceinline__ void tensor_load(uint32_t at, float (&v)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,"
        "%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
          "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at));
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tensor_load(uint32_t at, float (&v)[16]) {
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at));
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
// A lane's words of 1, 2, 4, 8 or 16 columns.
__device__ __forceinline__ void tensor_store(uint32_t at, const uint32_t (&w)[1]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(at), "r"(w[0]) : "memory");
}
__device__ __forceinline__ void tensor_store(uint32_t at, const uint32_t (&w)[2]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x2.b32 [%0], {%1, %2};" ::"r"(at), "r"(w[0]), "r"(w[1]) : "memory");
}
__device__ __forceinline__ void tensor_store(uint32_t at, const uint32_t (&w)[4]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
}
__device__ __forceinline__ void tensor_store(uint32_t at, const uint32_t (&w)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                 "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}

__device__ __forceinline__ void tensor_store(uint32_t at, const uint32_t (&w)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                 "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "r"(w[8]), "r"(w[9]), "r"(w[10]), "r"(w[11]), "r"(w[12]), "r"(w[13]), "r"(w[14]), "r"(w[15])
                 : "memory");
}

// ---- products

// Operand in shared memory, rows of 128 bytes swizzled as a tiled copy leaves them, eight rows a kilobyte.  Along k (8 rows
// are 8 values of the other index), or across it (8 rows are 8 values of k; `further`: bytes to the next 128 across).
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t further = 16) {
    return static_cast<uint64_t>((at & 0x3ffffu) >> 4) | static_cast<uint64_t>(further >> 4) << 16 | static_cast<uint64_t>(1024u >> 4) << 32 |
           uint64_t(1) << 46 | uint64_t(2) << 61;
}
// Types, orders and sizes of a product, as the instruction takes them.
__host__ __device__ constexpr uint32_t product_bf16(int m, int n, bool a_across, bool b_across) {
    return 1u << 4 | 1u << 7 | 1u << 10 | uint32_t(a_across) << 15 | uint32_t(b_across) << 16 | uint32_t(n / 8) << 17 | uint32_t(m / 16) << 24;
}
// (e4m3 twice, scales e8m0; `part`: which byte of the scales' words)
__host__ __device__ constexpr uint32_t product_e4m3(int m, int n, bool a_across, bool b_across) {
    return uint32_t(a_across) << 15 | uint32_t(b_across) << 16 | uint32_t(n / 8) << 17 | 1u << 23 | uint32_t(m / 16) << 24;
}
__device__ __forceinline__ uint32_t with_part(uint32_t product, uint32_t part) { return product | part << 4 | part << 29; }

template <bool PAIR>
__device__ __forceinline__ void multiply_e4m3(uint32_t d, uint64_t a, uint64_t b, uint32_t product, uint32_t scales_a, uint32_t scales_b, bool add) {
    if (PAIR)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(product), "r"(scales_a), "r"(scales_b), "r"(static_cast<uint32_t>(add))
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(product), "r"(scales_a), "r"(scales_b), "r"(static_cast<uint32_t>(add))
            : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void multiply_bf16(uint32_t d, uint64_t a, uint64_t b, uint32_t product, bool add) {
    if (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                     "r"(product), "r"(static_cast<uint32_t>(add))
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                     "r"(product), "r"(static_cast<uint32_t>(add))
                     : "memory");
}
// Arrives at the barrier (PAIR: of both blocks) once all products issued so far are done.
template <bool PAIR>
__device__ __forceinline__ void products_done(uint32_t bar) {
    if (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(uint16_t(3)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// ---- registers: a warpgroup's share, a thread, of those that the block was launched with

template <int REGISTERS>
__device__ __forceinline__ void more_registers() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGISTERS));
}
template <int REGISTERS>
__device__ __forceinline__ void fewer_registers() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGISTERS));
}

// ---- once a wait has run out

// Waits for the last copies that were asked for, `issued` stages of a ring in all.
template <int STAGES, bool CLUSTER = false>
__device__ __forceinline__ void land(uint32_t full, uint32_t issued) {
#pragma unroll 1
    for (uint32_t i = issued > STAGES ? issued - STAGES : 0; i < issued; ++i)
#pragma unroll 1
        for (int polls = 0; polls < kLandings && !barrier_passed<CLUSTER>(full + 8 * (i % STAGES), (i / STAGES) & 1); ++polls) {}
}
// What was not computed becomes NaN: a warp's 32 rows, a lane's own, of `width` columns.
template <class T>
__device__ __forceinline__ void spoil(T* out, int64_t ld, int64_t row, int64_t rows, int64_t col, int64_t cols, int width) {
    row += threadIdx.x & 31;
    if (row >= rows) return;
#pragma unroll 1
    for (int i = 0; i < width && col + i < cols; ++i) out[row * ld + col + i] = T(__uint_as_float(0x7fffffffu));
}

// ---- scales in tensor memory

// Four blocks' scale bytes along k for one index across it, as the product takes them: block 4 * four + i in byte i.
// Blocks behind the end, and indices behind it, get 1 (their codes are zeros; a NaN would not be lost in them).
// ACROSS: the matrix is [k][index], in tiles.
template <bool ACROSS>
__device__ __forceinline__ uint32_t scale_word(const Matrix& m, int64_t index, int four) {
    if (ACROSS) {
        if (index >= m.cols) return 0x7f7f7f7fu;
        const int64_t down = (m.rows + kBlock - 1) / kBlock;
        uint32_t w = 0x7f7f7f7fu;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * four + i < down)
                w = (w & ~(0xffu << (8 * i))) | static_cast<uint32_t>(__ldg(m.scales + (4 * four + i) * m.ld_scales + index / kBlock)) << (8 * i);
        return w;
    }
    if (index >= m.rows) return 0x7f7f7f7fu;
    const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(m.scales + (index >> m.shift) * m.ld_scales + 4 * four));
    const int valid = m.blocks - 4 * four;
    return valid >= 4 ? w : (w & ((1u << (8 * valid)) - 1u)) | (0x7f7f7f7fu << (8 * valid));
}
// The words of WORDS * 32 indices from `first` (a multiple of 128): lane r holds those of r, r + 32, ...
template <bool ACROSS, int WORDS>
__device__ __forceinline__ void scale_words(const Matrix& m, int64_t first, int four, uint32_t (&w)[WORDS]) {
    const int lane = threadIdx.x & 31;
    if (ACROSS || m.shift) {  // one scale for 128 of them
#pragma unroll
        for (int j = 0; j < WORDS; ++j) {
            if (j % 4 == 0) w[j] = scale_word<ACROSS>(m, first + 32 * j, four);
            else w[j] = w[j - j % 4];
        }
    } else {
#pragma unroll
        for (int j = 0; j < WORDS; ++j) w[j] = scale_word<ACROSS>(m, first + 32 * j + lane, four);
    }
}

// ---- host side

// A map of a matrix for tiled copies, in boxes of `box_x` values (128 bytes) by `box_y` rows.
enum class Element { kByte, kBf16, kF32 };
int tile_map(CUtensorMap* map, const void* p, Element type, int64_t rows, int64_t cols, int64_t ld, int box_x, int box_y);
// Allows a kernel its shared memory, once a device.
int allow_shared(const void* kernel, size_t bytes);
// Clusters of `size` thread blocks that run at once: fewer than the SMs hold blocks, since a cluster's lie in one part of the GPU
// (of blocks that take an SM each: 74 of 2, 33 of 4, 15 of 8).
int clusters_of(const void* kernel, unsigned threads, size_t shared, unsigned size, int* clusters);
// Registers a thread that a kernel is launched with.
int registers_of(const void* kernel, int* registers);

}  // namespace fp8
}  // namespace pvq
