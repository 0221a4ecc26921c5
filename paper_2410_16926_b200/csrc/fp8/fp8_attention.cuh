// What the attention kernels over the 8-bit cache share: how the work is cut, the pages' way to shared memory, parts of results.
//
// An item is a block of a sequence's query rows (query heads of a cache's head side by side, query for query) over one head of the
// cache; its units are the tiles of 128 tokens that some row of it sees, behind what its beginning and end cost, in tiles (one at least).
// The units of all items in a row are cut into equal shares, one a thread block, whatever the sequences' lengths; an item that is cut leaves parts (sums that are not yet
// divided, and what their weights are relative to) in the workspace, which a second kernel adds in the order of the tokens.
#pragma once
#include "fp8_cache.cuh"

namespace pvq {
namespace fp8 {

struct CacheMaps {
    CUtensorMap k, v;
};

// What an item costs besides its tiles, in tiles: of 256 rows, queries made codes, the first scores, the results, 10 to 20 us by 2.2 a tile.  A causal
// prompt's first blocks of rows are items of few tiles; thread blocks that got many of them ended last.  32 heads over 8 of 128 dims, in us, with 0, 4, 6
// and 10: 8192 causal tokens 829, 655, 640, 651; 8 of 1024 238, 211, 209, 216; 4096 seen by all 333, 324, 324, 332.  Few rows begin in a tile's time: 0.
template <int ROWS>
__host__ __device__ constexpr int item_units() {
    return ROWS == 256 ? 6 : 0;
}
constexpr int kLeastTiles = 2;   // of a block
constexpr int kScaleSlots = 8;   // tiles whose scales are on their way
constexpr float kNone = -INFINITY;
constexpr float kLargest = 0x1.fffffep127f;

// A part: fp32 sums [rows][128], then what the weights are relative to (as an exponent of 2) and their sum, a row each.
template <int ROWS>
__host__ __device__ constexpr size_t part_floats() {
    return size_t(ROWS) * (128 + 2);
}
struct PartHead {  // of a block's second part: the item that is continued by the blocks behind it
    int parts, row, q0, rows, head;  // parts 0: there is none
};
// The workspace: two parts a block (of an item that began before, of one that goes on behind), then their heads.
template <int ROWS>
__device__ __forceinline__ PartHead* part_heads(const AttentionArgs& a) {
    return reinterpret_cast<PartHead*>(a.workspace + 2 * size_t(gridDim.x) * part_floats<ROWS>());
}
__device__ __forceinline__ float row_lse(float relative, float all) { return all == 0.0f ? kNone : (relative + log2f(all)) * 0.693147180559945f; }

struct Item {
    int s, head, block;
    Sequence q;
    int q0, rows;        // its rows of the sequence's n * group
    int lo, hi;          // positions that some row sees
    __device__ __forceinline__ int tile0() const { return lo / kTile; }  // of those
    __device__ __forceinline__ int tiles() const { return hi > lo ? (hi + kTile - 1) / kTile - tile0() : 0; }
    template <int ROWS>
    __device__ __forceinline__ int units() const {
        return max(item_units<ROWS>() + tiles(), 1);
    }
};

// The first position that a row at `position` (negative in front of its sequence) sees.
__device__ __forceinline__ int first_seen(const AttentionArgs& a, int position) { return a.window > 0 && position >= a.window ? position - a.window + 1 : 0; }

template <int ROWS>
__device__ __forceinline__ void measure(const AttentionArgs& a, Item& it) {
    it.q0 = it.block * ROWS;
    it.rows = min(ROWS, it.q.n * a.group - it.q0);
    const int i0 = divide(it.q0, a.by_group), i1 = divide(it.q0 + it.rows - 1, a.by_group);
    it.hi = a.causal ? min(it.q.held, it.q.first + i1 + 1) : it.q.held;
    it.lo = first_seen(a, it.q.first + i0);
}
template <int ROWS>
__device__ __forceinline__ int blocks_of(const AttentionArgs& a, const Sequence& q) {
    return (q.n * a.group + ROWS - 1) / ROWS;
}

// A block's share: it begins `skip` units into an item.  (All units are fewer than 2^31: the host sees to that for sequences that do not
// overlap.  Where starts descend nobody has a share.)
struct Share {
    int s, head, block, skip;
    int begin, left;
    int all, blocks;  // units, and blocks that have a share
};
// The block whose share unit u is in: shares differ by one at most, larger ones first.
__device__ __forceinline__ int share_of(uint32_t all, uint32_t blocks, uint32_t u) {
    const uint32_t each = all / blocks, larger = all % blocks, edge = larger * (each + 1);
    return u < edge ? u / (each + 1) : larger + (u - edge) / each;
}
struct PlanShared {
    int sums[32], left, per_head, s;
    Sequence q;  // of the sequence that the share begins in
    Share share;
};

// All threads of the block; `keeper` is the one that will ask Walk::parts.
template <int THREADS, int ROWS>
__device__ __forceinline__ Share find_share(const AttentionArgs& a, PlanShared& sh, int keeper) {
    const int thread = threadIdx.x, lane = thread & 31, warp = thread >> 5, seqs = a.step.seqs;
    const int lanes = a.plan_lanes, per = THREADS / lanes;  // for a sequence; sequences at a time
    const bool leads = (thread & (lanes - 1)) == 0;
    int units = 0, of_head = 0, before = 0;
    bool descends = false;  // starts of some sequence so far
    Sequence q{};
    const auto chunk = [&](int first) {  // units of a sequence, and of those before it in the chunk; returns those of the chunk
        const int s = first + thread / lanes;
        units = 0;
        if (s < seqs) {
            Item it;
            it.q = sequence_of(a.step, s, a.cache.page_shift);
            if (a.status && blockIdx.x == 0 && it.q.n > 0 && (it.q.first < 0 || it.q.held < it.q.first + it.q.n)) atomicOr(a.status, PVQ_STATUS_BAD_PAGE);
            q = it.q;
            const int blocks = blocks_of<ROWS>(a, it.q);
            for (it.block = thread & (lanes - 1); it.block < blocks; it.block += lanes) {
                measure<ROWS>(a, it);
                units += it.units<ROWS>();
            }
        }
        for (int o = lanes >> 1; o > 0; o >>= 1) units += __shfl_xor_sync(0xffffffffu, units, o);
        of_head = units;
        units *= a.cache.heads;
        int sum = leads ? units : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int other = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += other;
        }
        if (first > 0) __syncthreads();
        if (lane == 31) sh.sums[warp] = sum;
        if (a.step.starts) descends |= __syncthreads_or(s < seqs && __ldg(a.step.starts + s + 1) < __ldg(a.step.starts + s));
        else __syncthreads();
        before = sum - (leads ? units : 0);
        int all = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) {
            const int here = sh.sums[w];
            before += w < warp ? here : 0;
            all += here;
        }
        return all;
    };
    Share r{};
    for (int first = 0; first < seqs; first += per) r.all = descends ? 0 : r.all + chunk(first);
    if (descends) {
        if (a.status && blockIdx.x == 0 && thread == 0) atomicOr(a.status, PVQ_STATUS_BAD_PAGE);
        r.all = 0;
    }
    r.blocks = min(static_cast<int>(gridDim.x), max(1, r.all / (item_units<ROWS>() + kLeastTiles)));
    const int c = blockIdx.x;
    if (r.all == 0 || c >= r.blocks) return r;
    const int each = static_cast<uint32_t>(r.all) / static_cast<uint32_t>(r.blocks), larger = r.all - each * r.blocks;
    r.begin = each * c + min(c, larger);
    r.left = each + (c < larger ? 1 : 0);
    int base = 0;
    if (seqs > per) __syncthreads();
    for (int first = 0; first < seqs && base <= r.begin; first += per) {
        const int here = seqs > per ? chunk(first) : r.all;
        if (leads && base + before <= r.begin && r.begin - base - before < units) {
            sh.s = first + thread / lanes;
            sh.left = r.begin - base - before;
            sh.per_head = of_head;
            sh.q = q;
        }
        base += here;
    }
    __syncthreads();
    r.s = sh.s;
    int rest = sh.left;
    const int per_head = sh.per_head;
    if (rest >= per_head) {
        r.head = static_cast<uint32_t>(rest) / static_cast<uint32_t>(per_head);
        rest -= r.head * per_head;
    }
    Item it;
    it.q = sh.q;
    const int blocks = blocks_of<ROWS>(a, it.q);
    for (int b0 = 0; b0 < blocks && blocks > 1; b0 += 32) {  // (every warp alike)
        it.block = b0 + lane;
        int sum = 0;
        if (it.block < blocks) {
            measure<ROWS>(a, it);
            sum = it.units<ROWS>();
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int other = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += other;
        }
        const uint32_t behind = __ballot_sync(0xffffffffu, it.block < blocks && sum > rest);
        if (behind) {
            const int at = __ffs(behind) - 1;
            r.block = b0 + at;
            if (at > 0) rest -= __shfl_sync(0xffffffffu, sum, at - 1);
            break;
        }
        rest -= __shfl_sync(0xffffffffu, sum, 31);
    }
    r.skip = rest;
    if (thread == keeper) sh.share = r;
    return r;
}

// Goes through a block's share, item by item.  Every role of the block does so by itself.
template <int ROWS>
struct Walk {
    const AttentionArgs& a;
    Item it;
    int left, skip, take;
    bool over = false;  // (of an item of a cluster's, which may leave a block no units)

    // Of one item, the units that are this block's of the cluster's `split`.
    __device__ __forceinline__ Walk(const AttentionArgs& args, int item, int rank, int split) : a(args), left(-1) {
        const uint32_t blocks = (a.group + ROWS - 1) / ROWS, each = a.cache.heads * blocks;  // (one row a sequence)
        it.s = item / each;
        const uint32_t rest = item - it.s * each;
        it.head = rest / blocks, it.block = rest - it.head * blocks;
        it.q = sequence_of(a.step, it.s, a.cache.page_shift);
        measure<ROWS>(a, it);
        const int units = it.template units<ROWS>();
        skip = units * rank / split;
        take = units * (rank + 1) / split - skip;
    }

    __device__ __forceinline__ Walk(const AttentionArgs& args, const Share& sh, const PlanShared& plan) : a(args), left(sh.left), skip(sh.skip), take(0) {
        if (left <= 0) return;
        it.s = sh.s, it.head = sh.head, it.block = sh.block;
        it.q = plan.q;
        measure<ROWS>(a, it);
        take = min(left, it.template units<ROWS>() - skip);
    }
    __device__ __forceinline__ bool there() const { return left > 0 || (left < 0 && !over); }
    // Tiles of this share (an item's other units are before them).
    __device__ __forceinline__ int before() const { return max(skip - item_units<ROWS>(), 0); }
    __device__ __forceinline__ int begin() const { return it.tile0() + before(); }
    __device__ __forceinline__ int count() const { return max(min(skip + take - item_units<ROWS>(), it.tiles()) - before(), 0); }
    __device__ __forceinline__ bool first() const { return skip == 0; }
    __device__ __forceinline__ bool last() const { return skip + take == it.template units<ROWS>(); }
    // Blocks that the item is shared by, from its first one on (called where first()).
    __device__ __forceinline__ int parts(const PlanShared& plan) const {
        return share_of(plan.share.all, plan.share.blocks, plan.share.begin + plan.share.left - left + it.template units<ROWS>() - 1) - blockIdx.x + 1;
    }
    __device__ __forceinline__ void next() {
        over = true;
        if (left < 0) return;
        left -= take;
        if (left <= 0) return;
        skip = 0;
        if (++it.block == blocks_of<ROWS>(a, it.q)) {
            it.block = 0;
            if (++it.head == a.cache.heads) {
                it.head = 0;
                do {
                    it.q = sequence_of(a.step, ++it.s, a.cache.page_shift);
                } while (it.q.n == 0 && it.s + 1 < a.step.seqs);
            }
        }
        measure<ROWS>(a, it);
        take = min(left, it.template units<ROWS>());
    }
};

// Where a row's result goes: its query's row and head.
struct RowPlace {
    int row, head;
};
__device__ __forceinline__ RowPlace place_of(const AttentionArgs& a, const Sequence& q, int head, int packed) {
    const int i = divide(packed, a.by_group);
    return {q.row + i, head * a.group + packed - i * a.group};
}

// The pages of a run of tiles, 32 at a time, a lane each: their numbers are asked for two turns ahead, their scales one (of the first
// turn by first_scales, behind the first copies).
struct Pages {
    const AttentionArgs& a;
    const int* table;
    int head, entry, end, id, id1, id2;
    uint32_t scales, scales1;

    __device__ __forceinline__ int ask(int e) const { return e < end ? __ldg(table + e) : -1; }
    __device__ __forceinline__ int known(int i, int e) const {  // -1: a page that is not there, zeros
        if (e >= end) return -1;
        if (i >= 0 && i < a.cache.pages) return i;
        if (a.status) atomicOr(a.status, PVQ_STATUS_BAD_PAGE);
        return -1;
    }
    __device__ __forceinline__ uint32_t ask_scales(int i) const {
        if (i < 0) return 127u | 127u << 8;
        const int64_t at = i * a.cache.scale_step + head;
        const int k = __ldg(a.cache.k_scales + at), v = __ldg(a.cache.v_scales + at);
        return static_cast<uint32_t>(min(max(k, kLeastScale), kMostScale)) | static_cast<uint32_t>(min(max(v, kLeastScale), kMostScale)) << 8;
    }
    __device__ __forceinline__ Pages(const AttentionArgs& args, const Item& it, int first_entry) : a(args) {
        table = a.step.table + it.s * a.step.ld;
        head = it.head;
        end = (it.q.held + (1 << a.cache.page_shift) - 1) >> a.cache.page_shift;
        entry = first_entry + (threadIdx.x & 31);
        id = ask(entry), id1 = ask(entry + 32), id2 = ask(entry + 64);
        id = known(id, entry);
    }
    __device__ __forceinline__ void first_scales() {
        scales = ask_scales(id);
        id1 = known(id1, entry + 32);
        scales1 = ask_scales(id1);
    }
    __device__ __forceinline__ void next() {
        entry += 32;
        id = id1, id1 = known(id2, entry + 32), id2 = ask(entry + 64);
        scales = scales1, scales1 = ask_scales(id1);
    }
};

// Waits as those of fp8_mma.cuh, whose polls are asked to take up to 20 us each: what a poll costs, others of the SM's quarter lack (a tile of
// 256 rows 2.23 us, so 2.16).
__device__ __forceinline__ bool passed_slowly(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 20000;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t"
        "}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done;
}
__device__ __forceinline__ bool thread_waits(uint32_t bar, uint32_t parity, const Bounds& b) {
#pragma unroll 1
    for (int i = 0; i < b.polls >> 6; ++i) {
        if (passed_slowly(bar, parity)) return true;
        if (*b.over) return false;
    }
    ran_out(b.over, b.status, b.blocks);
    return false;
}
__device__ __forceinline__ bool warp_waits(uint32_t bar, uint32_t parity, const Bounds& b) {
#pragma unroll 1
    for (int i = 0; i < b.polls >> 6; ++i) {
        if (__all_sync(0xffffffffu, passed_slowly(bar, parity))) return true;
        if (__any_sync(0xffffffffu, *b.over)) return false;
    }
    if ((threadIdx.x & 31) == 0) ran_out(b.over, b.status, b.blocks);
    __syncwarp();
    return false;
}

// In the bounds-checked build copies may be left out as in the products' kernels, and scales come late instead, each tile's by kLate ns, which
// the waits have time for: whoever does not wait for them reads those of another tile.
constexpr unsigned kLate = 10000;
__device__ __forceinline__ Withheld withheld_in(Bounds& b) {
    const Withheld w = withheld_of(b, blockIdx.x);
    if (w.scales && !w.copies) b.polls = kPolls;
    return w;
}

// One page of a head to shared memory.
__device__ __forceinline__ void load_page(uint32_t to, const CUtensorMap* map, int head, int page, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(to), "l"(map), "r"(0),
                 "r"(0), "r"(head), "r"(page), "r"(bar)
                 : "memory");
}

__device__ __forceinline__ float exp2_of(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// e4m3 operands without scales, sums in fp32.
__host__ __device__ constexpr uint32_t product_codes(int m, int n, bool a_across, bool b_across) {
    return 1u << 4 | uint32_t(a_across) << 15 | uint32_t(b_across) << 16 | uint32_t(n / 8) << 17 | uint32_t(m / 16) << 24;
}
__device__ __forceinline__ void multiply_codes(uint32_t d, uint64_t a, uint64_t b, uint32_t product, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                 "r"(product), "r"(static_cast<uint32_t>(add))
                 : "memory");
}

// A row's values times 2^-e, |values| at most 448, as two codes each: the nearest one, and the nearest one to what it leaves.
// Together they are a bf16 value but for 2^-17 of the row's largest.  (`apart`: a power of two by which the second code is larger than what it stands for.)
__device__ __forceinline__ void two_codes(float x, float y, uint32_t& hi, uint32_t& lo, float apart = 1.0f) {
    hi = codes_of(x, y);
    const float2 h = values_of(hi);
    lo = codes_of((x - h.x) * apart, (y - h.y) * apart);
}

// What a row's scores in codes are times, but for the key's scale.  Finite, so that a score of zero stays zero.
__device__ __forceinline__ float row_factor(uint32_t byte, float scale) { return fminf(scale_of(byte) * scale, kLargest); }

int cache_maps(const Cache& c, CacheMaps* maps);
int attention_few(const AttentionArgs& a, int rows, int blocks, cudaStream_t s);  // 4, 8, 16 or 32 rows an item
int attention_many(const AttentionArgs& a, int blocks, cudaStream_t s);           // 256

}  // namespace fp8
}  // namespace pvq
