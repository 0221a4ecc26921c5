// Which kernel does an attention call, over how many thread blocks; and what adds the parts of items that several blocks shared.
#include "fp8_attention.cuh"

namespace pvq {
namespace fp8 {
namespace {

constexpr int kJoinRows = 4;  // of a block, one a warp
// Clusters of single tokens' items: their blocks that run at once, two an SM (a cluster's lie in one part of the GPU: 33 of four and 15 of eight with
// one an SM), and the tiles of a block up to which they are taken.
constexpr int kAtOnce[] = {2 * kSms, 2 * kSms, 66 * 4, 30 * 8};  // of 1, 2, 4, 8
constexpr int kClusterTiles = 16;

// Block c of a group adds the item that block c of the attention was the first, but not the last, to work on.
template <int ROWS>
__global__ void __launch_bounds__(32 * kJoinRows) attention_join_kernel(const __grid_constant__ AttentionArgs p) {
    dependency_wait();
    launch_dependents();
    const PartHead head = part_heads<ROWS>(p)[blockIdx.x];
    const int lane = threadIdx.x & 31;
    const auto part = [&](int i) { return p.workspace + (2 * (int64_t(blockIdx.x) + i) + (i == 0 ? 1 : 0)) * part_floats<ROWS>(); };
    if (head.parts == 0) return;
    for (int n = blockIdx.y * kJoinRows + (threadIdx.x >> 5); n < head.rows; n += gridDim.y * kJoinRows) {
        float top = kNone;
        for (int i = lane; i < head.parts; i += 32) {
            const float m = part(i)[ROWS * 128 + n];
            top = m != m ? m : fmaxf(top, m);
            if (m != m) break;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const float other = __shfl_xor_sync(0xffffffffu, top, o);
            top = top != top ? top : (other != other ? other : fmaxf(top, other));
        }
        const float against = top == kNone ? 0.0f : top;
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        float all = 0.0f;
        for (int i0 = 0; i0 < head.parts; i0 += 32) {
            float less = 0.0f, weights = 0.0f;
            if (i0 + lane < head.parts) {
                less = exp2_of(part(i0 + lane)[ROWS * 128 + n] - against);
                weights = part(i0 + lane)[ROWS * 129 + n];
            }
            const int here = min(32, head.parts - i0);
#pragma unroll 4
            for (int i = 0; i < here; ++i) {
                const float f = __shfl_sync(0xffffffffu, less, i), w = __shfl_sync(0xffffffffu, weights, i);
                float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);  // (behind the dims there may be anything)
                if (lane * 4 < p.cache.dim) v = *reinterpret_cast<const float4*>(part(i0 + i) + n * 128 + lane * 4);
                sum.x = fmaf(v.x, f, sum.x), sum.y = fmaf(v.y, f, sum.y), sum.z = fmaf(v.z, f, sum.z), sum.w = fmaf(v.w, f, sum.w);
                all = fmaf(w, f, all);
            }
        }
        const int packed = head.q0 + n, query = divide(packed, p.by_group);
        const int64_t row = head.row + query;
        const int q_head = head.head * p.group + packed - query * p.group;
        const float one = all == 0.0f ? 0.0f : 1.0f / all;
        if (lane * 4 < p.cache.dim)
            *reinterpret_cast<uint2*>(p.out + row * p.out_row + q_head * p.out_head + lane * 4) =
                make_uint2(bf16x2_of(sum.x * one, sum.y * one), bf16x2_of(sum.z * one, sum.w * one));
        if (p.lse && lane == 0) p.lse[row * p.heads + q_head] = row_lse(top, all);
    }
}

// Rows of an item, thread blocks, and how many of them make a cluster that shares an item (0: all share all work).
struct Form {
    int rows, blocks, split;
};
// By the mean: lengths and starts are on the device.  A step of both kinds takes one kernel's time for the other's work (255 single tokens behind 4096
// and a prompt of 4096 1461 us, apart 328 and 222).
Form form_of(const Cache& c, const Step& p, int heads) {
    const int group = heads / c.heads;
    const int64_t each = (int64_t(p.rows) * group + p.seqs - 1) / p.seqs;  // rows of a sequence and head
    if (each > 32) return {256, kSms, 0};
    Form f{each <= 4 ? 4 : (each <= 8 ? 8 : (each <= 16 ? 16 : 32)), 2 * kSms, 0};
    // Single tokens of few sequences whose tables are short: an item for a cluster, whose blocks find their work without a scan and join it without
    // a second kernel.  8 heads, in us, so and with shares: one sequence of 100 tokens 4.6 and 10.3, of 1000 6.2 and 9.5, of 16000 17.2 and 21.8; 37 of 2000
    // (one block an item) 28.8 and 31.4, of a quarter of that and up 21.3 and 25.5; 4 of 8000 20.0 and 18.3.
    const int64_t items = int64_t(p.seqs) * c.heads, tiles = ((int64_t(p.width) << c.page_shift) + kTile - 1) / kTile;
    if (!p.starts && f.rows <= 16 && items <= kAtOnce[0]) {
        int log = 0;
        while (log < 3 && (1 << log) < tiles && items << (log + 1) <= kAtOnce[log + 1]) ++log;
        if (tiles <= int64_t(kClusterTiles) << log) f.split = 1 << log, f.blocks = static_cast<int>(items) << log;
    }
    return f;
}

size_t bytes_of(const Form& f) { return f.split ? 0 : f.blocks * (2 * size_t(f.rows) * (128 + 2) * sizeof(float) + sizeof(PartHead)); }

template <int ROWS>
int join(const AttentionArgs& a, int blocks, cudaStream_t s) {
    return launch_early(attention_join_kernel<ROWS>, dim3(static_cast<unsigned>(blocks), ROWS >= 64 ? 8 : (ROWS + kJoinRows - 1) / kJoinRows), 32 * kJoinRows, 0, 0, s, a);
}

}  // namespace

size_t attention_workspace(const Cache& c, const Step& p, int heads) { return bytes_of(form_of(c, p, heads)); }

int attention(const AttentionArgs& call, cudaStream_t s) {
    AttentionArgs a = call;
    const int64_t seqs = a.step.seqs, rows = a.step.rows;
    const Form f = form_of(a.cache, a.step, a.heads);
    a.split = f.split;
    // (items of all sequences, each of at most as many tiles as a table holds, and its other units)
    const int64_t items = rows * a.group / f.rows + seqs, units = ((int64_t(a.step.width) << a.cache.page_shift) + kTile - 1) / kTile + (f.rows == 256 ? item_units<256>() : 1);
    if (items * a.cache.heads >= int64_t(1) << 31 || items * a.cache.heads * units >= int64_t(1) << 31) return PVQ_ERR_UNSUPPORTED;
    a.by_group = division_by(a.group);
    const int threads = 128;  // (the least of a kernel's: a sequence's lanes for all of them, where there are few)
    a.plan_lanes = 1;
    while (a.plan_lanes < 32 && seqs * a.plan_lanes * 2 <= threads && rows * a.group > f.rows * seqs * a.plan_lanes) a.plan_lanes *= 2;
    int st = f.rows == 256 ? attention_many(a, f.blocks, s) : attention_few(a, f.rows, f.blocks, s);
    if (st != PVQ_OK || f.split) return st;
    if (f.rows == 4) return join<4>(a, f.blocks, s);
    if (f.rows == 8) return join<8>(a, f.blocks, s);
    if (f.rows == 16) return join<16>(a, f.blocks, s);
    return f.rows == 32 ? join<32>(a, f.blocks, s) : join<256>(a, f.blocks, s);
}

}  // namespace fp8
}  // namespace pvq
