// Which kernel does an attention call, over how many thread blocks; and what adds the parts of items that several blocks shared.
#include "fp8_attention.cuh"

namespace pvq {
namespace fp8 {
namespace {

constexpr int kJoinRows = 4;  // of a block, one a warp

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

// Rows of an item, and thread blocks, for a call of this size.
struct Form {
    int rows, blocks;
};
Form form_of(int64_t seqs, int64_t rows, int heads, int kv_heads) {
    const int64_t each = (rows * (heads / kv_heads) + seqs - 1) / seqs;  // of a sequence and head
    if (each > 32) return {256, kSms};
    return {each <= 4 ? 4 : (each <= 8 ? 8 : (each <= 16 ? 16 : 32)), 2 * kSms};
}

size_t bytes_of(const Form& f) { return f.blocks * (2 * size_t(f.rows) * (128 + 2) * sizeof(float) + sizeof(PartHead)); }

template <int ROWS>
int join(const AttentionArgs& a, int blocks, cudaStream_t s) {
    return launch_early(attention_join_kernel<ROWS>, dim3(static_cast<unsigned>(blocks), ROWS >= 64 ? 8 : (ROWS + kJoinRows - 1) / kJoinRows), 32 * kJoinRows, 0, 0, s, a);
}

}  // namespace

size_t attention_workspace(int64_t seqs, int64_t rows, int heads, int kv_heads) { return bytes_of(form_of(seqs, rows, heads, kv_heads)); }

int attention(const AttentionArgs& call, cudaStream_t s) {
    AttentionArgs a = call;
    const int64_t seqs = a.step.seqs, rows = a.step.rows;
    const Form f = form_of(seqs, rows, a.heads, a.cache.heads);
    // (items of all sequences, each of at most as many tiles as a table holds)
    const int64_t items = rows * a.group / f.rows + seqs, tiles = ((int64_t(a.step.width) << a.cache.page_shift) + kTile - 1) / kTile;
    if (items * a.cache.heads >= int64_t(1) << 31 || items * a.cache.heads * tiles >= int64_t(1) << 31) return PVQ_ERR_UNSUPPORTED;
    a.by_group = division_by(a.group);
    const int threads = 128;  // (the least of a kernel's: a sequence's lanes for all of them, where there are few)
    a.plan_lanes = 1;
    while (a.plan_lanes < 32 && seqs * a.plan_lanes * 2 <= threads && rows * a.group > f.rows * seqs * a.plan_lanes) a.plan_lanes *= 2;
    int st = f.rows == 256 ? attention_many(a, f.blocks, s) : attention_few(a, f.rows, f.blocks, s);
    if (st != PVQ_OK) return st;
    if (f.rows == 4) return join<4>(a, f.blocks, s);
    if (f.rows == 8) return join<8>(a, f.blocks, s);
    if (f.rows == 16) return join<16>(a, f.blocks, s);
    return f.rows == 32 ? join<32>(a, f.blocks, s) : join<256>(a, f.blocks, s);
}

}  // namespace fp8
}  // namespace pvq
