// What the kernels of the 8-bit key and value cache share: the cache and a step over it as they see them.
#pragma once
#include "fp8_mma.cuh"

namespace pvq {
namespace fp8 {

constexpr int kLeastScale = 87, kMostScale = 167;  // bytes of a page's scale: 2^-40 and 2^40
constexpr int kTile = 128;                         // tokens that attention takes at a time; whole pages

// Codes [page][head][token of the page][dim] and scales [page][head], keys and values apart but laid out alike.
struct Cache {
    uint8_t *k, *v, *k_scales, *v_scales;
    int64_t page_step, head_step, token_step, scale_step;  // bytes
    int pages, heads, page_shift, dim;                     // tokens of a page: 1 << page_shift
};

// The new tokens of a step: rows starts[s] to starts[s + 1] are sequence s's last ones (without starts: row s is its last).
struct Step {
    const int *table, *lengths, *starts;
    int64_t ld;
    int width, seqs, rows;
};

struct Sequence {
    int row, n;  // first row and their number
    int first;   // position of the first; negative where the sequence is said to be shorter than its rows
    int held;    // tokens that its pages can hold of its length
};
__device__ __forceinline__ Sequence sequence_of(const Step& p, int s, int page_shift) {
    Sequence q;
    const int length = max(__ldg(p.lengths + s), 0);
    if (p.starts) {
        q.row = min(max(__ldg(p.starts + s), 0), p.rows);
        q.n = min(max(__ldg(p.starts + s + 1), q.row), p.rows) - q.row;
    } else {
        q.row = s;
        q.n = 1;
    }
    q.first = length - q.n;
    q.held = min(length, p.width << page_shift);
    return q;
}

// The exponent byte of a page whose largest finite magnitude has the bits `amax`: as scale_byte, from 2^-40 to 2^40; zeros
// get the smallest, so that what comes behind them decides.
__device__ __forceinline__ int page_scale_byte(uint32_t amax) {
    const int e = static_cast<int>((amax + 0x1fffffu) >> 23) - 8;
    return min(max(e, kLeastScale), kMostScale);
}

// launches
struct Rows {  // [row][head][dim] of values, steps in elements
    void *k, *v;
    int64_t k_row, k_head, v_row, v_head;
};
int cache_write(const Cache& c, const Step& p, const Rows& x, bool bf16, uint32_t* status, cudaStream_t s);
int cache_read(const Cache& c, const Step& p, const Rows& x, bool bf16, uint32_t* status, cudaStream_t s);

struct AttentionArgs {
    Cache cache;
    Step step;
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    float* lse;  // [row][head], or null
    int64_t q_row, q_head, out_row, out_head;
    int heads, group;  // of queries; of them a head of the cache
    Division by_group;
    int plan_lanes;    // that add up a sequence's work: a power of two up to 32
    int split;         // of few rows: blocks of a cluster that an item is shared by; 0: shares of all items' work
    int causal, window;
    float scale;  // of the scores, times log2 e
    uint32_t* status;
    float* workspace;
};
size_t attention_workspace(const Cache& c, const Step& p, int heads);
int attention(const AttentionArgs& a, cudaStream_t s);

}  // namespace fp8
}  // namespace pvq
