// The entry points of the 8-bit cache: argument checks, then the launches.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <limits>

#include "fp8_cache.cuh"

using namespace pvq;

namespace {

constexpr int64_t kFar = int64_t(1) << 40;  // a step of a tiled copy ends here

int checked(const pvq_fp8_cache* c, fp8::Cache* out) {
    if (!c || !c->d_k || !c->d_v || !c->d_k_scales || !c->d_v_scales) return PVQ_ERR_INVALID_ARG;
    if (c->pages < 1 || c->heads < 1 || c->dim < 1 || c->page < 1) return PVQ_ERR_INVALID_ARG;
    if (c->page_step < c->dim || c->head_step < c->dim || c->token_step < c->dim || c->scale_step < c->heads) return PVQ_ERR_INVALID_ARG;
    if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return PVQ_ERR_UNSUPPORTED;
    if (c->dim % 16 != 0 || c->dim > 128 || c->pages >= int64_t(1) << 31 || c->heads >= 1 << 16) return PVQ_ERR_UNSUPPORTED;
    if (c->page_step >= kFar || c->head_step >= kFar || c->token_step >= kFar || c->scale_step >= kFar) return PVQ_ERR_UNSUPPORTED;
    if (!is_aligned(c->d_k, 16) || !is_aligned(c->d_v, 16) || c->page_step % 16 != 0 || c->head_step % 16 != 0 || c->token_step % 16 != 0)
        return PVQ_ERR_ALIGNMENT;
    int shift = 4;
    while ((1 << shift) < c->page) ++shift;
    *out = {c->d_k, c->d_v, c->d_k_scales, c->d_v_scales, c->page_step, c->head_step, c->token_step, c->scale_step, static_cast<int>(c->pages), c->heads, shift, c->dim};
    return PVQ_OK;
}

// `heads`: of a row, whose number of rows times them stays below 2^31.
int checked(const pvq_fp8_step* p, const fp8::Cache& c, int64_t heads, fp8::Step* out) {
    if (!p || !p->d_table || !p->d_lengths || p->seqs < 1 || p->rows < 1 || p->width < 1 || p->ld_table < p->width) return PVQ_ERR_INVALID_ARG;
    if (!p->d_starts && p->rows != p->seqs) return PVQ_ERR_INVALID_ARG;
    if (p->seqs >= 1 << 24 || p->rows >= 1 << 28 || p->rows * heads >= int64_t(1) << 31 || p->ld_table >= int64_t(1) << 31) return PVQ_ERR_UNSUPPORTED;
    if (p->width >= int64_t(1) << 30 || p->width << c.page_shift > int64_t(1) << 30) return PVQ_ERR_UNSUPPORTED;
    if (!is_aligned(p->d_table, 4) || !is_aligned(p->d_lengths, 4) || (p->d_starts && !is_aligned(p->d_starts, 4))) return PVQ_ERR_ALIGNMENT;
    *out = {p->d_table, p->d_lengths, p->d_starts, p->ld_table, static_cast<int>(p->width), static_cast<int>(p->seqs), static_cast<int>(p->rows)};
    return PVQ_OK;
}

// Rows of heads of `dim` values.
int checked_rows(const void* p, int dtype, int dim, int64_t row, int64_t head) {
    if (dtype != PVQ_DTYPE_F32 && dtype != PVQ_DTYPE_BF16) return PVQ_ERR_INVALID_ARG;
    if (!p || row < dim || head < dim) return PVQ_ERR_INVALID_ARG;
    if (row >= int64_t(1) << 35 || head >= int64_t(1) << 35) return PVQ_ERR_UNSUPPORTED;
    const int unit = dtype == PVQ_DTYPE_BF16 ? 8 : 4;
    if (!is_aligned(p, 16) || row % unit != 0 || head % unit != 0) return PVQ_ERR_ALIGNMENT;
    return PVQ_OK;
}

#define CHECKED(call)                          \
    do {                                       \
        const int status_ = (call);            \
        if (status_ != PVQ_OK) return status_; \
    } while (0)

}  // namespace

extern "C" int pvq_fp8_cache_write(const pvq_fp8_cache* cache, const pvq_fp8_step* step, const void* d_k, int64_t k_row, int64_t k_head, const void* d_v,
                                   int64_t v_row, int64_t v_head, int dtype, uint32_t* d_status, pvq_stream_t stream) {
    fp8::Cache c;
    fp8::Step p;
    CHECKED(checked(cache, &c));
    CHECKED(checked(step, c, c.heads, &p));
    CHECKED(checked_rows(d_k, dtype, c.dim, k_row, k_head));
    CHECKED(checked_rows(d_v, dtype, c.dim, v_row, v_head));
    const fp8::Rows x{const_cast<void*>(d_k), const_cast<void*>(d_v), k_row, k_head, v_row, v_head};
    return fp8::cache_write(c, p, x, dtype == PVQ_DTYPE_BF16, d_status, static_cast<cudaStream_t>(stream));
}

extern "C" int pvq_fp8_cache_read(const pvq_fp8_cache* cache, const pvq_fp8_step* step, void* d_k, int64_t k_row, int64_t k_head, void* d_v, int64_t v_row,
                                  int64_t v_head, int dtype, uint32_t* d_status, pvq_stream_t stream) {
    fp8::Cache c;
    fp8::Step p;
    CHECKED(checked(cache, &c));
    CHECKED(checked(step, c, c.heads, &p));
    CHECKED(checked_rows(d_k, dtype, c.dim, k_row, k_head));
    CHECKED(checked_rows(d_v, dtype, c.dim, v_row, v_head));
    return fp8::cache_read(c, p, {d_k, d_v, k_row, k_head, v_row, v_head}, dtype == PVQ_DTYPE_BF16, d_status, static_cast<cudaStream_t>(stream));
}

extern "C" size_t pvq_fp8_attention_workspace(const pvq_fp8_cache* cache, const pvq_fp8_step* step, int heads) {
    fp8::Cache c;
    fp8::Step p;
    if (checked(cache, &c) != PVQ_OK || heads < 1 || heads % c.heads != 0 || heads / c.heads > 128 || checked(step, c, heads, &p) != PVQ_OK) return 0;
    return fp8::attention_workspace(c, p, heads);
}

extern "C" int pvq_fp8_attention(const pvq_fp8_cache* cache, const pvq_fp8_step* step, const void* d_q, int heads, int64_t q_row, int64_t q_head, int causal,
                                 int64_t window, float scale, void* d_out, int64_t out_row, int64_t out_head, float* d_lse, void* d_workspace,
                                 size_t workspace_bytes, uint32_t* d_status, pvq_stream_t stream) {
    fp8::AttentionArgs a{};
    CHECKED(checked(cache, &a.cache));
    if (heads < 1 || heads % a.cache.heads != 0 || (causal != 0 && causal != 1) || window < 0 || (window > 0 && !causal)) return PVQ_ERR_INVALID_ARG;
    if (!(scale > 0.0f) || !std::isfinite(scale)) return PVQ_ERR_INVALID_ARG;
    if (heads / a.cache.heads > 128) return PVQ_ERR_UNSUPPORTED;
    CHECKED(checked(step, a.cache, heads, &a.step));
    CHECKED(checked_rows(d_q, PVQ_DTYPE_BF16, a.cache.dim, q_row, q_head));
    CHECKED(checked_rows(d_out, PVQ_DTYPE_BF16, a.cache.dim, out_row, out_head));
    if (d_lse && !is_aligned(d_lse, 4)) return PVQ_ERR_ALIGNMENT;
    const size_t needed = fp8::attention_workspace(a.cache, a.step, heads);
    if (needed > 0 && !d_workspace) return PVQ_ERR_INVALID_ARG;
    if (workspace_bytes < needed) return PVQ_ERR_TABLE_TOO_SMALL;
    if (d_workspace && !is_aligned(d_workspace, 16)) return PVQ_ERR_ALIGNMENT;
    a.q = static_cast<const __nv_bfloat16*>(d_q), a.out = static_cast<__nv_bfloat16*>(d_out), a.lse = d_lse;
    a.q_row = q_row, a.q_head = q_head, a.out_row = out_row, a.out_head = out_head;
    a.heads = heads, a.group = heads / a.cache.heads;
    a.causal = causal;
    a.window = static_cast<int>(std::min<int64_t>(window, INT32_MAX));  // (positions are below that)
    a.scale = std::fmin(scale * 1.44269504088896f, std::numeric_limits<float>::max());
    a.status = d_status;
    a.workspace = static_cast<float*>(d_workspace);
    try {  // (the launchers keep small maps of what they asked the driver, and there may be no memory for them)
        return fp8::attention(a, static_cast<cudaStream_t>(stream));
    } catch (...) {
        return set_cuda_error(cudaErrorMemoryAllocation);
    }
}
