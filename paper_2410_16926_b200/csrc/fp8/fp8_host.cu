// The entry points of the 8-bit floating-point operators: argument checks, then the launches.
#include "fp8_internal.cuh"

using namespace pvq;

namespace {

// Checks a matrix of the format, which the calls read or write, and puts it as the kernels see it.
int checked(const pvq_fp8_matrix* m, fp8::Matrix* out) {
    if (!m || !m->d_codes || !m->d_scales || m->rows < 1 || m->cols < 1 || (m->tile != 0 && m->tile != 1)) return PVQ_ERR_INVALID_ARG;
    const int64_t blocks = (m->cols + fp8::kBlock - 1) / fp8::kBlock;
    if (m->ld_codes < m->cols || m->ld_scales < blocks) return PVQ_ERR_INVALID_ARG;
    if (m->rows >= int64_t(1) << 31 || m->cols >= int64_t(1) << 31 || m->ld_codes >= int64_t(1) << 36) return PVQ_ERR_UNSUPPORTED;
    if (m->rows * blocks >= int64_t(1) << 31) return PVQ_ERR_UNSUPPORTED;
    if (!is_aligned(m->d_codes, 16) || m->ld_codes % 16 != 0 || !is_aligned(m->d_scales, 4) || m->ld_scales % 4 != 0) return PVQ_ERR_ALIGNMENT;
    *out = {m->d_codes, m->d_scales, m->rows, m->cols, m->ld_codes, m->ld_scales, m->tile ? 7 : 0, static_cast<int>(blocks)};
    return PVQ_OK;
}

// Checks a matrix of fp32 or bf16 values with `cols` columns.
int checked_values(const void* p, int dtype, int64_t cols, int64_t ld) {
    if (dtype != PVQ_DTYPE_F32 && dtype != PVQ_DTYPE_BF16) return PVQ_ERR_INVALID_ARG;
    if (!p || ld < cols) return PVQ_ERR_INVALID_ARG;
    if (ld >= int64_t(1) << 35) return PVQ_ERR_UNSUPPORTED;
    if (!is_aligned(p, 16) || ld % (dtype == PVQ_DTYPE_BF16 ? 8 : 4) != 0) return PVQ_ERR_ALIGNMENT;
    return PVQ_OK;
}

bool same_shape(const fp8::Matrix& a, const fp8::Matrix& b) { return a.rows == b.rows && a.cols == b.cols; }

// Nothing is thrown across the C boundary: the launchers of the products keep small maps of what they asked the driver, and
// there may be no memory for them.
template <class F>
int without_exceptions(F&& f) {
    try {
        return f();
    } catch (...) {
        return set_cuda_error(cudaErrorMemoryAllocation);
    }
}

#define CHECKED(call)                          \
    do {                                       \
        const int status_ = (call);            \
        if (status_ != PVQ_OK) return status_; \
    } while (0)

}  // namespace

extern "C" size_t pvq_fp8_scale_row_stride(int64_t cols) {
    return cols < 1 ? 0 : (static_cast<size_t>((cols + fp8::kBlock - 1) / fp8::kBlock) + 3u) & ~static_cast<size_t>(3u);
}

extern "C" int pvq_fp8_quantize(const void* d_x, int dtype, int64_t ld, const pvq_fp8_matrix* q, pvq_stream_t stream) {
    fp8::Matrix m;
    CHECKED(checked(q, &m));
    CHECKED(checked_values(d_x, dtype, m.cols, ld));
    return fp8::quantize(d_x, dtype == PVQ_DTYPE_BF16, ld, m, static_cast<cudaStream_t>(stream));
}

extern "C" int pvq_fp8_dequantize(const pvq_fp8_matrix* q, void* d_out, int dtype, int64_t ld_out, pvq_stream_t stream) {
    fp8::Matrix m;
    CHECKED(checked(q, &m));
    CHECKED(checked_values(d_out, dtype, m.cols, ld_out));
    return fp8::dequantize(m, d_out, dtype == PVQ_DTYPE_BF16, ld_out, static_cast<cudaStream_t>(stream));
}

extern "C" int pvq_fp8_matmul(const pvq_fp8_matrix* a, const pvq_fp8_matrix* b, int transposed, void* d_out, int dtype, int64_t ld_out,
                              uint32_t* d_status, pvq_stream_t stream) {
    fp8::Matrix ma, mb;
    CHECKED(checked(a, &ma));
    CHECKED(checked(b, &mb));
    if (transposed != 0 && transposed != 1) return PVQ_ERR_INVALID_ARG;
    if (ma.cols != (transposed ? mb.rows : mb.cols)) return PVQ_ERR_INVALID_ARG;
    CHECKED(checked_values(d_out, dtype, transposed ? mb.cols : mb.rows, ld_out));
    if (transposed && !mb.shift) return PVQ_ERR_UNSUPPORTED;  // the scales would change inside a block of the sum
    return without_exceptions(
        [&] { return fp8::matmul(ma, mb, transposed != 0, d_out, dtype == PVQ_DTYPE_BF16, ld_out, d_status, static_cast<cudaStream_t>(stream)); });
}

extern "C" int pvq_fp8_gated(const void* d_gate, int64_t ld_gate, const void* d_up, int64_t ld_up, int dtype, int act, const pvq_fp8_matrix* h,
                             const pvq_fp8_matrix* gate, const pvq_fp8_matrix* up, pvq_stream_t stream) {
    if (act != PVQ_ACT_SILU && act != PVQ_ACT_GELU) return PVQ_ERR_INVALID_ARG;
    if (!gate != !up) return PVQ_ERR_INVALID_ARG;
    fp8::GatedArgs a{};
    CHECKED(checked(h, &a.h));
    if (gate) {
        CHECKED(checked(gate, &a.gate8));
        CHECKED(checked(up, &a.up8));
        if (!same_shape(a.h, a.gate8) || !same_shape(a.h, a.up8)) return PVQ_ERR_INVALID_ARG;
    }
    if (a.h.shift || a.gate8.shift || a.up8.shift) return PVQ_ERR_INVALID_ARG;
    CHECKED(checked_values(d_gate, dtype, a.h.cols, ld_gate));
    CHECKED(checked_values(d_up, dtype, a.h.cols, ld_up));
    a.gate = d_gate, a.ld_gate = ld_gate, a.up = d_up, a.ld_up = ld_up;
    return fp8::gated(a, dtype == PVQ_DTYPE_BF16, act, static_cast<cudaStream_t>(stream));
}

extern "C" int pvq_fp8_gated_backward(const void* d_dh, int64_t ld_dh, int dtype, const pvq_fp8_matrix* gate, const pvq_fp8_matrix* up, int act,
                                      void* d_dgate, int64_t ld_dgate, void* d_dup, int64_t ld_dup, pvq_stream_t stream) {
    if (act != PVQ_ACT_SILU && act != PVQ_ACT_GELU) return PVQ_ERR_INVALID_ARG;
    fp8::GatedBackwardArgs a{};
    CHECKED(checked(gate, &a.gate8));
    CHECKED(checked(up, &a.up8));
    if (!same_shape(a.gate8, a.up8) || a.gate8.shift || a.up8.shift) return PVQ_ERR_INVALID_ARG;
    CHECKED(checked_values(d_dh, dtype, a.gate8.cols, ld_dh));
    CHECKED(checked_values(d_dgate, dtype, a.gate8.cols, ld_dgate));
    CHECKED(checked_values(d_dup, dtype, a.gate8.cols, ld_dup));
    a.dh = d_dh, a.ld_dh = ld_dh, a.dgate = d_dgate, a.ld_dgate = ld_dgate, a.dup = d_dup, a.ld_dup = ld_dup;
    return fp8::gated_backward(a, dtype == PVQ_DTYPE_BF16, act, static_cast<cudaStream_t>(stream));
}

extern "C" size_t pvq_fp8_weight_grad_workspace(int64_t rows, int64_t inner, int64_t outer) {
    return rows < 1 || inner < 1 || outer < 1 ? 0 : fp8::weight_grad_workspace(rows, inner, outer);
}

extern "C" int pvq_fp8_weight_grad(const void* d_dy, int64_t outer, int64_t ld_dy, const pvq_fp8_matrix* x, void* d_out, int dtype, int64_t ld_out,
                                   void* d_workspace, size_t workspace_bytes, uint32_t* d_status, pvq_stream_t stream) {
    fp8::Matrix m;
    CHECKED(checked(x, &m));
    if (outer < 1) return PVQ_ERR_INVALID_ARG;
    if (outer >= int64_t(1) << 31) return PVQ_ERR_UNSUPPORTED;
    CHECKED(checked_values(d_dy, PVQ_DTYPE_BF16, outer, ld_dy));
    CHECKED(checked_values(d_out, dtype, m.cols, ld_out));
    if (d_workspace) {
        if (workspace_bytes < fp8::weight_grad_workspace(m.rows, m.cols, outer)) return PVQ_ERR_TABLE_TOO_SMALL;
        if (!is_aligned(d_workspace, 16)) return PVQ_ERR_ALIGNMENT;
    }
    return without_exceptions([&] {
        return fp8::weight_grad(d_dy, outer, ld_dy, m, d_out, dtype == PVQ_DTYPE_BF16, ld_out, d_workspace, d_status, static_cast<cudaStream_t>(stream));
    });
}
