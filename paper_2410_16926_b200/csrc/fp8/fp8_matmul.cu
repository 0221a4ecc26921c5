// Which kernel makes an 8-bit product.
#include <algorithm>

#include "fp8_matmul.cuh"

namespace pvq {
namespace fp8 {

int matmul(const Matrix& a, const Matrix& b, bool transposed, void* out, bool bf16, int64_t ld, uint32_t* status, cudaStream_t s) {
    const MatmulArgs p{a, b, out, a.rows, transposed ? b.cols : b.rows, a.cols, ld, status};
    const int64_t blocks = (p.inner + kBlock - 1) / kBlock;
    const int64_t pairs = ((p.rows + 255) / 256) * ((p.outs + 255) / 256);
    if (p.rows > 128 && pairs >= 48) return matmul_many(p, transposed, bf16, s);
    const int64_t high = p.rows <= 16 ? 16 : (p.rows <= 32 ? 32 : (p.rows <= 64 ? 64 : 128));
    const int64_t tiles = ((p.outs + 127) / 128) * ((p.rows + high - 1) / high);
    if ((p.rows + high - 1) / high > 65535) return matmul_many(p, transposed, bf16, s);
    int split = 1;
    while (split < 8 && tiles * split * 2 <= 2 * kSms && blocks >= 4 * split * 2) split *= 2;
    return matmul_few(p, transposed, bf16, split, s);
}

}  // namespace fp8
}  // namespace pvq
