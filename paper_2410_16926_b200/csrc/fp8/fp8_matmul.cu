// Which kernel makes an 8-bit product.
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
    // k is split until the thread blocks fill the GPU, two an SM up to 32 rows and one above, as long as each has four blocks of
    // 128 along it; up to 32 rows not where one an SM is nearly enough, since blocks of their own start sooner than clusters.
    // One row, 14336 to 4096 (32 tiles): 13.4 us with k in eight parts, 14.6 in four, 28 in one; 4096 to 14336 (112 tiles): 12.9 us
    // in one, 13.9 in two, 16.4 in four.  33 rows, 14336 to 4096: 14.9 us in four, 19 in two, 30 in eight.
    const int64_t room = high <= 32 ? 2 * kSms : kSms;
    int split = 1;
    if (high > 32 || tiles < 104)
        while (split < 8 && tiles * split * 2 <= room && blocks >= 4 * split * 2) split *= 2;
    if (!bf16)  // (long fp32 sums in parts, as matmul_many's)
        while (split < 8 && blocks > 64 * split) split *= 2;
    return matmul_few(p, transposed, bf16, split, s);
}

}  // namespace fp8
}  // namespace pvq
