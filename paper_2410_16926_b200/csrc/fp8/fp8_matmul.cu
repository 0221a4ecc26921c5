// Which kernel makes an 8-bit product.
#include "fp8_matmul.cuh"

namespace pvq {
namespace fp8 {

int matmul(const Matrix& a, const Matrix& b, bool transposed, void* out, bool bf16, int64_t ld, uint32_t* status, cudaStream_t s) {
    const MatmulArgs p{a, b, out, a.rows, transposed ? b.cols : b.rows, a.cols, ld, status};
    const int64_t blocks = (p.inner + kBlock - 1) / kBlock;
    const int64_t high = p.rows <= 16 ? 16 : (p.rows <= 32 ? 32 : (p.rows <= 64 ? 64 : 128));
    const int64_t tiles = ((p.outs + 127) / 128) * ((p.rows + high - 1) / high);
    // Tiles of 128 x 128 where one round of them does it, else pairs of thread blocks.  512 rows, 4096 to 4736 (148 tiles) 14.0 us
    // and 16.6 in pairs, 4096 to 5120 (160 tiles) 24.1 and 17.3; 1024 rows, 14336 to 2560 57.1 and 42.8.
    if (p.rows > 128 && tiles > kSms) return matmul_many(p, transposed, bf16, s);
    // k is split over clusters as long as they all run at once, with one thread block an SM, or two up to 32 rows (more than that
    // only for long parts), and each part has four blocks of 128; up to 32 rows not where the tiles alone nearly fill the SMs,
    // since blocks of their own start sooner than clusters.  One row, 4096 to 4096 (32 tiles): 4.8 us with k in four parts, 5.2
    // in eight, 8.7 in one; 14336 to 4096: 12.8 us in eight, 13.5 in four; 4096 to 14336 (112 tiles): 12.9 us in one, 13.9 in two.
    // 33 rows, 14336 to 4096: 14.9 us in four, 19 in two; to 4480 (35 tiles, 33 clusters of four at once): 17.7 in two, 25 in four.
    int split = 1;
    if (high > 32 || tiles < 104)
        for (int next = 2; next <= 8 && blocks >= 4 * next; next *= 2) {
            int clusters = 0;
            const int st = matmul_few_clusters(static_cast<int>(high), next, &clusters);
            if (st != PVQ_OK) return st;
            const bool second = high <= 32 && (tiles <= 2 * clusters || (tiles * next <= 2 * kSms && blocks >= 12 * next));
            if (tiles > clusters && !second) break;
            split = next;
        }
    if (!bf16)  // (long fp32 sums in parts, as matmul_many's; eight of them have runs beyond that)
        while (split < 8 && blocks > 64 * split) split *= 2;
    return matmul_few(p, transposed, bf16, split, s);
}

}  // namespace fp8
}  // namespace pvq
