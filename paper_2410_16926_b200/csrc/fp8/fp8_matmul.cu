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
    // only for long parts), and each part has four blocks of 128.  One row, 4096 to 4096 (32 tiles): 5.1 us with k in four parts, 5.2
    // in eight, 8.7 in one; 14336 to 4096: 12.9 us in eight, 13.5 in four.  33 rows, 14336 to 4096: 15.2 us in four, 19 in two; to 4480
    // (35 tiles, 33 clusters of four at once): 17.7 in two, 25 in four.
    // Up to 32 rows, tiles that take more than half of the SMs are split where k has 40 blocks: blocks of their own start
    // sooner than clusters, which end sooner.  One row, in us, not split and in two:
    //   k        76 to 80 tiles   96         112        148 tiles
    //   2048     6.4   6.4    6.5   7.0    7.0   7.6    9.8   9.5
    //   4096    11.8  12.2   12.5  12.8   13.1  13.2   15.7  16.0
    //   5120    14.1  13.8   14.9  14.5   15.9  15.3   19.0  18.6
    //   8192    20.5  19.7   22.2  20.8   24.3  22.2   29.5  27.2
    //   14336   32.6  31.0   35.1  32.3   37.7  34.4   45.6  43.5
    // and with 74 tiles 6.4 and 5.4 for 2048, 11.6 and 10.6 for 4096.  (20 rows: the same order everywhere, 3 to 5% more.)
    int split = 1;
    if (high > 32 || tiles <= kSms / 2 || blocks >= 40)
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
