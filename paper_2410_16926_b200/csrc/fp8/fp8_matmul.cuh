// The two kernels of the 8-bit product and what they take.
#pragma once
#include "fp8_mma.cuh"

namespace pvq {
namespace fp8 {

struct MatmulArgs {
    Matrix a, b;
    void* out;
    int64_t rows, outs, inner, ld;  // a.rows, columns of the result, k
    uint32_t* status;
};
// Few rows: 128 columns of the result by up to 128 rows a thread block, k split over `split` blocks of a cluster
// (1, 2, 4 or 8, at most the blocks along k).
int matmul_few(const MatmulArgs& p, bool transposed, bool bf16, int split, cudaStream_t s);
// Clusters of `split` of its blocks for up to `high` rows (16, 32, 64, 128) that run at once, where a block has an SM.
int matmul_few_clusters(int high, int split, int* n);
// Many rows: 256 x 256 of the result a pair of thread blocks.
int matmul_many(const MatmulArgs& p, bool transposed, bool bf16, cudaStream_t s);

}  // namespace fp8
}  // namespace pvq
