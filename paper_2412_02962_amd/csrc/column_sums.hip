// The launches of the column sums alone (see column_sums.h).

#include "column_sums.h"

namespace pcpp {

namespace {

__global__ __launch_bounds__(256) void sum_partials_kernel(PartialSums a) {
    __shared__ float lds[16 * 17];
    sum_partials(a, blockIdx.x, lds);
}

__global__ __launch_bounds__(256) void column_partials_kernel(const bf16* x, int64_t rows, int C, float* partial,
                                                              int runs) {
    __shared__ float lds[COLUMN_LDS];
    column_partials(x, rows, C, partial, blockIdx.x, runs, lds);
}

}  // namespace

int column_partial_rows(int64_t rows) {
    const int64_t n = (rows + 127) / 128;
    return (int)(n < 512 ? n : 512);
}

hipError_t launch_column_partials(const bf16* x, int64_t rows, int C, float* partial, hipStream_t s) {
    column_partials_kernel<<<column_partial_blocks(rows, C), 256, 0, s>>>(x, rows, C, partial, column_partial_rows(rows));
    return hipGetLastError();
}

hipError_t launch_sum_partials(const PartialSums& a, hipStream_t s) {
    const int blocks = partial_sum_blocks(a);
    if (blocks == 0) return hipSuccess;
    sum_partials_kernel<<<blocks, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace pcpp
