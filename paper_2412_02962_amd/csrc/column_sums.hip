// The launch of the column sums alone (see column_sums.h).

#include "column_sums.h"

namespace pcpp {

namespace {

__global__ __launch_bounds__(256) void sum_partials_kernel(PartialSums a) {
    __shared__ float lds[16 * 17];
    sum_partials(a, blockIdx.x, lds);
}

}  // namespace

int column_partial_rows(int64_t rows) {
    const int64_t n = (rows + 127) / 128;
    return (int)(n < 512 ? n : 512);
}

hipError_t launch_sum_partials(const PartialSums& a, hipStream_t s) {
    const int blocks = partial_sum_blocks(a);
    if (blocks == 0) return hipSuccess;
    sum_partials_kernel<<<blocks, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace pcpp
