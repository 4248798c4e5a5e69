// Sums of the columns of a [rows][cols] fp32 array, always in the same order: the second step of gradients that are summed
// over all tokens, whose first step leaves one row per CTA.  A block takes 8 columns; 32 threads to a column take every
// 32nd row each, and their sums join in a tree.
#include "common.cuh"

namespace based {

namespace {
constexpr int kCols = 8, kRows = 32;
}
// columns 0 .. split - 1 go to a, the others to b
__global__ void __launch_bounds__(kCols * kRows) column_sums_kernel(const float* __restrict__ part, long long rows, int cols,
                                                                    float* __restrict__ a, int split, float* __restrict__ b) {
    __shared__ float sm[kRows][kCols + 1];
    enter_dependent();
    const int x = threadIdx.x % kCols, y = threadIdx.x / kCols, c = blockIdx.x * kCols + x;
    float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
    if (c < cols) {
        long long i = y;
        for (; i + 3 * kRows < rows; i += 4 * kRows) {           // (four loads under way)
            s0 += part[i * cols + c];
            s1 += part[(i + kRows) * cols + c];
            s2 += part[(i + 2 * kRows) * cols + c];
            s3 += part[(i + 3 * kRows) * cols + c];
        }
        for (; i < rows; i += kRows) s0 += part[i * cols + c];
    }
    sm[y][x] = (s0 + s1) + (s2 + s3);
    __syncthreads();
#pragma unroll
    for (int d = kRows / 2; d > 0; d /= 2) {
        if (y < d) sm[y][x] += sm[y + d][x];
        __syncthreads();
    }
    if (y == 0 && c < cols) {
        if (c < split) a[c] = sm[0][x];
        else b[c - split] = sm[0][x];
    }
}

based_status launch_column_sums(const float* part, long long rows, int cols, float* a, int split, float* b, cudaStream_t stream) {
    const cudaError_t e = launch_ex(column_sums_kernel, dim3((cols + kCols - 1) / kCols), dim3(kCols * kRows), 0, 1, true, stream, part,
                                    rows, cols, a, split, b);
    note_launch();
    const based_status st = check_launch("column_sums_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}

}  // namespace based
