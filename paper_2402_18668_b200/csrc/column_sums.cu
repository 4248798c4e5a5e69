// Sums of the columns of a [rows][cols] fp32 array, always in the same order: the second step of gradients that are summed
// over all tokens, whose first step leaves one row per CTA.  A block takes 8 columns; ROWS threads to a column (32, or 128 above 128
// rows: 592 of them took 4.2 us behind the kernel that writes them with 32) take every ROWS'th row each, and their sums join in a tree.
#include "common.cuh"

namespace based {

namespace {
constexpr int kCols = 8;
}
// columns 0 .. split - 1 go to a, the others to b
template <int ROWS>
__global__ void __launch_bounds__(kCols * ROWS) column_sums_kernel(const float* __restrict__ part, long long rows, int cols,
                                                                   float* __restrict__ a, int split, float* __restrict__ b) {
    constexpr int kWarps = kCols * ROWS / 32;
    __shared__ float sm[kWarps][kCols + 1];
    enter_dependent();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, x = lane % kCols, y = threadIdx.x / kCols, c = blockIdx.x * kCols + x;
    float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
    if (c < cols) {
        long long i = y;
        for (; i + 3 * ROWS < rows; i += 4 * ROWS) {             // (four loads under way)
            s0 += part[i * cols + c];
            s1 += part[(i + ROWS) * cols + c];
            s2 += part[(i + 2 * ROWS) * cols + c];
            s3 += part[(i + 3 * ROWS) * cols + c];
        }
        if (i < rows) s0 += part[i * cols + c];
        if (i + ROWS < rows) s1 += part[(i + ROWS) * cols + c];
        if (i + 2 * ROWS < rows) s2 += part[(i + 2 * ROWS) * cols + c];
    }
    float s = (s0 + s1) + (s2 + s3);
    s += __shfl_xor_sync(0xffffffffu, s, 8);                     // the warp's four rows
    s += __shfl_xor_sync(0xffffffffu, s, 16);
    if (lane < kCols) sm[warp][x] = s;
    __syncthreads();
    if (warp >= kCols) return;
    s = lane < kWarps ? sm[lane][warp] : 0.f;                    // one warp per column
#pragma unroll
    for (int d = kWarps / 2; d > 0; d /= 2) s += __shfl_xor_sync(0xffffffffu, s, d);
    const int col = blockIdx.x * kCols + warp;
    if (lane == 0 && col < cols) {
        if (col < split) a[col] = s;
        else b[col - split] = s;
    }
}

based_status launch_column_sums(const float* part, long long rows, int cols, float* a, int split, float* b, cudaStream_t stream) {
    const dim3 grid((cols + kCols - 1) / kCols);
    const cudaError_t e = rows > 128 ? launch_ex(column_sums_kernel<128>, grid, dim3(kCols * 128), 0, 1, true, stream, part, rows, cols, a, split, b)
                                     : launch_ex(column_sums_kernel<32>, grid, dim3(kCols * 32), 0, 1, true, stream, part, rows, cols, a, split, b);
    note_launch();
    const based_status st = check_launch("column_sums_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}

}  // namespace based
