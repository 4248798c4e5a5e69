// swa_backward, fp32 io, on multiply-adds: gradients of the sliding-window softmax attention of swa_forward.  With c = scale,
// row i over its keys j = max(0, i-w+1) .. i:
//
//   P_ij = exp(c (s_ij - m_i)) / l_i,  dP_ij = dout_i . v_j,  D_i = sum_j P_ij dP_ij,  dS_ij = c P_ij (dP_ij - D_i),
//   dq_i = sum_j dS_ij k_j,   dk_j = sum_i dS_ij q_i,   dv_j = sum_i P_ij dout_i        (s = q k^T)
//
// Two kernels on tiles of 64 x 64 pairs, 4 x 4 of them per thread, operands as padded fp32 rows in shared memory.  The first
// takes 64 queries: their scores and dP against all the keys they see (two or three tiles of 64, held in registers) give the
// row statistics m, 1/l, D, then dS and dq.  The second takes 64 keys and recomputes P and dS of the queries that see them
// from the statistics.  Neither adds into memory that another CTA writes, so results do not depend on any order.
#include "common.cuh"

namespace based {

namespace {
constexpr int kT = 64, kHD = 64, kStride = kHD + 4, kThreads = 256;
constexpr int kTile = kT * kStride;
constexpr size_t kSmemQ = 5 * kTile * sizeof(float), kSmemK = 6 * kTile * sizeof(float) + kT * sizeof(float4);

// rows r0 .. r0 + 63 of [L][64] into a padded tile, zeros outside [0, L)
__device__ __forceinline__ void load_tile(float* dst, const float* src, int r0, int L) {
    for (int i = threadIdx.x; i < kT * kHD / 4; i += kThreads) {
        const int row = i / (kHD / 4), col = (i % (kHD / 4)) * 4;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r0 + row >= 0 && r0 + row < L) x = *reinterpret_cast<const float4*>(src + (size_t)(r0 + row) * kHD + col);
        *reinterpret_cast<float4*>(dst + row * kStride + col) = x;
    }
}
__device__ __forceinline__ float4 lds(const float* p) { return *reinterpret_cast<const float4*>(p); }
// acc[i][j] += a[row ty + 16 i] . b[row tx + 16 j] over 64
__device__ __forceinline__ void dots(float (&acc)[4][4], const float* a, const float* b, int ty, int tx) {
#pragma unroll 4
    for (int d = 0; d < kHD; d += 4) {
        float4 x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = lds(a + (ty + 16 * i) * kStride + d);
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = lds(b + (tx + 16 * j) * kStride + d);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[i][j] = fmaf(x[i].w, y[j].w, fmaf(x[i].z, y[j].z, fmaf(x[i].y, y[j].y, fmaf(x[i].x, y[j].x, acc[i][j]))));
    }
}
// acc[i][0..3] += sum_k a[row ty + 16 i][k] b[k][4 tx ..]
__device__ __forceinline__ void product(float (&acc)[4][4], const float* a, const float* b, int ty, int tx) {
#pragma unroll 4
    for (int k = 0; k < kT; k += 4) {
        float4 x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = lds(a + (ty + 16 * i) * kStride + k);
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = lds(b + (k + j) * kStride + 4 * tx);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc[i][0] = fmaf(w[j], y[j].x, acc[i][0]);
                acc[i][1] = fmaf(w[j], y[j].y, acc[i][1]);
                acc[i][2] = fmaf(w[j], y[j].z, acc[i][2]);
                acc[i][3] = fmaf(w[j], y[j].w, acc[i][3]);
            }
        }
    }
}
__device__ __forceinline__ void store_rows(float* dst, const float (&acc)[4][4], int r0, int L, int ty, int tx) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = r0 + ty + 16 * i;
        if (row >= L) continue;
        *reinterpret_cast<float4*>(dst + (size_t)row * kHD + 4 * tx) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
    }
}
__device__ __forceinline__ float max16(float x) {
#pragma unroll
    for (int o = 8; o > 0; o /= 2) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}
__device__ __forceinline__ float sum16(float x) {
#pragma unroll
    for (int o = 8; o > 0; o /= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
}  // namespace

// 64 queries against TILES tiles of 64 keys (the last of them their own); stats: (m, 1 / l, D, 0) per row
template <int TILES>
__global__ void __launch_bounds__(kThreads) swa_backward_queries_kernel(const float* __restrict__ q, const float* __restrict__ k,
                                                                        const float* __restrict__ v, const float* __restrict__ dout,
                                                                        float* __restrict__ dq, float4* __restrict__ stats, int L, int window,
                                                                        float scale) {
    extern __shared__ __align__(16) float smem[];
    float *sQ = smem, *sO = sQ + kTile, *sK = sO + kTile, *sV = sK + kTile, *sD = sV + kTile;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, i0 = blockIdx.x * kT;
    const size_t head = (size_t)blockIdx.y * L * kHD;
    enter_dependent();
    load_tile(sQ, q + head, i0, L);
    load_tile(sO, dout + head, i0, L);
    float s[TILES][4][4], dp[TILES][4][4];
    const float c = scale * 1.4426950408889634f;
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        const int j0 = i0 - (TILES - 1 - t) * kT;
        __syncthreads();
        load_tile(sK, k + head, j0, L);
        load_tile(sV, v + head, j0, L);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i >> 2][i & 3] = dp[t][i >> 2][i & 3] = 0.f;
        dots(s[t], sQ, sK, ty, tx);
        dots(dp[t], sO, sV, ty, tx);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int qi = i0 + ty + 16 * i, kj = j0 + tx + 16 * j;
                const bool seen = kj >= 0 && kj <= qi && kj > qi - window;
                s[t][i][j] = seen ? s[t][i][j] : -INFINITY;
                dp[t][i][j] = seen ? dp[t][i][j] : 0.f;
                mx[i] = fmaxf(mx[i], s[t][i][j]);
            }
    }
    float inv[4], D[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        mx[i] = max16(mx[i]);                                    // (finite: a row sees its own key)
        float l = 0.f, w = 0.f;
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[t][i][j] = exp2f((s[t][i][j] - mx[i]) * c);
                l += s[t][i][j];
                w = fmaf(s[t][i][j], dp[t][i][j], w);
            }
        inv[i] = 1.f / sum16(l);
        D[i] = sum16(w) * inv[i];
        if (tx == 0 && i0 + ty + 16 * i < L)
            stats[(size_t)blockIdx.y * L + i0 + ty + 16 * i] = make_float4(mx[i], inv[i], D[i], 0.f);
    }
    float acc[4][4] = {};
    // the last tile of keys is still in shared memory
#pragma unroll
    for (int t = TILES - 1; t >= 0; --t) {
        __syncthreads();
        if (t < TILES - 1) load_tile(sK, k + head, i0 - (TILES - 1 - t) * kT, L);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                sD[(ty + 16 * i) * kStride + tx + 16 * j] = s[t][i][j] * inv[i] * (dp[t][i][j] - D[i]) * scale;
        __syncthreads();
        product(acc, sD, sK, ty, tx);
    }
    store_rows(dq + head, acc, i0, L, ty, tx);
}

// 64 keys and the TILES tiles of queries that see them (the first of them their own)
template <int TILES>
__global__ void __launch_bounds__(kThreads) swa_backward_keys_kernel(const float* __restrict__ q, const float* __restrict__ k,
                                                                     const float* __restrict__ v, const float* __restrict__ dout,
                                                                     const float4* __restrict__ stats, float* __restrict__ dk,
                                                                     float* __restrict__ dv, int L, int window, float scale) {
    extern __shared__ __align__(16) float smem[];
    float *sK = smem, *sV = sK + kTile, *sQ = sV + kTile, *sO = sQ + kTile, *sP = sO + kTile, *sD = sP + kTile;
    float4* sS = reinterpret_cast<float4*>(sD + kTile);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, j0 = blockIdx.x * kT;
    const size_t head = (size_t)blockIdx.y * L * kHD;
    enter_dependent();
    load_tile(sK, k + head, j0, L);
    load_tile(sV, v + head, j0, L);
    const float c = scale * 1.4426950408889634f;
    float ak[4][4] = {}, av[4][4] = {};
    for (int t = 0; t < TILES; ++t) {
        const int i0 = j0 + t * kT;
        if (i0 >= L) break;
        __syncthreads();
        load_tile(sQ, q + head, i0, L);
        load_tile(sO, dout + head, i0, L);
        if (threadIdx.x < kT)
            sS[threadIdx.x] = i0 + threadIdx.x < L ? stats[(size_t)blockIdx.y * L + i0 + threadIdx.x] : make_float4(0.f, 0.f, 0.f, 0.f);
        __syncthreads();
        float s[4][4] = {}, dp[4][4] = {};
        dots(s, sQ, sK, ty, tx);
        dots(dp, sO, sV, ty, tx);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 st = sS[ty + 16 * i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int qi = i0 + ty + 16 * i, kj = j0 + tx + 16 * j;
                const bool seen = kj <= qi && kj > qi - window && qi < L;
                const float P = seen ? exp2f((s[i][j] - st.x) * c) * st.y : 0.f;
                const int at = (tx + 16 * j) * kStride + ty + 16 * i;          // [key][query]
                sP[at] = P;
                sD[at] = seen ? P * (dp[i][j] - st.z) * scale : 0.f;
            }
        }
        __syncthreads();
        product(av, sP, sO, ty, tx);
        product(ak, sD, sQ, ty, tx);
    }
    store_rows(dk + head, ak, j0, L, ty, tx);
    store_rows(dv + head, av, j0, L, ty, tx);
}

template <int TILES>
static based_status launch_tiles(const void* q, const void* k, const void* v, const void* dout, void* dq, void* dk, void* dv, float* stats,
                                 int BH, int L, int window, float scale, cudaStream_t stream) {
    auto kq = swa_backward_queries_kernel<TILES>;
    auto kk = swa_backward_keys_kernel<TILES>;
    // per-device attributes; setting them on every call keeps multi-device processes correct
    if (cudaFuncSetAttribute(kq, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemQ) != cudaSuccess ||
        cudaFuncSetAttribute(kk, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemK) != cudaSuccess)
        return BASED_ERR_CUDA;
    const dim3 grid((L + kT - 1) / kT, BH);
    auto in = [](const void* p) { return static_cast<const float*>(p); };
    cudaError_t e = launch_ex(kq, grid, dim3(kThreads), kSmemQ, 1, true, stream, in(q), in(k), in(v), in(dout), static_cast<float*>(dq),
                              reinterpret_cast<float4*>(stats), L, window, scale);
    if (e == cudaSuccess)
        e = launch_ex(kk, grid, dim3(kThreads), kSmemK, 1, true, stream, in(q), in(k), in(v), in(dout),
                      reinterpret_cast<const float4*>(stats), static_cast<float*>(dk), static_cast<float*>(dv), L, window, scale);
    note_launch();
    note_launch();
    const based_status st = check_launch("swa_backward_queries_kernel, swa_backward_keys_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}

based_status launch_swa_backward_f32(const void* q, const void* k, const void* v, const void* dout, void* dq, void* dk, void* dv,
                                     float* stats, int BH, int L, int window, float scale, cudaStream_t stream) {
    // a query's first key lies window - 1 before it: one tile of 64 back, or two
    return window <= kT + 1 ? launch_tiles<2>(q, k, v, dout, dq, dk, dv, stats, BH, L, window, scale, stream)
                            : launch_tiles<3>(q, k, v, dout, dq, dk, dv, stats, BH, L, window, scale, stream);
}

}  // namespace based
