// swa_backward, fp32 io, on multiply-adds: gradients of the sliding-window softmax attention of swa_forward.  With c = scale,
// row i over its keys j = max(0, i-w+1) .. i:
//
//   P_ij = exp(c (s_ij - m_i)) / l_i,  dP_ij = dout_i . v_j,  D_i = sum_j P_ij dP_ij,  dS_ij = c P_ij (dP_ij - D_i),
//   dq_i = sum_j dS_ij k_j,   dk_j = sum_i dS_ij q_i,   dv_j = sum_i P_ij dout_i        (s = q k^T)
//
// Two kernels of 64, 128 or 256 threads on one, two or four strips of 16 rows: 64 threads work on a strip and the NB blocks of 16 rows of
// the other side that it meets (the queries i meet the keys i - 64 .. i: 80 of them for windows up to 65, 144 for those up to
// 128), 4 x NB pairs per thread in registers.  The first kernel takes queries: scores and dP give the row statistics m, 1/l, D,
// then dS and dq.  The second takes keys and recomputes P and dS of the queries that see them from the statistics.  Neither adds
// into memory that another CTA writes, so results do not depend on any order.
//
// Bound by the multiply-adds (7 products of 16 x 16 NB x 64 per strip; their pipe is what issue waits for most), with shared memory's
// reads, at 53 and 58 % of their peak, close behind.  Scores and dP take even and odd elements in pairs, which halves their
// instructions.  Lanes that read the same 16 bytes are neighbours, which serves half a warp at a time (half-warps that read the same
// rows: 40 us for 38, 255 for 235).
// Measured: 16 heads x 1000 queries, window 64: 38 us, window 128: 70; 32 x 4096: 235 and 481 (56 % of the multiply-adds' rate with
// window 64).  On tiles of 64 x 64, half of whose pairs lie outside the band, these took 68, 98, 511 and 709.
#include "common.cuh"
#include "pairs.cuh"

namespace based {
using namespace pairs;

namespace {
constexpr int kS = 16, kHD = 64, kStride = kHD + 4;
template <int NB, int STRIPS> struct Cfg {
    static constexpr int kT = kS * STRIPS, kThreads = 64 * STRIPS;   // rows of a CTA, threads
    static constexpr int kFar = kT - kS + kS * NB;                   // rows of the other side: those of four strips
    static constexpr int kPStride = kS * NB + 4;                     // of a row of P or dS
    static constexpr int kNear = 2 * kT * kStride, kWeights = 2 * kT * kPStride;
    static constexpr size_t kSmemQ = (kNear + 2 * kFar * kStride) * sizeof(float);
    static constexpr size_t kSmemK = ((kNear > kWeights ? kNear : kWeights) + 2 * kFar * kStride) * sizeof(float) + kFar * sizeof(float4);
    static_assert(kT * kPStride <= kFar * kStride && kSmemK <= 232448 && kSmemQ <= 232448, "shared memory");
};

// ROWS rows from r0 on of [L][64] into padded rows, zeros outside [0, L)
template <int ROWS, int THREADS> __device__ __forceinline__ void load_rows(float* dst, const float* src, int r0, int L) {
#pragma unroll 8
    for (int i = threadIdx.x; i < ROWS * kHD / 4; i += THREADS) {
        const int row = i / (kHD / 4), col = (i % (kHD / 4)) * 4, r = r0 + row;
        const bool in = r >= 0 && r < L;
        copy_async16(dst + row * kStride + col, src + (size_t)(in ? r : 0) * kHD + col, in);
    }
}
// the 64 threads of a strip
__device__ __forceinline__ void strip_sync(int strip) { asm volatile("bar.sync %0, 64;" ::"r"(1 + strip) : "memory"); }
__device__ __forceinline__ float4 lds(const float* p) { return *reinterpret_cast<const float4*>(p); }
// out[i][j] = a[row ty + 4 i] . b[row tx + 16 j] over 64
template <int NB> __device__ __forceinline__ void dots(float (&out)[4][NB], const float* a, const float* b, int ty, int tx) {
    pair acc[4][NB];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = 0;
#pragma unroll 2
    for (int d = 0; d < kHD; d += 4) {
        ulonglong2 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const ulonglong2*>(a + (ty + 4 * i) * kStride + d);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(b + (tx + 16 * j) * kStride + d);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i][j] = fma2(x[i].y, y.y, fma2(x[i].x, y.x, acc[i][j]));
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const float2 f = split(acc[i][j]);
            out[i][j] = f.x + f.y;
        }
}
// acc[i][0..3] = sum over the strip's 16 NB of a[row ty + 4 i][k] b[k][4 tx ..]
template <int NB> __device__ __forceinline__ void product(float (&acc)[4][4], const float* a, const float* b, int ty, int tx) {
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i >> 2][i & 3] = 0.f;
#pragma unroll 4
    for (int k = 0; k < kS * NB; k += 4) {
        float4 x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = lds(a + (ty + 4 * i) * (kS * NB + 4) + k);
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
        const int row = r0 + ty + 4 * i;
        if (row >= L) continue;
        *reinterpret_cast<float4*>(dst + (size_t)row * kHD + 4 * tx) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
    }
}
__device__ __forceinline__ float max16(float x) {
#pragma unroll
    for (int o = 16; o > 1; o /= 2) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}
__device__ __forceinline__ float sum16(float x) {
#pragma unroll
    for (int o = 16; o > 1; o /= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
}  // namespace

// 16 STRIPS queries; stats: (m, 1 / l, D, 0) per row
template <int NB, int STRIPS>
__global__ void __launch_bounds__(64 * STRIPS, NB == 5 ? 8 / STRIPS : 4 / STRIPS)
    swa_backward_queries_kernel(const float* __restrict__ q, const float* __restrict__ k, const float* __restrict__ v,
                                const float* __restrict__ dout, float* __restrict__ dq, float4* __restrict__ stats, int L, int window,
                                float scale) {
    using C = Cfg<NB, STRIPS>;
    constexpr int kT = C::kT, kThreads = C::kThreads;
    extern __shared__ __align__(16) float smem[];
    float *sQ = smem, *sO = sQ + kT * kStride, *sK = sO + kT * kStride, *sV = sK + C::kFar * kStride, *sD = sV;      // (dS over V)
    const int tx = (threadIdx.x >> 1) & 15, ty = (threadIdx.x & 1) + ((threadIdx.x >> 4) & 2), strip = threadIdx.x >> 6, i0 = blockIdx.x * kT;
    const size_t head = (size_t)blockIdx.y * L * kHD;
    const int r0 = kS * strip, first = i0 + r0 - kS * (NB - 1);      // the strip's first row, and its first key
    enter_dependent();
    load_rows<kT, kThreads>(sQ, q + head, i0, L);
    load_rows<C::kFar, kThreads>(sK, k + head, i0 - kS * (NB - 1), L);
    copy_async_commit();
    load_rows<kT, kThreads>(sO, dout + head, i0, L);
    load_rows<C::kFar, kThreads>(sV, v + head, i0 - kS * (NB - 1), L);
    copy_async_commit();
    copy_async_wait<1>();
    __syncthreads();
    float s[4][NB], dp[4][NB];
    dots<NB>(s, sQ + r0 * kStride, sK + r0 * kStride, ty, tx);
    copy_async_wait<0>();
    __syncthreads();
    dots<NB>(dp, sO + r0 * kStride, sV + r0 * kStride, ty, tx);
    __syncthreads();                                                 // (everyone is done with V)
    const float c = scale * 1.4426950408889634f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int qi = i0 + r0 + ty + 4 * i;
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int kj = first + tx + 16 * j;
            const bool seen = kj >= 0 && kj <= qi && kj > qi - window;
            s[i][j] = seen ? s[i][j] : -INFINITY;
            dp[i][j] = seen ? dp[i][j] : 0.f;
            mx = fmaxf(mx, s[i][j]);
        }
        mx = max16(mx);                                              // (finite: a row sees its own key)
        float l = 0.f, w = 0.f;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            s[i][j] = exp2f((s[i][j] - mx) * c);
            l += s[i][j];
            w = fmaf(s[i][j], dp[i][j], w);
        }
        const float inv = 1.f / sum16(l), D = sum16(w) * inv;
        if (tx == 0 && qi < L) stats[(size_t)blockIdx.y * L + qi] = make_float4(mx, inv, D, 0.f);
#pragma unroll
        for (int j = 0; j < NB; ++j) sD[(r0 + ty + 4 * i) * C::kPStride + tx + 16 * j] = s[i][j] * inv * (dp[i][j] - D) * scale;
    }
    strip_sync(strip);
    float acc[4][4];
    product<NB>(acc, sD + r0 * C::kPStride, sK + r0 * kStride, ty, tx);
    store_rows(dq + head, acc, i0 + r0, L, ty, tx);
}

// 16 STRIPS keys and the queries that see them
template <int NB, int STRIPS>
__global__ void __launch_bounds__(64 * STRIPS, NB == 5 ? 8 / STRIPS : 4 / STRIPS)
    swa_backward_keys_kernel(const float* __restrict__ q, const float* __restrict__ k, const float* __restrict__ v,
                             const float* __restrict__ dout, const float4* __restrict__ stats, float* __restrict__ dk, float* __restrict__ dv,
                             int L, int window, float scale) {
    using C = Cfg<NB, STRIPS>;
    constexpr int kT = C::kT, kThreads = C::kThreads;
    extern __shared__ __align__(16) float smem[];
    float *sQ = smem, *sO = sQ + C::kFar * kStride, *sK = sO + C::kFar * kStride + C::kFar * 4, *sV = sK + kT * kStride;
    float *sP = sK, *sD = sP + kT * C::kPStride;                     // (over K and V)
    float4* sS = reinterpret_cast<float4*>(sO + C::kFar * kStride);
    const int tx = (threadIdx.x >> 1) & 15, ty = (threadIdx.x & 1) + ((threadIdx.x >> 4) & 2), strip = threadIdx.x >> 6, j0 = blockIdx.x * kT, r0 = kS * strip;
    const size_t head = (size_t)blockIdx.y * L * kHD;
    enter_dependent();
    load_rows<kT, kThreads>(sK, k + head, j0, L);
    load_rows<C::kFar, kThreads>(sQ, q + head, j0, L);
    copy_async_commit();
    load_rows<kT, kThreads>(sV, v + head, j0, L);
    load_rows<C::kFar, kThreads>(sO, dout + head, j0, L);
    for (int i = threadIdx.x; i < C::kFar; i += kThreads) copy_async16(sS + i, stats + (size_t)blockIdx.y * L + min(j0 + i, L - 1), j0 + i < L);
    copy_async_commit();
    copy_async_wait<1>();
    __syncthreads();
    float s[4][NB], dp[4][NB];
    dots<NB>(s, sK + r0 * kStride, sQ + r0 * kStride, ty, tx);
    copy_async_wait<0>();
    __syncthreads();
    dots<NB>(dp, sV + r0 * kStride, sO + r0 * kStride, ty, tx);
    __syncthreads();                                                 // (everyone is done with K and V)
    const float c = scale * 1.4426950408889634f;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int qi = j0 + r0 + tx + 16 * j;
        const float4 st = sS[r0 + tx + 16 * j];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int kj = j0 + r0 + ty + 4 * i, at = (r0 + ty + 4 * i) * C::kPStride + tx + 16 * j;
            const bool seen = kj <= qi && kj > qi - window && qi < L;
            const float P = seen ? exp2f((s[i][j] - st.x) * c) * st.y : 0.f;
            sP[at] = P;
            sD[at] = seen ? P * (dp[i][j] - st.z) * scale : 0.f;
        }
    }
    strip_sync(strip);
    float acc[4][4];
    product<NB>(acc, sP + r0 * C::kPStride, sO + r0 * kStride, ty, tx);
    store_rows(dv + head, acc, j0 + r0, L, ty, tx);
    product<NB>(acc, sD + r0 * C::kPStride, sQ + r0 * kStride, ty, tx);
    store_rows(dk + head, acc, j0 + r0, L, ty, tx);
}

template <int NB, int STRIPS>
static based_status launch_strips(const void* q, const void* k, const void* v, const void* dout, void* dq, void* dk, void* dv, float* stats,
                                 int BH, int L, int window, float scale, cudaStream_t stream) {
    using C = Cfg<NB, STRIPS>;
    auto kq = swa_backward_queries_kernel<NB, STRIPS>;
    auto kk = swa_backward_keys_kernel<NB, STRIPS>;
    // per-device attributes; setting them on every call keeps multi-device processes correct
    if (cudaFuncSetAttribute(kq, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kSmemQ) != cudaSuccess ||
        cudaFuncSetAttribute(kk, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kSmemK) != cudaSuccess)
        return BASED_ERR_CUDA;
    const dim3 grid((L + C::kT - 1) / C::kT, BH);
    auto in = [](const void* p) { return static_cast<const float*>(p); };
    cudaError_t e = launch_ex(kq, grid, dim3(C::kThreads), C::kSmemQ, 1, true, stream, in(q), in(k), in(v), in(dout), static_cast<float*>(dq),
                              reinterpret_cast<float4*>(stats), L, window, scale);
    if (e == cudaSuccess)
        e = launch_ex(kk, grid, dim3(C::kThreads), C::kSmemK, 1, true, stream, in(q), in(k), in(v), in(dout),
                      reinterpret_cast<const float4*>(stats), static_cast<float*>(dk), static_cast<float*>(dv), L, window, scale);
    note_launch();
    note_launch();
    const based_status st = check_launch("swa_backward_queries_kernel, swa_backward_keys_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}

based_status launch_swa_backward_f32(const void* q, const void* k, const void* v, const void* dout, void* dq, void* dk, void* dv,
                                     float* stats, int BH, int L, int window, float scale, cudaStream_t stream) {
    // A query's first key lies window - 1 before it: 64 / 16 blocks back, or 128 / 16.  Strips per CTA: four where the chip is full of
    // such CTAs, fewer (more CTAs, less for each) where they are few.  us with 1 / 2 / 4, heads x queries, window 64: 4 x 100 16 / 16 / 23,
    // 8 x 700 25 / 32 / 40, 16 x 700 39 / 33 / 41, 16 x 1000 46 / 44 / 40; window 128: 8 x 300 27 / 31 / 38, 8 x 700 48 / 43 / 38
    const long long fours = ((long long)L + 63) / 64 * BH;
    if (window <= 65) {
        if (4 * fours <= 3 * kSMs) return launch_strips<5, 1>(q, k, v, dout, dq, dk, dv, stats, BH, L, window, scale, stream);
        if (2 * fours <= 3 * kSMs) return launch_strips<5, 2>(q, k, v, dout, dq, dk, dv, stats, BH, L, window, scale, stream);
        return launch_strips<5, 4>(q, k, v, dout, dq, dk, dv, stats, BH, L, window, scale, stream);
    }
    if (2 * fours <= kSMs) return launch_strips<9, 1>(q, k, v, dout, dq, dk, dv, stats, BH, L, window, scale, stream);
    return launch_strips<9, 4>(q, k, v, dout, dq, dk, dv, stats, BH, L, window, scale, stream);
}

}  // namespace based
