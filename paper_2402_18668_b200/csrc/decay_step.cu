// Decay attention, one new token per sequence:  S <- exp(-rate) S + k v^T,  o = scale q S,  in one pass over the fp32 state.
//
// Bound by HBM: the state is read once and written once, 8 d_k d_v bytes a head against 5 d_k d_v flop.  One CTA of 256 threads per head;
// d_v / 4 consecutive threads cover a row with 16 bytes each, all of a thread's rows (at most 16) are asked for before the first is used, and
// the rows' shares of o join through shared memory in a fixed order.
#include "decay.cuh"

namespace based {

namespace {

constexpr int kThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kThreads) decay_step_kernel(const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v,
                                                              const float* __restrict__ rate, const float* state_in, T* __restrict__ out,
                                                              float* state_out, int H, int dk, int dv, float scale) {
    __shared__ float sq[kDecayMaxWidth], sk[kDecayMaxWidth];
    __shared__ __align__(16) float part[kThreads * 4];
    enter_dependent();
    const long long head = blockIdx.x;
    const int tid = threadIdx.x, cols = dv / 4, groups = kThreads / cols, c = tid % cols, g = tid / cols;
    const bool mine = g < groups;
    const long long base = head * dk * dv;
    float4 s[16];
    const int rows = mine ? (dk - g + groups - 1) / groups : 0;              // rows g, g + groups, ...: 16 at most
    const float4* in = reinterpret_cast<const float4*>(state_in + base) + c;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < rows) s[i] = in[(long long)(g + i * groups) * cols];
    if (tid < dk) {
        sq[tid] = to_f32(q[head * dk + tid]) * scale;
        sk[tid] = to_f32(k[head * dk + tid]);
    }
    const float a = faded(rate_of(rate[head % H]), 1);
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f), acc = x;
    if (mine) x = make_float4(to_f32(v[head * dv + 4 * c]), to_f32(v[head * dv + 4 * c + 1]), to_f32(v[head * dv + 4 * c + 2]), to_f32(v[head * dv + 4 * c + 3]));
    __syncthreads();
    float4* to = reinterpret_cast<float4*>(state_out + base) + c;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < rows) {
            const int r = g + i * groups;
            const float kr = sk[r], qr = sq[r];
            if (a == 0.f) s[i] = make_float4(0.f, 0.f, 0.f, 0.f);        // dropped, whatever it holds, as in the prompt's kernels
            s[i] = make_float4(fmaf(a, s[i].x, kr * x.x), fmaf(a, s[i].y, kr * x.y), fmaf(a, s[i].z, kr * x.z), fmaf(a, s[i].w, kr * x.w));
            acc = make_float4(fmaf(qr, s[i].x, acc.x), fmaf(qr, s[i].y, acc.y), fmaf(qr, s[i].z, acc.z), fmaf(qr, s[i].w, acc.w));
            to[(long long)r * cols] = s[i];
        }
    if (mine) *reinterpret_cast<float4*>(part + 4 * tid) = acc;
    __syncthreads();
    if (tid < dv) {
        float o = 0.f;
        for (int i = 0; i < groups; ++i) o += part[i * dv + tid];
        out[head * dv + tid] = from_f32<T>(o);
    }
}

template <typename T>
based_status launch_t(const void* q, const void* k, const void* v, const float* rate, const float* state_in, void* out, float* state_out,
                      long long BH, int H, int dk, int dv, float scale, cudaStream_t stream) {
    static std::atomic<bool> split[64];
    if (prefer_l1(decay_step_kernel<T>, 25, split) != cudaSuccess) return BASED_ERR_CUDA;
    const cudaError_t e = launch_ex(decay_step_kernel<T>, dim3((unsigned)BH), dim3(kThreads), 0, 1, true, stream, static_cast<const T*>(q),
                                    static_cast<const T*>(k), static_cast<const T*>(v), rate, state_in, static_cast<T*>(out), state_out, H, dk,
                                    dv, scale);
    note_launch();
    const based_status st = check_launch("decay_step_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}

}  // namespace

based_status launch_decay_step(const void* q, const void* k, const void* v, const float* rate, const float* state_in, void* out,
                               float* state_out, long long BH, int H, int dk, int dv, float scale, based_dtype io, cudaStream_t stream) {
    return io == BASED_F32 ? launch_t<float>(q, k, v, rate, state_in, out, state_out, BH, H, dk, dv, scale, stream)
                           : launch_t<__nv_bfloat16>(q, k, v, rate, state_in, out, state_out, BH, H, dk, dv, scale, stream);
}

}  // namespace based
