// Two fp32 values in a 64-bit register, worked on by one instruction (sm_100a), and 16-byte pieces of rows as such pairs.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

namespace based {
namespace pairs {

using pair = uint64_t;

__device__ __forceinline__ pair make(float lo, float hi) {
    pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ pair both(float x) { return make(x, x); }
__device__ __forceinline__ float2 split(pair a) {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(a));
    return f;
}
__device__ __forceinline__ pair fma2(pair a, pair b, pair c) {
    pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ pair mul2(pair a, pair b) {
    pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ pair add2(pair a, pair b) {
    pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// -a: the sign bits
__device__ __forceinline__ pair neg2(pair a) { return a ^ 0x8000000080000000ull; }
__device__ __forceinline__ pair shfl_up2(pair a, int d) { return __shfl_up_sync(0xffffffffu, a, d); }

// 16 bytes of a row: 8 bf16 or 4 fp32 values as V / 2 pairs
template <typename T> struct Piece;
template <> struct Piece<__nv_bfloat16> {
    static constexpr int V = 8;
    static __device__ __forceinline__ void unpack(const uint4& u, pair (&x)[4]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = make(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
    static __device__ __forceinline__ uint4 pack(const pair (&x)[4]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = split(x[i]);
            const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Piece<float> {
    static constexpr int V = 4;
    static __device__ __forceinline__ void unpack(const uint4& u, pair (&x)[2]) {
        x[0] = make(__uint_as_float(u.x), __uint_as_float(u.y));
        x[1] = make(__uint_as_float(u.z), __uint_as_float(u.w));
    }
    static __device__ __forceinline__ uint4 pack(const pair (&x)[2]) {
        const float2 a = split(x[0]), b = split(x[1]);
        return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
    }
};
// 2 N consecutive fp32 values
template <int N> __device__ __forceinline__ void load_f32(const float* p, pair (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const ulonglong2 u = *reinterpret_cast<const ulonglong2*>(p + 2 * i);
        x[i] = u.x;
        x[i + 1] = u.y;
    }
}
template <int N> __device__ __forceinline__ void store_f32(float* p, const pair (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 2) *reinterpret_cast<ulonglong2*>(p + 2 * i) = make_ulonglong2(x[i], x[i + 1]);
}

// 16 bytes global -> shared beside the registers; zeros where `in` is false (src is then not read)
__device__ __forceinline__ void copy_async16(void* smem_dst, const void* src, bool in) {
    const uint32_t dst = static_cast<uint32_t>(__cvta_generic_to_shared(smem_dst));
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

}  // namespace pairs
}  // namespace based
