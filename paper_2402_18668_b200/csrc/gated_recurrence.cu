// based_gated_recurrence_forward / _step / _backward: the gated linear recurrence, a token mixer with one fp32 state per
// channel.  Per sequence and channel, from the state given (or 0):
//
//   s = sigmoid(r),  a = exp(-rate s),  m = sqrt(1 - a^2),     h_t = a_t h_{t-1} + m_t sigmoid(g_t) x_t
//
// A run of tokens maps the state before it to the state behind it by h -> A h + H, and two runs in a row join to
// (A2 A1, A2 H1 + H2).  A thread takes TOK consecutive tokens of one 16-byte piece of channels, the four token groups of a
// warp join by shuffles, the warps of a CTA and the CTAs of a cluster through shared memory, and every thread then replays
// its own tokens from the state that reaches it.  So the inputs are read once, whatever the sequence's length, and the loop
// along the sequence carries nothing but the state.  The backward pass is the same scan from the last token to the first, of
//
//   E_t = a_t (dout_t + E_{t+1}),     G_t = dout_t + E_{t+1} the gradient of h_t,
//   dx = G m i,  dg = G m x i (1 - i),  dlog a = a G h_{t-1} - (a^2 / m) G i x,  dr = -rate dlog a s (1 - s),
//   drate = -sum dlog a s  (i = sigmoid(g); h_{t-1} is read from the output that the caller kept).
//
// A thread's inputs come by asynchronous copies into a slot of shared memory that only it reads (no barrier), those of the
// next step while this one is computed.
#include <type_traits>

#include "common.cuh"
#include "pairs.cuh"

namespace based {
using namespace pairs;

namespace {
constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kLanes = 8;                        // pieces of 16 bytes side by side: 128 bytes of a row
constexpr int kGroups = kThreads / kLanes;       // groups of TOK consecutive tokens
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float root(float x) {
    float y;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rroot(float x) {
    float y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// (a NaN stays one)
__device__ __forceinline__ float min_nan(float x, float y) {
    float z;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
    return z;
}
__device__ __forceinline__ float max_nan(float x, float y) {
    float z;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
    return z;
}

// 1 + exp(-x).  The exponent is held at 2^60, so that the product of two of them and its reciprocal stay finite: a
// sigmoid below 2^-60 is taken as 2^-60
__device__ __forceinline__ pair one_plus_exp_neg(pair x) {
    const float2 t = split(mul2(x, both(-kLog2e)));
    return add2(make(ex2(min_nan(t.x, 60.f)), ex2(min_nan(t.y, 60.f))), both(1.f));
}
__device__ __forceinline__ pair rcp2(pair x) {
    const float2 t = split(x);
    return make(rcp(t.x), rcp(t.y));
}
// exp(la) - 1 for la <= 0.  Near 0 by its power series (to 2^-24 of la from -1/4 on: six terms), so that 1 - a^2 = -p (2 + p)
// keeps its digits where the decay is slow.  SMALL: every la is in that range
template <bool SMALL> __device__ __forceinline__ pair exp_less_one(pair la) {
    pair y = fma2(la, both(1.f / 720.f), both(1.f / 120.f));
    y = fma2(la, y, both(1.f / 24.f));
    y = fma2(la, y, both(1.f / 6.f));
    y = fma2(la, y, both(0.5f));
    y = fma2(la, y, both(1.f));
    y = mul2(la, y);
    if constexpr (!SMALL) {
        const float2 l = split(la), f = split(y), e = split(mul2(la, both(kLog2e)));
        y = make(l.x > -0.25f ? f.x : ex2(e.x) - 1.f, l.y > -0.25f ? f.y : ex2(e.y) - 1.f);
    }
    return y;
}
// 1 - a^2 from p = a - 1
__device__ __forceinline__ pair one_less_square(pair p) { return mul2(neg2(p), add2(p, both(2.f))); }

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive_wait() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// 16 bytes into the same place of another CTA's shared memory
__device__ __forceinline__ void store_remote(const void* own, uint32_t rank, ulonglong2 v) {
    uint32_t addr;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(own))), "r"(rank));
    asm volatile("st.shared::cluster.v2.b64 [%0], {%1, %2};" ::"r"(addr), "l"(v.x), "l"(v.y) : "memory");
}

// The joins of a step.  Shared memory holds two sets, used in turn: a set is written again two steps on, when every thread has
// passed the barrier of the step between and so has read it.
template <int P2, int PARTS> struct Joins {                      // P2: pairs of channels per thread
    ulonglong2 warp[2][kWarps][P2][kLanes];                      // A (P2 / 2 words), then H
    ulonglong2 part[2][PARTS > 1 ? PARTS : 1][P2][kLanes];
};
// A, H: what the thread's tokens do to the state.  h: the state before this step, on return the one behind it.  Returns the
// state that reaches the thread's first token in `first`.
template <int P2, int PARTS>
__device__ __forceinline__ void join(Joins<P2, PARTS>& sm, int turn, int rank, pair (&A)[P2], pair (&H)[P2], pair (&h)[P2],
                                     pair (&first)[P2]) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = lane & (kLanes - 1);
    // inclusive over the warp's four groups
#pragma unroll
    for (int d = kLanes; d < 32; d *= 2) {
#pragma unroll
        for (int e = 0; e < P2; ++e) {
            const pair a = shfl_up2(A[e], d), b = shfl_up2(H[e], d);
            if (lane >= d) {
                H[e] = fma2(A[e], b, H[e]);
                A[e] = mul2(A[e], a);
            }
        }
    }
    if (lane >= 32 - kLanes) {
#pragma unroll
        for (int w = 0; w < P2 / 2; ++w) {
            sm.warp[turn][warp][w][col] = make_ulonglong2(A[2 * w], A[2 * w + 1]);
            sm.warp[turn][warp][P2 / 2 + w][col] = make_ulonglong2(H[2 * w], H[2 * w + 1]);
        }
    }
    // exclusive
#pragma unroll
    for (int e = 0; e < P2; ++e) {
        A[e] = shfl_up2(A[e], kLanes);
        H[e] = shfl_up2(H[e], kLanes);
        if (lane < kLanes) {
            A[e] = both(1.f);
            H[e] = 0;
        }
    }
    __syncthreads();
    if constexpr (PARTS > 1) {
        // the CTA's total, and in front of the own warp's tokens the prefix of the warps before it
        pair ta[P2], th[P2], pa[P2], ph[P2];
#pragma unroll
        for (int e = 0; e < P2; ++e) {
            ta[e] = both(1.f);
            th[e] = 0;
        }
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w == warp) {
#pragma unroll
                for (int e = 0; e < P2; ++e) {
                    pa[e] = ta[e];
                    ph[e] = th[e];
                }
            }
#pragma unroll
            for (int u = 0; u < P2 / 2; ++u) {
                const ulonglong2 a = sm.warp[turn][w][u][col], b = sm.warp[turn][w][P2 / 2 + u][col];
                th[2 * u] = fma2(a.x, th[2 * u], b.x);
                th[2 * u + 1] = fma2(a.y, th[2 * u + 1], b.y);
                ta[2 * u] = mul2(a.x, ta[2 * u]);
                ta[2 * u + 1] = mul2(a.y, ta[2 * u + 1]);
            }
        }
        // the total goes to every CTA of the cluster, and the state runs through the totals of the CTAs before this one
        if (lane < kLanes) {
#pragma unroll
            for (int to = 0; to < PARTS; ++to) {
                if ((to & (kWarps - 1)) != warp) continue;
#pragma unroll
                for (int u = 0; u < P2 / 2; ++u) {
                    store_remote(&sm.part[turn][rank][u][col], to, make_ulonglong2(ta[2 * u], ta[2 * u + 1]));
                    store_remote(&sm.part[turn][rank][P2 / 2 + u][col], to, make_ulonglong2(th[2 * u], th[2 * u + 1]));
                }
            }
        }
        cluster_arrive_wait();
        pair hs[P2];
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
            if (q == rank) {
#pragma unroll
                for (int e = 0; e < P2; ++e) hs[e] = h[e];
            }
#pragma unroll
            for (int u = 0; u < P2 / 2; ++u) {
                const ulonglong2 a = sm.part[turn][q][u][col], b = sm.part[turn][q][P2 / 2 + u][col];
                h[2 * u] = fma2(a.x, h[2 * u], b.x);
                h[2 * u + 1] = fma2(a.y, h[2 * u + 1], b.y);
            }
        }
#pragma unroll
        for (int e = 0; e < P2; ++e) first[e] = fma2(A[e], fma2(pa[e], hs[e], ph[e]), H[e]);
    } else {
        pair hs[P2];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w == warp) {
#pragma unroll
                for (int e = 0; e < P2; ++e) hs[e] = h[e];
            }
#pragma unroll
            for (int u = 0; u < P2 / 2; ++u) {
                const ulonglong2 a = sm.warp[turn][w][u][col], b = sm.warp[turn][w][P2 / 2 + u][col];
                h[2 * u] = fma2(a.x, h[2 * u], b.x);
                h[2 * u + 1] = fma2(a.y, h[2 * u + 1], b.y);
            }
        }
#pragma unroll
        for (int e = 0; e < P2; ++e) first[e] = fma2(A[e], hs[e], H[e]);
    }
}
}  // namespace

// grid: clusters of PARTS CTAs, one per sequence and slab of 8 pieces of channels; the CTAs of a cluster take runs of
// 16 TOK tokens in turn.
template <typename T, int TOK, int PARTS>
__global__ void __launch_bounds__(kThreads, 4)
    gated_recurrence_kernel(const T* __restrict__ x, const T* __restrict__ r, const T* __restrict__ g, const float* __restrict__ rate,
                            const float* state_in, T* __restrict__ out, float* state_out, int N, int C, int slabs) {
    constexpr int V = Piece<T>::V, P2 = V / 2, kRun = kGroups * TOK;
    extern __shared__ uint4 stage[];                             // [2][3][TOK][kThreads]
    __shared__ Joins<P2, PARTS> sm;
    enter_dependent();
    const int tid = threadIdx.x, lane = tid & 31;
    const int rank = PARTS > 1 ? (int)cluster_rank() : 0;
    const int work = blockIdx.x / PARTS, b = work / slabs;
    const int c0 = (work - b * slabs) * (kLanes * V) + (lane & (kLanes - 1)) * V;
    const bool mine = c0 < C;
    const size_t base = (size_t)b * N * C + (mine ? c0 : 0);
    const int group = tid / kLanes;
    const int steps = (int)(((long long)N + kRun * PARTS - 1) / (kRun * PARTS));

    pair nrate[P2], h[P2];
#pragma unroll
    for (int e = 0; e < P2; ++e) nrate[e] = h[e] = 0;
    if (mine) {
        load_f32<P2>(rate + c0, nrate);
#pragma unroll
        for (int e = 0; e < P2; ++e) nrate[e] = neg2(nrate[e]);
        if (state_in) load_f32<P2>(state_in + (size_t)b * C + c0, h);
    }
    bool small = true;
#pragma unroll
    for (int e = 0; e < P2; ++e) {
        const float2 f = split(nrate[e]);
        small = small && f.x > -0.25f && f.y > -0.25f;
    }
    small = __all_sync(0xffffffffu, small);

    auto first_token = [&](int s) { return (s * (long long)PARTS + rank) * kRun + group * TOK; };
    auto fetch = [&](int s) {
        const long long t0 = first_token(s);
        uint4* to = stage + (size_t)(s & 1) * 3 * TOK * kThreads + tid;
#pragma unroll
        for (int j = 0; j < TOK; ++j) {
            const bool in = mine && t0 + j < N;
            const size_t at = base + (in ? (size_t)(t0 + j) * C : 0);
            copy_async16(to + (0 * TOK + j) * kThreads, r + at, in);
            copy_async16(to + (1 * TOK + j) * kThreads, g + at, in);
            copy_async16(to + (2 * TOK + j) * kThreads, x + at, in);
        }
    };
    fetch(0);
    copy_async_commit();
    if constexpr (PARTS > 1) cluster_arrive_wait();              // every CTA of the cluster runs: its shared memory may be written
    for (int s = 0; s < steps; ++s) {
        if (s + 1 < steps) fetch(s + 1);
        copy_async_commit();
        copy_async_wait<1>();
        const uint4* from = stage + (size_t)(s & 1) * 3 * TOK * kThreads + tid;
        const long long t0 = first_token(s);
        pair a[TOK][P2], u[TOK][P2];                             // a_t, m_t i_t x_t
        auto load = [&](auto small_tag) {
            constexpr bool SMALL = decltype(small_tag)::value;
#pragma unroll
            for (int j = 0; j < TOK; ++j) {
                pair rv[P2], gv[P2], xv[P2];
                Piece<T>::unpack(from[(0 * TOK + j) * kThreads], rv);
                Piece<T>::unpack(from[(1 * TOK + j) * kThreads], gv);
                Piece<T>::unpack(from[(2 * TOK + j) * kThreads], xv);
                const bool in = t0 + j < N;
#pragma unroll
                for (int e = 0; e < P2; ++e) {
                    const pair er = one_plus_exp_neg(rv[e]), eg = one_plus_exp_neg(gv[e]), q = rcp2(mul2(er, eg));
                    const pair p = exp_less_one<SMALL>(mul2(nrate[e], mul2(q, eg)));
                    const float2 m2 = split(one_less_square(p));
                    u[j][e] = mul2(make(root(m2.x), root(m2.y)), mul2(mul2(q, er), xv[e]));
                    a[j][e] = in ? add2(p, both(1.f)) : both(1.f);   // (behind the sequence: nothing happens)
                }
            }
        };
        if (small) load(std::true_type{});
        else load(std::false_type{});
        pair A[P2], H[P2], first[P2];
#pragma unroll
        for (int e = 0; e < P2; ++e) {
            A[e] = a[0][e];
            H[e] = u[0][e];
#pragma unroll
            for (int j = 1; j < TOK; ++j) {
                H[e] = fma2(a[j][e], H[e], u[j][e]);
                A[e] = mul2(A[e], a[j][e]);
            }
        }
        join<P2, PARTS>(sm, s & 1, rank, A, H, h, first);
#pragma unroll
        for (int j = 0; j < TOK; ++j) {
#pragma unroll
            for (int e = 0; e < P2; ++e) first[e] = fma2(a[j][e], first[e], u[j][e]);
            if (mine && t0 + j < N) __stcs(reinterpret_cast<uint4*>(out + base + (size_t)(t0 + j) * C), Piece<T>::pack(first));
        }
    }
    if (state_out && mine && rank == 0 && tid < kLanes) store_f32<P2>(state_out + (size_t)b * C + c0, h);
}

// The scan from the last token to the first: "time" tau = N - 1 - t.  part: [sequences x PARTS][C] sums of drate
template <typename T, int TOK, int PARTS>
__global__ void __launch_bounds__(kThreads, 4)
    gated_recurrence_backward_kernel(const T* __restrict__ x, const T* __restrict__ r, const T* __restrict__ g,
                                     const float* __restrict__ rate, const float* __restrict__ state_in, const T* __restrict__ out,
                                     const T* __restrict__ dout, const float* dstate_out, T* __restrict__ dx, T* __restrict__ dr,
                                     T* __restrict__ dg, float* __restrict__ part, float* dstate_in, int N, int C, int slabs) {
    constexpr int V = Piece<T>::V, P2 = V / 2, kRun = kGroups * TOK;
    extern __shared__ uint4 stage[];                             // [2][5][TOK][kThreads]
    __shared__ Joins<P2, PARTS> sm;
    __shared__ pair sums[kWarps][P2][kLanes];
    enter_dependent();
    const int tid = threadIdx.x, lane = tid & 31;
    const int rank = PARTS > 1 ? (int)cluster_rank() : 0;
    const int work = blockIdx.x / PARTS, b = work / slabs;
    const int c0 = (work - b * slabs) * (kLanes * V) + (lane & (kLanes - 1)) * V;
    const bool mine = c0 < C;
    const size_t base = (size_t)b * N * C + (mine ? c0 : 0);
    const int group = tid / kLanes;
    const int steps = (int)(((long long)N + kRun * PARTS - 1) / (kRun * PARTS));

    pair nrate[P2], E[P2], drate[P2];
#pragma unroll
    for (int e = 0; e < P2; ++e) nrate[e] = E[e] = drate[e] = 0;
    if (mine) {
        load_f32<P2>(rate + c0, nrate);
#pragma unroll
        for (int e = 0; e < P2; ++e) nrate[e] = neg2(nrate[e]);
        if (dstate_out) load_f32<P2>(dstate_out + (size_t)b * C + c0, E);
    }
    bool small = true;
#pragma unroll
    for (int e = 0; e < P2; ++e) {
        const float2 f = split(nrate[e]);
        small = small && f.x > -0.25f && f.y > -0.25f;
    }
    small = __all_sync(0xffffffffu, small);

    auto last_token = [&](int s) { return N - 1 - ((s * (long long)PARTS + rank) * kRun + group * TOK); };
    auto fetch = [&](int s) {
        const long long t0 = last_token(s);
        uint4* to = stage + (size_t)(s & 1) * 5 * TOK * kThreads + tid;
#pragma unroll
        for (int j = 0; j < TOK; ++j) {
            const bool in = mine && t0 - j >= 0, prev = mine && t0 - j >= 1;
            const size_t at = base + (in ? (size_t)(t0 - j) * C : 0);
            copy_async16(to + (0 * TOK + j) * kThreads, r + at, in);
            copy_async16(to + (1 * TOK + j) * kThreads, dout + at, in);
            copy_async16(to + (2 * TOK + j) * kThreads, g + at, in);
            copy_async16(to + (3 * TOK + j) * kThreads, x + at, in);
            copy_async16(to + (4 * TOK + j) * kThreads, out + (prev ? at - C : base), prev);
        }
    };
    fetch(0);
    copy_async_commit();
    if constexpr (PARTS > 1) cluster_arrive_wait();              // every CTA of the cluster runs: its shared memory may be written
    for (int s = 0; s < steps; ++s) {
        if (s + 1 < steps) fetch(s + 1);
        copy_async_commit();
        copy_async_wait<1>();
        const uint4* from = stage + (size_t)(s & 1) * 5 * TOK * kThreads + tid;
        const long long t0 = last_token(s);
        pair p[TOK][P2], sg[TOK][P2];                            // a_t - 1, sigmoid(r_t)
        pair A[P2], H[P2], first[P2];
#pragma unroll
        for (int e = 0; e < P2; ++e) {
            A[e] = both(1.f);
            H[e] = 0;
        }
        auto load = [&](auto small_tag) {
            constexpr bool SMALL = decltype(small_tag)::value;
#pragma unroll
            for (int j = 0; j < TOK; ++j) {
                pair rv[P2], dv[P2];
                Piece<T>::unpack(from[(0 * TOK + j) * kThreads], rv);
                Piece<T>::unpack(from[(1 * TOK + j) * kThreads], dv);
                const bool in = t0 - j >= 0;
#pragma unroll
                for (int e = 0; e < P2; ++e) {
                    sg[j][e] = rcp2(one_plus_exp_neg(rv[e]));
                    const pair q = exp_less_one<SMALL>(mul2(nrate[e], sg[j][e]));
                    p[j][e] = in ? q : 0;                        // (before the sequence: nothing happens)
                    const pair a = add2(p[j][e], both(1.f));
                    H[e] = mul2(a, add2(H[e], dv[e]));
                    A[e] = mul2(A[e], a);
                }
            }
        };
        if (small) load(std::true_type{});
        else load(std::false_type{});
        join<P2, PARTS>(sm, s & 1, rank, A, H, E, first);
#pragma unroll
        for (int j = 0; j < TOK; ++j) {
            pair dv[P2], gv[P2], xv[P2], hv[P2], ox[P2], orr[P2], og[P2];
            Piece<T>::unpack(from[(1 * TOK + j) * kThreads], dv);
            Piece<T>::unpack(from[(2 * TOK + j) * kThreads], gv);
            Piece<T>::unpack(from[(3 * TOK + j) * kThreads], xv);
            Piece<T>::unpack(from[(4 * TOK + j) * kThreads], hv);
            if (mine && t0 - j == 0 && state_in) load_f32<P2>(state_in + (size_t)b * C + c0, hv);
            const bool in = mine && t0 - j >= 0;
#pragma unroll
            for (int e = 0; e < P2; ++e) {
                const pair G = add2(dv[e], first[e]), a = add2(p[j][e], both(1.f));
                const pair i = rcp2(one_plus_exp_neg(gv[e]));
                const pair m2 = one_less_square(p[j][e]);
                const float2 f = split(m2);
                // 1 / m; where nothing decays (m = 0) a number so large that products with it stay finite
                const pair im = make(rroot(max_nan(f.x, 1e-36f)), rroot(max_nan(f.y, 1e-36f)));
                const pair Gi = mul2(G, i), Gmi = mul2(Gi, mul2(m2, im));
                ox[e] = Gmi;
                og[e] = mul2(mul2(Gmi, xv[e]), fma2(neg2(i), both(1.f), both(1.f)));
                // dlog a = a (G h - a / m G i x)
                const pair dla = mul2(a, fma2(G, hv[e], neg2(mul2(mul2(a, im), mul2(Gi, xv[e])))));
                const pair ds = mul2(dla, sg[j][e]);
                if (in) drate[e] = add2(drate[e], neg2(ds));
                orr[e] = mul2(mul2(nrate[e], ds), fma2(neg2(sg[j][e]), both(1.f), both(1.f)));
                first[e] = mul2(a, G);
            }
            if (in) {
                const size_t at = base + (size_t)(t0 - j) * C;
                __stcs(reinterpret_cast<uint4*>(dx + at), Piece<T>::pack(ox));
                __stcs(reinterpret_cast<uint4*>(dr + at), Piece<T>::pack(orr));
                __stcs(reinterpret_cast<uint4*>(dg + at), Piece<T>::pack(og));
            }
        }
    }
    if (dstate_in && mine && rank == 0 && tid < kLanes) store_f32<P2>(dstate_in + (size_t)b * C + c0, E);
    // drate over the CTA's tokens: the warp's groups, then the warps
#pragma unroll
    for (int e = 0; e < P2; ++e) {
#pragma unroll
        for (int d = kLanes; d < 32; d *= 2) drate[e] = add2(drate[e], __shfl_xor_sync(0xffffffffu, drate[e], d));
        if (lane < kLanes) sums[tid >> 5][e][lane] = drate[e];
    }
    __syncthreads();
    if (tid < kLanes && mine) {
        pair t[P2];
#pragma unroll
        for (int e = 0; e < P2; ++e) t[e] = add2(add2(sums[0][e][tid], sums[1][e][tid]), add2(sums[2][e][tid], sums[3][e][tid]));
        store_f32<P2>(part + ((size_t)b * PARTS + rank) * C + c0, t);
    }
}

// One token: 16 bytes of io values per thread
template <typename T>
__global__ void __launch_bounds__(kThreads)
    gated_recurrence_step_kernel(const T* __restrict__ x, const T* __restrict__ r, const T* __restrict__ g, const float* __restrict__ rate,
                                 const float* state_in, T* __restrict__ out, float* state_out, long long pieces, int per_row) {
    constexpr int V = Piece<T>::V, P2 = V / 2;
    enter_dependent();
    const long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (i >= pieces) return;
    const int c0 = (int)(i % per_row) * V;
    const uint4 ru = __ldcs(reinterpret_cast<const uint4*>(r) + i), gu = __ldcs(reinterpret_cast<const uint4*>(g) + i),
                xu = __ldcs(reinterpret_cast<const uint4*>(x) + i);
    pair h[P2], nrate[P2], rv[P2], gv[P2], xv[P2];
#pragma unroll
    for (int e = 0; e < P2; ++e) h[e] = 0;
    if (state_in) load_f32<P2>(state_in + i * V, h);
    load_f32<P2>(rate + c0, nrate);
    Piece<T>::unpack(ru, rv);
    Piece<T>::unpack(gu, gv);
    Piece<T>::unpack(xu, xv);
#pragma unroll
    for (int e = 0; e < P2; ++e) {
        const pair er = one_plus_exp_neg(rv[e]), eg = one_plus_exp_neg(gv[e]), q = rcp2(mul2(er, eg));
        const pair p = exp_less_one<false>(mul2(neg2(nrate[e]), mul2(q, eg)));
        const float2 m2 = split(one_less_square(p));
        h[e] = fma2(add2(p, both(1.f)), h[e], mul2(make(root(m2.x), root(m2.y)), mul2(mul2(q, er), xv[e])));
    }
    if (state_out) store_f32<P2>(state_out + i * V, h);
    __stcs(reinterpret_cast<uint4*>(out) + i, Piece<T>::pack(h));
}

namespace {
constexpr int kTok = 4;

// CTAs per sequence and slab
int parts_for(long long units, int N) {
    int parts = 1;
    while (parts < 8 && units * parts < 4 * kSMs && (long long)parts * kGroups * kTok < N) parts *= 2;
    return parts;
}
int slabs_of(int C, based_dtype io) {
    const int per = kLanes * (io == BASED_F32 ? 4 : 8);
    return (int)(((long long)C + per - 1) / per);
}
template <typename K> cudaError_t allow_smem(K kernel, size_t bytes, std::atomic<bool> (&done)[64]) {
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || dev < 0 || dev >= 64) return e != cudaSuccess ? e : cudaErrorInvalidDevice;
    if (done[dev].load(std::memory_order_acquire)) return cudaSuccess;
    const cudaError_t f = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (f == cudaSuccess) done[dev].store(true, std::memory_order_release);
    return f;
}
template <typename F> based_status with_parts(int parts, F f) {
    switch (parts) {
        case 1: return f(std::integral_constant<int, 1>{});
        case 2: return f(std::integral_constant<int, 2>{});
        case 4: return f(std::integral_constant<int, 4>{});
        default: return f(std::integral_constant<int, 8>{});
    }
}
template <int TOK> constexpr size_t stage_bytes(int arrays) { return (size_t)2 * arrays * TOK * kThreads * 16; }

template <typename T>
based_status forward_t(const void* x, const void* r, const void* g, const float* rate, const float* state_in, void* out,
                       float* state_out, int B, int N, int C, based_dtype io, cudaStream_t stream) {
    const int slabs = slabs_of(C, io);
    return with_parts(parts_for((long long)B * slabs, N), [&](auto tag) {
        constexpr int PARTS = decltype(tag)::value;
        static std::atomic<bool> ready[64];
        constexpr size_t smem = stage_bytes<kTok>(3);
        auto kernel = gated_recurrence_kernel<T, kTok, PARTS>;
        cudaError_t e = allow_smem(kernel, smem, ready);
        if (e == cudaSuccess)
            e = launch_ex(kernel, dim3((unsigned)((long long)B * slabs * PARTS)), dim3(kThreads), smem, PARTS, true, stream,
                          static_cast<const T*>(x), static_cast<const T*>(r), static_cast<const T*>(g), rate, state_in,
                          static_cast<T*>(out), state_out, N, C, slabs);
        note_launch();
        const based_status st = check_launch("gated_recurrence_kernel");
        return e == cudaSuccess ? st : BASED_ERR_CUDA;
    });
}
template <typename T>
based_status backward_t(const void* x, const void* r, const void* g, const float* rate, const float* state_in, const void* out,
                        const void* dout, const float* dstate_out, void* dx, void* dr, void* dg, float* drate, float* dstate_in,
                        int B, int N, int C, float* part, based_dtype io, cudaStream_t stream) {
    const int slabs = slabs_of(C, io), parts = parts_for((long long)B * slabs, N);
    const based_status st = with_parts(parts, [&](auto tag) {
        constexpr int PARTS = decltype(tag)::value;
        static std::atomic<bool> ready[64];
        constexpr size_t smem = stage_bytes<kTok>(5);
        auto kernel = gated_recurrence_backward_kernel<T, kTok, PARTS>;
        cudaError_t e = allow_smem(kernel, smem, ready);
        if (e == cudaSuccess)
            e = launch_ex(kernel, dim3((unsigned)((long long)B * slabs * PARTS)), dim3(kThreads), smem, PARTS, true, stream,
                          static_cast<const T*>(x), static_cast<const T*>(r), static_cast<const T*>(g), rate, state_in,
                          static_cast<const T*>(out), static_cast<const T*>(dout), dstate_out, static_cast<T*>(dx),
                          static_cast<T*>(dr), static_cast<T*>(dg), part, dstate_in, N, C, slabs);
        note_launch();
        const based_status s = check_launch("gated_recurrence_backward_kernel");
        return e == cudaSuccess ? s : BASED_ERR_CUDA;
    });
    if (st != BASED_OK) return st;
    return launch_column_sums(part, (long long)B * parts, C, drate, C, nullptr, stream);
}
}  // namespace

long long gated_recurrence_blocks(int B, int N, int C, based_dtype io) {
    const long long units = (long long)B * slabs_of(C, io);
    return units * parts_for(units, N);
}
size_t gated_recurrence_backward_bytes(int B, int N, int C, based_dtype io) {
    return (size_t)B * parts_for((long long)B * slabs_of(C, io), N) * C * sizeof(float);
}

based_status launch_gated_recurrence(const void* x, const void* r, const void* g, const float* rate, const float* state_in, void* out,
                                     float* state_out, int B, int N, int C, based_dtype io, cudaStream_t stream) {
    if (N > 1) {
        return io == BASED_F32 ? forward_t<float>(x, r, g, rate, state_in, out, state_out, B, N, C, io, stream)
                               : forward_t<__nv_bfloat16>(x, r, g, rate, state_in, out, state_out, B, N, C, io, stream);
    }
    auto step = [&](auto zero) {
        using T = decltype(zero);
        const int per_row = C / Piece<T>::V;
        const long long pieces = (long long)B * per_row;
        return launch_ex(gated_recurrence_step_kernel<T>, dim3((unsigned)((pieces + kThreads - 1) / kThreads)), dim3(kThreads), 0, 1,
                         true, stream, static_cast<const T*>(x), static_cast<const T*>(r), static_cast<const T*>(g), rate, state_in,
                         static_cast<T*>(out), state_out, pieces, per_row);
    };
    const cudaError_t e = io == BASED_F32 ? step(0.f) : step(__nv_bfloat16{});
    note_launch();
    const based_status st = check_launch("gated_recurrence_step_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}

based_status launch_gated_recurrence_backward(const void* x, const void* r, const void* g, const float* rate, const float* state_in,
                                              const void* out, const void* dout, const float* dstate_out, void* dx, void* dr, void* dg,
                                              float* drate, float* dstate_in, int B, int N, int C, float* part, based_dtype io,
                                              cudaStream_t stream) {
    return io == BASED_F32 ? backward_t<float>(x, r, g, rate, state_in, out, dout, dstate_out, dx, dr, dg, drate, dstate_in, B, N, C,
                                               part, io, stream)
                           : backward_t<__nv_bfloat16>(x, r, g, rate, state_in, out, dout, dstate_out, dx, dr, dg, drate, dstate_in, B,
                                                       N, C, part, io, stream);
}

}  // namespace based
