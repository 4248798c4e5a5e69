// based_gated_recurrence_forward / _step / _backward: the gated linear recurrence, a token mixer with one fp32 state per
// channel.  Per sequence and channel, from the state given (or 0):
//
//   s = sigmoid(r),  a = exp(-rate s),  m = sqrt(1 - a^2),     h_t = a_t h_{t-1} + m_t sigmoid(g_t) x_t
//
// A run of tokens maps the state before it to the state behind it by h -> A h + H, and two runs in a row join to
// (A2 A1, A2 H1 + H2).  A thread takes TOK consecutive tokens of 4 channels; the two token groups of a warp join by a shuffle, the
// warps of a CTA and the CTAs of a cluster through shared memory, and every thread then replays its own tokens from the state that
// reaches it.  So the inputs are read once, whatever the sequence's length, and the loop along the sequence carries nothing but the
// state.  The backward pass is the same scan from the last token to the first, of
//
//   E_t = a_t (dout_t + E_{t+1}),     G_t = dout_t + E_{t+1} the gradient of h_t,
//   dx = G m i,  dg = G m x i (1 - i),  dlog a = a G h_{t-1} - (a^2 / m) G i x,  dr = -rate dlog a s (1 - s),
//   drate = -sum dlog a s  (i = sigmoid(g); h_{t-1} is read from the output that the caller kept).
//
// HBM bound by its bytes (4 values a token and channel forward, 8 backward), with little to spare: at the pace of HBM an SM has 43 cycles
// for 32 elements forward on a sub-core, and the element's 3 special-function calls take 24 of them, its multiply-adds 24, which
// together come to 31 at best (measured, without loads).  So one reciprocal root serves both gates and the root of 1 - a^2, cubics
// stand for what is left of the exponential where all rates of a slab are at most 1/4 (else 5 calls), two channels share an instruction
// (half the issue slots, the same pipe time), and tiles of tokens x 128 bytes come by TMA, which needs no address arithmetic and reads
// views with strides as they lie.
// B8 N4096 C2048 bf16, on two cards: forward 114 and 119 us = 4.7 and 4.5 TB/s (256 CTAs on 148 SMs: two on most, which is what bounds
// it; its loads and stores without the arithmetic take 87, the arithmetic without them 97), backward 204 and 222 us = 5.3 and 4.8 TB/s;
// with rates up to 1 on the first card 139 and 235 us.  B1 N32768 C1000 fp32 forward 92 and 99 us = 5.7 and 5.3 TB/s.
#include <type_traits>

#include "common.cuh"
#include "pairs.cuh"
#include "sm100.cuh"

namespace based {
using namespace pairs;
using namespace sm100;

namespace {
constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kV = 4, kP = kV / 2;               // channels of a thread, and pairs of them
// threads side by side, whose channels make a tile's rows 128 bytes; groups of TOK consecutive tokens
template <typename T> __host__ __device__ constexpr int lanes_of() { return sizeof(T) == 4 ? 8 : 16; }
template <typename T> __host__ __device__ constexpr int slab_of() { return lanes_of<T>() * kV; }
template <typename T> __host__ __device__ constexpr int groups_of() { return kThreads / lanes_of<T>(); }
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
__device__ __forceinline__ float max_nan(float x, float y) {
    float z;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
    return z;
}

// Four values of a row, as two pairs
template <typename T> struct Four;
// A gate is taken as -41 at least, so that exp(-x) stays below 2^60 (see Gates): a sigmoid below 2^-59 counts as 2^-59.  A NaN stays one.
constexpr float kLeast = -41.f;
template <> struct Four<float> {
    using Raw = float4;
    static __device__ __forceinline__ void values(const Raw& u, pair (&x)[kP]) {
        x[0] = make(u.x, u.y);
        x[1] = make(u.z, u.w);
    }
    static __device__ __forceinline__ Raw gate(const Raw& u) {
        return make_float4(max_nan(u.x, kLeast), max_nan(u.y, kLeast), max_nan(u.z, kLeast), max_nan(u.w, kLeast));
    }
    static __device__ __forceinline__ Raw pack(const pair (&x)[kP]) {
        const float2 a = split(x[0]), b = split(x[1]);
        return make_float4(a.x, a.y, b.x, b.y);
    }
};
template <> struct Four<__nv_bfloat16> {
    using Raw = uint2;
    static __device__ __forceinline__ void values(const Raw& u, pair (&x)[kP]) {
        x[0] = make(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u));
        x[1] = make(__uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
    }
    static __device__ __forceinline__ Raw gate(Raw u) {
        constexpr uint32_t least = 0xc224c224u;                      // -41 twice
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(u.x) : "r"(least));
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(u.y) : "r"(least));
        return u;
    }
    static __device__ __forceinline__ Raw pack(const pair (&x)[kP]) {
        const float2 a = split(x[0]), b = split(x[1]);
        const __nv_bfloat162 lo = __floats2bfloat162_rn(a.x, a.y), hi = __floats2bfloat162_rn(b.x, b.y);
        return make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    }
};
template <typename T> __device__ __forceinline__ void values4(const void* p, pair (&x)[kP]) {
    Four<T>::values(*static_cast<const typename Four<T>::Raw*>(p), x);
}
template <typename T> __device__ __forceinline__ void gate4(const void* p, pair (&x)[kP]) {
    Four<T>::values(Four<T>::gate(*static_cast<const typename Four<T>::Raw*>(p)), x);
}
template <typename T> __device__ __forceinline__ void write4(T* p, const pair (&x)[kP]) {
    __stcs(reinterpret_cast<typename Four<T>::Raw*>(p), Four<T>::pack(x));
}

// exp(-x)
__device__ __forceinline__ pair exp_neg(pair x) {
    const float2 t = split(mul2(x, both(-kLog2e)));
    return make(ex2(t.x), ex2(t.y));
}
__device__ __forceinline__ pair rroot2(pair x) {
    const float2 t = split(x);
    return make(rroot(t.x), rroot(t.y));
}
__device__ __forceinline__ pair sigmoid(pair x) {
    const float2 t = split(add2(exp_neg(x), both(1.f)));
    return make(rcp(t.x), rcp(t.y));
}
// Both gates of an element from one reciprocal root: with A = 1 + exp(-r), B = 1 + exp(-g) it is t = A^-1/2 B^-1 = sqrt(sigmoid(r))
// sigmoid(g), and w = t B the root of sigmoid(r), which is what sqrt(1 - a^2) holds of r.  B is taken times 2^-30 (t comes out
// times 2^30), so that A B^2, which would reach 2^178, stays below 2^119.
constexpr float kDown = 9.313225746154785e-10f;                      // 2^-30
struct Gates {
    pair A, t, w;
};
__device__ __forceinline__ Gates gates(pair r, pair g) {
    Gates z;
    z.A = add2(exp_neg(r), both(1.f));
    const pair B = fma2(exp_neg(g), both(kDown), both(kDown));
    z.t = rroot2(mul2(z.A, mul2(B, B)));
    z.w = mul2(z.t, B);
    return z;
}
// On -1/4 <= la <= 0, by the cubics that interpolate them at the interval's Chebyshev points, coefficients rounded to fp32:
// (exp(la) - 1) / la (off by 2.6e-7 relative at most) and sqrt((1 - exp(2 la)) / (-2 la)) (4.4e-7)
__device__ __forceinline__ pair cubic(pair x, float c0, float c1, float c2, float c3) {
    return fma2(x, fma2(x, fma2(x, both(c3), both(c2)), both(c1)), both(c0));
}
__device__ __forceinline__ pair slope(pair la) { return cubic(la, 0.999999762f, 0.499969989f, 0.166062251f, 0.0377289727f); }
__device__ __forceinline__ pair share(pair la) { return cubic(la, 0.999999642f, 0.499950707f, 0.207340196f, 0.0560273491f); }
// A decay a = exp(la) and p = a - 1, both with all their digits: p near a = 1, so that 1 - a^2 = -p (2 + p) keeps them, and a below la =
// -1/4, where 1 + (a - 1) would be off by 2^-25, which is all there is of a fast decay
__device__ __forceinline__ void decay(pair la, pair& a, pair& p) {
    const pair f2 = mul2(la, slope(la)), f1 = add2(f2, both(1.f));
    const float2 l = split(la), f = split(f2), g = split(f1), e = split(mul2(la, both(kLog2e)));
    const pair x2 = make(ex2(e.x), ex2(e.y)), y2 = add2(x2, both(-1.f));
    const float2 x = split(x2), y = split(y2);
    const bool u = l.x > -0.25f, v = l.y > -0.25f;
    a = make(u ? g.x : x.x, v ? g.y : x.y);
    p = make(u ? f.x : y.x, v ? f.y : y.y);
}
// The one of the two that has them, to keep in one register: p has its sign bit set, -0 included, and a has not.  (No rate is taken as
// +0 for that, see minus_rate.)  SMALL: la >= -1/4, always p
template <bool SMALL> __device__ __forceinline__ pair decay_kept(pair la) {
    const pair f2 = mul2(la, slope(la));
    if constexpr (SMALL) return f2;
    const float2 l = split(la), f = split(f2), e = split(mul2(la, both(kLog2e)));
    return make(l.x > -0.25f ? f.x : ex2(e.x), l.y > -0.25f ? f.y : ex2(e.y));
}
// 1 where a - 1 is kept, else 0
template <bool SMALL> __device__ __forceinline__ pair decay_one(pair v) {
    if constexpr (SMALL) return both(1.f);
    const float2 x = split(v);
    return make(__int_as_float((__float_as_int(x.x) >> 31) & 0x3f800000), __int_as_float((__float_as_int(x.y) >> 31) & 0x3f800000));
}
template <bool SMALL> __device__ __forceinline__ pair decay_stay() { return SMALL ? 0 : 0x8000000080000000ull; }      // a = 1
__device__ __forceinline__ pair minus_rate(pair rate) {
    const float2 r = split(rate);
    return make(r.x == 0.f ? -0.f : -r.x, r.y == 0.f ? -0.f : -r.y);
}
// 1 - a^2 from p = a - 1
__device__ __forceinline__ pair one_less_square(pair p) { return mul2(p, fma2(p, both(-1.f), both(-2.f))); }
// Decay and input of a token: a = exp(la), u = sqrt(1 - a^2) sigmoid(g) x, la = -rate sigmoid(r).  SMALL: la >= -1/4, and
// sqrt(1 - a^2) = sqrt(-2 la) share(la) = sqrt(2 rate) w share(la); c: sqrt(2 rate) 2^-30
template <bool SMALL>
__device__ __forceinline__ void token(const Gates& z, pair nrate, pair c, pair x, pair& a, pair& u) {
    const pair la = mul2(nrate, mul2(z.w, z.w));
    if constexpr (SMALL) {
        a = fma2(la, slope(la), both(1.f));
        u = mul2(mul2(z.t, c), mul2(x, share(la)));              // (t's 2^30 never meets x, which may be large)
    } else {
        pair p;
        decay(la, a, p);
        const float2 m2 = split(one_less_square(p));
        u = mul2(make(root(m2.x), root(m2.y)), mul2(mul2(mul2(z.t, both(kDown)), mul2(z.A, z.w)), x));
    }
}
// whether the rates of all threads keep -rate sigmoid in the cubics' range
__device__ __forceinline__ bool all_small(const pair (&nrate)[kP]) {
    const float2 a = split(nrate[0]), b = split(nrate[1]);
    return __syncthreads_and(a.x >= -0.25f && a.y >= -0.25f && b.x >= -0.25f && b.y >= -0.25f);
}
// sqrt(2 rate) times f
__device__ __forceinline__ pair root_rate(pair nrate, float f) {
    const float2 r = split(nrate);
    return make(sqrtf(-2.f * r.x) * f, sqrtf(-2.f * r.y) * f);
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive_wait() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// 16 bytes into the same place of another CTA's shared memory, counted by its barrier
__device__ __forceinline__ void store_remote(const void* own, uint64_t* own_bar, uint32_t rank, pair x, pair y) {
    uint32_t addr, bar;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(smem_u32(own)), "r"(rank));
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(bar) : "r"(smem_u32(own_bar)), "r"(rank));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b64 [%0], {%1, %2}, [%3];" ::"r"(addr), "l"(x), "l"(y), "r"(bar)
                 : "memory");
}

// What a CTA shares.  The joins of a step use one of two sets in turn: a set is written again two steps on, when every thread has
// passed the barrier of the step between and so has read it.
template <int LANES, int PARTS> struct Shared {
    ulonglong2 warp[2][kWarps][2][LANES];                        // A, H of a warp's tokens
    ulonglong2 part[2][PARTS > 1 ? PARTS : 1][2][LANES];         // of a CTA's
    pair sums[kWarps][kP][LANES];
    uint64_t full[4], arrived[2];                                // a stage's tiles; the parts of a set
    uint32_t abort_flag;
};
// A, H: what the thread's tokens do to the state.  h: the state before this step, on return the one behind it.  first: the state
// that reaches the thread's first token.  after_barrier: run once every thread of the CTA has come this far.
template <int LANES, int PARTS, typename F>
__device__ __forceinline__ bool join(Shared<LANES, PARTS>& sm, int step, int rank, pair (&A)[kP], pair (&H)[kP], pair (&h)[kP],
                                     pair (&first)[kP], F after_barrier) {
    constexpr int kPer = 32 / LANES;                             // groups of a warp: 2 or 4
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = lane & (LANES - 1), turn = step & 1;
    // over the warp's groups, inclusive; then exclusive (with two groups the upper one has what it needs from the first shuffle)
    pair xa[kP], xh[kP];
#pragma unroll
    for (int d = LANES; d < 32; d *= 2) {
#pragma unroll
        for (int e = 0; e < kP; ++e) {
            xa[e] = shfl_up2(A[e], d);
            xh[e] = shfl_up2(H[e], d);
            if (lane >= d) {
                H[e] = fma2(A[e], xh[e], H[e]);
                A[e] = mul2(A[e], xa[e]);
            }
        }
    }
    if (lane >= 32 - LANES) {
        sm.warp[turn][warp][0][col] = make_ulonglong2(A[0], A[1]);
        sm.warp[turn][warp][1][col] = make_ulonglong2(H[0], H[1]);
    }
    if constexpr (kPer > 2) {
#pragma unroll
        for (int e = 0; e < kP; ++e) {
            xa[e] = shfl_up2(A[e], LANES);
            xh[e] = shfl_up2(H[e], LANES);
        }
    }
    __syncthreads();
    after_barrier();
    bool ok = true;
    pair x[kP];                                                  // the state that reaches the warp
    if constexpr (PARTS > 1) {
        // the CTA's total, and of it what lies before the warp
        pair ta[kP] = {both(1.f), both(1.f)}, th[kP] = {0, 0}, pa[kP], ph[kP];
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w == warp) {
#pragma unroll
                for (int e = 0; e < kP; ++e) {
                    pa[e] = ta[e];
                    ph[e] = th[e];
                }
            }
            const ulonglong2 a = sm.warp[turn][w][0][col], b = sm.warp[turn][w][1][col];
            th[0] = fma2(a.x, th[0], b.x);
            th[1] = fma2(a.y, th[1], b.y);
            ta[0] = mul2(a.x, ta[0]);
            ta[1] = mul2(a.y, ta[1]);
        }
        // it goes to every CTA of the cluster
        if (threadIdx.x == 0) mbar_arrive_expect_tx(&sm.arrived[turn], PARTS * 2 * LANES * 16);
#pragma unroll
        for (int to = 0; to < PARTS; ++to) {
            if ((to & (kWarps - 1)) != warp) continue;
            if (lane < LANES) store_remote(&sm.part[turn][rank][0][col], &sm.arrived[turn], to, ta[0], ta[1]);
            else if (lane < 2 * LANES) store_remote(&sm.part[turn][rank][1][col], &sm.arrived[turn], to, th[0], th[1]);
        }
        ok = mbar_wait(&sm.arrived[turn], (step >> 1) & 1, &sm.abort_flag);
        pair hs[kP];
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
            if (q == rank) {
#pragma unroll
                for (int e = 0; e < kP; ++e) hs[e] = h[e];
            }
            const ulonglong2 a = sm.part[turn][q][0][col], b = sm.part[turn][q][1][col];
            h[0] = fma2(a.x, h[0], b.x);
            h[1] = fma2(a.y, h[1], b.y);
        }
#pragma unroll
        for (int e = 0; e < kP; ++e) x[e] = fma2(pa[e], hs[e], ph[e]);
    } else {
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w == warp) {
#pragma unroll
                for (int e = 0; e < kP; ++e) x[e] = h[e];
            }
            const ulonglong2 a = sm.warp[turn][w][0][col], b = sm.warp[turn][w][1][col];
            h[0] = fma2(a.x, h[0], b.x);
            h[1] = fma2(a.y, h[1], b.y);
        }
    }
#pragma unroll
    for (int e = 0; e < kP; ++e) first[e] = lane < LANES ? x[e] : fma2(xa[e], x[e], xh[e]);
    return ok;
}
template <int LANES, int PARTS> __device__ __forceinline__ void begin(Shared<LANES, PARTS>& sm) {
    if (threadIdx.x == 0) {
        for (uint64_t& bar : sm.full) mbar_init(&bar, 1);
        for (int s = 0; s < 2; ++s) mbar_init(&sm.arrived[s], 1);
        sm.abort_flag = 0;
        fence_mbar_init();
    }
    __syncthreads();
    if constexpr (PARTS > 1) cluster_arrive_wait();              // every CTA of the cluster runs, its barriers are set up
}
// Waits that have run out leave a flag and the loops run on without waiting (every thread still meets every barrier); copies that
// may be under way then get time to land.
template <int LANES, int PARTS> __device__ __forceinline__ void finish(Shared<LANES, PARTS>& sm, bool ok, unsigned int* err) {
    if (!ok) atomicOr(err, 1u);
    __syncthreads();
    if (*(volatile uint32_t*)&sm.abort_flag) {
        for (int it = 0; it < 200; ++it) __nanosleep(1000);
    }
    // No CTA leaves before what others send it has arrived; and every thread of the cluster has read the state that it started from, whose
    // place the new one may take
    if constexpr (PARTS > 1) cluster_arrive_wait();
}
// Tokens per thread, stages of tiles, and CTAs that an SM holds.  us, tokens x CTAs per SM: B8 N4096 C2048 bf16 forward 8 x 3 119, 8 x 4 123,
// 4 x 4 136, 16 x 2 121 (more tokens spread a join over more elements, more registers keep constants where they are), backward 4 x 3
// 217, 4 x 4 252, 2 x 5 271; B1 N32768 C1000 fp32 8 x 2 98, 4 x 4 121; backward B3 N1111 C1000 fp32 2 x 3 27, 4 x 1 39.  More
// stages change nothing.
template <typename T, bool BACK> struct Plan;
template <> struct Plan<__nv_bfloat16, false> { static constexpr int kTok = 8, kStages = 2, kBlocks = 3; };
template <> struct Plan<float, false> { static constexpr int kTok = 8, kStages = 2, kBlocks = 2; };
template <> struct Plan<__nv_bfloat16, true> { static constexpr int kTok = 4, kStages = 3, kBlocks = 3; };
template <> struct Plan<float, true> { static constexpr int kTok = 2, kStages = 3, kBlocks = 3; };
// tokens of a step, of one CTA; bytes of a tile
template <typename T, bool BACK> __host__ __device__ constexpr int run_tokens() { return groups_of<T>() * Plan<T, BACK>::kTok; }
template <typename T, bool BACK> __host__ __device__ constexpr uint32_t tile_bytes() { return run_tokens<T, BACK>() * slab_of<T>() * sizeof(T); }
}  // namespace

struct RecurrenceMaps {
    CUtensorMap r, g, x, dout, out;
};

// grid: clusters of PARTS CTAs, one per sequence and slab of channels (64, fp32 32); the CTAs of a cluster take runs of tokens in turn.
template <typename T, int PARTS>
__global__ void __launch_bounds__(kThreads, Plan<T, false>::kBlocks)
    gated_recurrence_kernel(const __grid_constant__ RecurrenceMaps maps, const float* __restrict__ rate, const float* state_in,
                            T* __restrict__ out, float* state_out, unsigned int* err, int N, int C, int slabs) {
    constexpr int TOK = Plan<T, false>::kTok, kStages = Plan<T, false>::kStages, kRun = run_tokens<T, false>(), LANES = lanes_of<T>(), kSlab = slab_of<T>();
    constexpr uint32_t kTile = tile_bytes<T, false>(), kRow = kSlab * sizeof(T);
    extern __shared__ __align__(128) uint8_t stage[];            // [kStages][r, g, x][kRun][kSlab]
    __shared__ Shared<LANES, PARTS> sm;
    begin(sm);
    enter_dependent();
    const int tid = threadIdx.x, lane = tid & (LANES - 1), group = tid / LANES;
    const int rank = PARTS > 1 ? (int)cluster_rank() : 0;
    const int work = blockIdx.x / PARTS, b = work / slabs, slab0 = (work - b * slabs) * kSlab, c0 = slab0 + lane * kV;
    const bool mine = c0 < C;
    const int steps = (int)(((long long)N + kRun * PARTS - 1) / (kRun * PARTS));

    auto fetch = [&](int s) {
        const int st = s % kStages;
        uint8_t* to = stage + st * 3 * kTile;
        const int t0 = (int)((s * (long long)PARTS + rank) * kRun);
        mbar_arrive_expect_tx(&sm.full[st], 3 * kTile);
        tma_load_3d(to, &maps.r, &sm.full[st], slab0, t0, b);
        tma_load_3d(to + kTile, &maps.g, &sm.full[st], slab0, t0, b);
        tma_load_3d(to + 2 * kTile, &maps.x, &sm.full[st], slab0, t0, b);
    };
    if (tid == 0)
        for (int s = 0; s < kStages && s < steps; ++s) fetch(s);
    pair nrate[kP] = {0, 0}, h[kP] = {0, 0};
    if (mine) {
        load_f32<kP>(rate + c0, nrate);
        nrate[0] = minus_rate(nrate[0]);
        nrate[1] = minus_rate(nrate[1]);
        if (state_in) load_f32<kP>(state_in + (size_t)b * C + c0, h);
    }
    T* const to = out + (size_t)b * N * C + c0;
    const pair c[kP] = {root_rate(nrate[0], kDown), root_rate(nrate[1], kDown)};
    bool ok = true;
    auto walk = [&](auto small_tag) {
        for (int s = 0; s < steps; ++s) {
            ok = mbar_wait(&sm.full[s % kStages], (s / kStages) & 1, &sm.abort_flag) && ok;
            const uint8_t* from = stage + (s % kStages) * 3 * kTile + group * TOK * kRow + lane * kV * sizeof(T);
            const long long t0 = (s * (long long)PARTS + rank) * kRun + group * TOK;
            pair a[TOK][kP], u[TOK][kP];                         // a_t, m_t i_t x_t
#pragma unroll
            for (int j = 0; j < TOK; ++j) {
                pair rv[kP], gv[kP], xv[kP];
                gate4<T>(from + j * kRow, rv);
                gate4<T>(from + kTile + j * kRow, gv);
                values4<T>(from + 2 * kTile + j * kRow, xv);
#pragma unroll
                for (int e = 0; e < kP; ++e) token<decltype(small_tag)::value>(gates(rv[e], gv[e]), nrate[e], c[e], xv[e], a[j][e], u[j][e]);
            }
            if (t0 + TOK > N) {                                  // behind the sequence nothing happens (x reads as 0 there)
#pragma unroll
                for (int j = 0; j < TOK; ++j)
#pragma unroll
                    for (int e = 0; e < kP; ++e)
                        if (t0 + j >= N) a[j][e] = both(1.f);
            }
            pair A[kP], H[kP], first[kP];
#pragma unroll
            for (int e = 0; e < kP; ++e) {
                A[e] = a[0][e];
                H[e] = u[0][e];
#pragma unroll
                for (int j = 1; j < TOK; ++j) {
                    H[e] = fma2(a[j][e], H[e], u[j][e]);
                    A[e] = mul2(A[e], a[j][e]);
                }
            }
            ok = join<LANES, PARTS>(sm, s, rank, A, H, h, first, [&] {      // (the stage has been read)
                if (tid == 0 && s + kStages < steps) fetch(s + kStages);
            }) && ok;
#pragma unroll
            for (int j = 0; j < TOK; ++j) {
#pragma unroll
                for (int e = 0; e < kP; ++e) first[e] = fma2(a[j][e], first[e], u[j][e]);
                if (mine && t0 + j < N) write4<T>(to + (size_t)(t0 + j) * C, first);
            }
        }
    };
    if (all_small(nrate)) walk(std::true_type{});
    else walk(std::false_type{});
    finish(sm, ok, err);
    if (state_out && mine && rank == 0 && group == 0) store_f32<kP>(state_out + (size_t)b * C + c0, h);
}

// The scan from the last token to the first: "time" tau = N - 1 - t, tiles lie with the last token of a run below.  part: [sequences
// x PARTS][C] sums of drate
template <typename T, int PARTS>
__global__ void __launch_bounds__(kThreads, Plan<T, true>::kBlocks)
    gated_recurrence_backward_kernel(const __grid_constant__ RecurrenceMaps maps, const float* __restrict__ rate,
                                     const float* __restrict__ state_in, const float* dstate_out, T* __restrict__ dx, T* __restrict__ dr,
                                     T* __restrict__ dg, float* __restrict__ part, float* dstate_in, unsigned int* err, int N, int C, int slabs) {
    constexpr int TOK = Plan<T, true>::kTok, kStages = Plan<T, true>::kStages, kRun = run_tokens<T, true>(), LANES = lanes_of<T>(), kSlab = slab_of<T>();
    constexpr uint32_t kTile = tile_bytes<T, true>(), kRow = kSlab * sizeof(T);
    extern __shared__ __align__(128) uint8_t stage[];            // [kStages][r, dout, g, x, out of the token before][kRun][kSlab]
    __shared__ Shared<LANES, PARTS> sm;
    begin(sm);
    enter_dependent();
    const int tid = threadIdx.x, lane = tid & (LANES - 1), group = tid / LANES;
    const int rank = PARTS > 1 ? (int)cluster_rank() : 0;
    const int work = blockIdx.x / PARTS, b = work / slabs, slab0 = (work - b * slabs) * kSlab, c0 = slab0 + lane * kV;
    const bool mine = c0 < C;
    const int steps = (int)(((long long)N + kRun * PARTS - 1) / (kRun * PARTS));

    auto fetch = [&](int s) {
        const int st = s % kStages;
        uint8_t* to = stage + st * 5 * kTile;
        const int t0 = (int)(N - (s * (long long)PARTS + rank + 1) * kRun);       // (may be below 0: rows before the sequence read as 0)
        mbar_arrive_expect_tx(&sm.full[st], 5 * kTile);
        tma_load_3d(to, &maps.r, &sm.full[st], slab0, t0, b);
        tma_load_3d(to + kTile, &maps.dout, &sm.full[st], slab0, t0, b);
        tma_load_3d(to + 2 * kTile, &maps.g, &sm.full[st], slab0, t0, b);
        tma_load_3d(to + 3 * kTile, &maps.x, &sm.full[st], slab0, t0, b);
        tma_load_3d(to + 4 * kTile, &maps.out, &sm.full[st], slab0, t0 - 1, b);
    };
    if (tid == 0)
        for (int s = 0; s < kStages - 1 && s < steps; ++s) fetch(s);
    pair nrate[kP] = {0, 0}, E[kP] = {0, 0}, drate[kP] = {0, 0};
    if (mine) {
        load_f32<kP>(rate + c0, nrate);
        nrate[0] = minus_rate(nrate[0]);
        nrate[1] = minus_rate(nrate[1]);
        if (dstate_out) load_f32<kP>(dstate_out + (size_t)b * C + c0, E);
    }
    const size_t base = (size_t)b * N * C + c0;
    bool ok = true;
    auto walk = [&](auto small_tag) {
        constexpr bool SMALL = decltype(small_tag)::value;
        for (int s = 0; s < steps; ++s) {
            ok = mbar_wait(&sm.full[s % kStages], (s / kStages) & 1, &sm.abort_flag) && ok;
            // the thread's tokens t0, t0 - 1, ...
            const uint8_t* from = stage + (s % kStages) * 5 * kTile + (kRun - 1 - group * TOK) * kRow + lane * kV * sizeof(T);
            const long long t0 = N - 1 - ((s * (long long)PARTS + rank) * kRun + group * TOK);
            pair v[TOK][kP], sg[TOK][kP];                        // the decay, sigmoid(r_t)
            pair A[kP] = {both(1.f), both(1.f)}, H[kP] = {0, 0}, first[kP];
#pragma unroll
            for (int j = 0; j < TOK; ++j) {
                pair rv[kP], dv[kP];
                gate4<T>(from - j * kRow, rv);
                values4<T>(from + kTile - j * kRow, dv);
#pragma unroll
                for (int e = 0; e < kP; ++e) {
                    sg[j][e] = sigmoid(rv[e]);
                    v[j][e] = decay_kept<SMALL>(mul2(nrate[e], sg[j][e]));
                    if (t0 - j < 0) v[j][e] = decay_stay<SMALL>();             // (before the sequence nothing happens)
                    const pair a = add2(v[j][e], decay_one<SMALL>(v[j][e]));
                    H[e] = mul2(a, add2(H[e], dv[e]));
                    A[e] = mul2(A[e], a);
                }
            }
            ok = join<LANES, PARTS>(sm, s, rank, A, H, E, first, [&] {      // (the stage of the step before has been read)
                if (tid == 0 && s + kStages - 1 < steps) fetch(s + kStages - 1);
            }) && ok;
#pragma unroll
            for (int j = 0; j < TOK; ++j) {
                pair dv[kP], gv[kP], xv[kP], hv[kP], ox[kP], orr[kP], og[kP];
                values4<T>(from + kTile - j * kRow, dv);
                gate4<T>(from + 2 * kTile - j * kRow, gv);
                values4<T>(from + 3 * kTile - j * kRow, xv);
                values4<T>(from + 4 * kTile - j * kRow, hv);
                const bool in = mine && t0 - j >= 0;
                if (in && t0 - j == 0 && state_in) load_f32<kP>(state_in + (size_t)b * C + c0, hv);
#pragma unroll
                for (int e = 0; e < kP; ++e) {
                    const pair one = decay_one<SMALL>(v[j][e]), a = add2(v[j][e], one), i = sigmoid(gv[e]);
                    const pair m2 = one_less_square(SMALL ? v[j][e] : add2(v[j][e], add2(one, both(-1.f))));
                    const float2 f = split(m2);
                    // 1 / m; where nothing decays (m = 0) a number so large that products with it stay finite
                    const pair im = make(rroot(max_nan(f.x, 1e-36f)), rroot(max_nan(f.y, 1e-36f))), m = mul2(m2, im);
                    const pair G = add2(dv[e], first[e]), Gi = mul2(G, i), Gix = mul2(Gi, xv[e]);
                    ox[e] = mul2(Gi, m);
                    og[e] = mul2(mul2(Gix, m), fma2(i, both(-1.f), both(1.f)));
                    // -dlog a = a^2 / m G i x - a G h
                    first[e] = mul2(a, G);
                    const pair nd = fma2(mul2(a, a), mul2(im, Gix), neg2(mul2(first[e], hv[e])));
                    const pair ds = mul2(nd, sg[j][e]);
                    if (in) drate[e] = add2(drate[e], ds);
                    orr[e] = mul2(mul2(nrate[e], ds), fma2(sg[j][e], both(1.f), both(-1.f)));
                }
                if (in) {
                    const size_t at = base + (size_t)(t0 - j) * C;
                    write4<T>(dx + at, ox);
                    write4<T>(dr + at, orr);
                    write4<T>(dg + at, og);
                }
            }
        }
    };
    if (all_small(nrate)) walk(std::true_type{});
    else walk(std::false_type{});
    // drate over the CTA's tokens: the warp's groups, then the warps
#pragma unroll
    for (int e = 0; e < kP; ++e) {
#pragma unroll
        for (int d = LANES; d < 32; d *= 2) drate[e] = add2(drate[e], __shfl_xor_sync(0xffffffffu, drate[e], d));
        if ((tid & 31) < LANES) sm.sums[tid >> 5][e][lane] = drate[e];
    }
    __syncthreads();
    if (group == 0 && mine) {
        pair t[kP];
#pragma unroll
        for (int e = 0; e < kP; ++e) {
            t[e] = sm.sums[0][e][lane];
#pragma unroll
            for (int w = 1; w < kWarps; ++w) t[e] = add2(t[e], sm.sums[w][e][lane]);
        }
        store_f32<kP>(part + ((size_t)b * PARTS + rank) * C + c0, t);
    }
    finish(sm, ok, err);
    if (dstate_in && mine && rank == 0 && group == 0) store_f32<kP>(dstate_in + (size_t)b * C + c0, E);
}

// One token: 4 channels per thread
template <typename T>
__global__ void __launch_bounds__(kThreads)
    gated_recurrence_step_kernel(const Tokens x, const Tokens r, const Tokens g, const float* __restrict__ rate, const float* state_in,
                                 T* __restrict__ out, float* state_out, long long pieces, int per_row) {
    enter_dependent();
    const long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (i >= pieces) return;
    const long long b = i / per_row;
    const int c0 = (int)(i - b * per_row) * kV;
    using Raw = typename Four<T>::Raw;
    auto at = [&](const Tokens& t) { return __ldcs(reinterpret_cast<const Raw*>(static_cast<const T*>(t.data) + b * t.batch_stride + c0)); };
    const Raw ru = at(r), gu = at(g), xu = at(x);
    pair h[kP] = {0, 0}, nrate[kP], rv[kP], gv[kP], xv[kP];
    if (state_in) load_f32<kP>(state_in + i * kV, h);
    load_f32<kP>(rate + c0, nrate);
    Four<T>::values(Four<T>::gate(ru), rv);
    Four<T>::values(Four<T>::gate(gu), gv);
    Four<T>::values(xu, xv);
#pragma unroll
    for (int e = 0; e < kP; ++e) {
        pair a, u;
        token<false>(gates(rv[e], gv[e]), minus_rate(nrate[e]), 0, xv[e], a, u);
        h[e] = fma2(a, h[e], u);
    }
    if (state_out) store_f32<kP>(state_out + i * kV, h);
    write4<T>(out + i * kV, h);
}

namespace {
// CTAs per sequence and slab: as many as are resident at once and the sequence has runs for (each goes along its whole sequence, so
// a second wave would run with the chip half empty).  Up to 8, the clusters that every launch may have; 16 where each CTA has an SM to
// itself (us, 8 / 16: B1 N32000 C256 bf16 forward 108 / 70, backward 205 / 122; with two CTAs per SM, B1 N2000 C1024 backward 20 / 23,
// B3 N1000 C512 7 / 10)
int parts_for(long long units, long long runs, int blocks) {
    int parts = 1;
    while (parts < 8 && units * parts * 2 <= (long long)blocks * kSMs && 2 * parts <= runs) parts *= 2;
    return parts == 8 && units * 16 <= kSMs && 16 <= runs ? 16 : parts;
}
template <typename T> int slabs_of(int C) { return (int)(((long long)C + slab_of<T>() - 1) / slab_of<T>()); }
template <typename T, bool BACK> int parts_of(int B, int N, int C) {
    constexpr int run = run_tokens<T, BACK>();
    return parts_for((long long)B * slabs_of<T>(C), ((long long)N + run - 1) / run, Plan<T, BACK>::kBlocks);
}
// Whether a launch comes in while the grid ahead drains: only one with at most a CTA per SM, and backward of a step or two.  Others crowd on the SMs
// that the grid ahead leaves first and stay there to their end (us behind itself, dependent / plain: bf16 B1 N16000 C1600 97 / 74, backward
// 166 / 133; B8 N4096 C2048 159 / 122; backward B1 N8000 C512 73 / 55, B2 N2000 C512 24 / 20; but B1 N128 C512 3.1 / 3.7, backward 4.4 / 4.9)
template <bool BACK> bool beside(long long ctas, long long steps) { return ctas <= kSMs && (!BACK || steps <= 2); }
template <typename K> cudaError_t allow(K kernel, size_t bytes, int cluster, std::atomic<bool> (&done)[64]) {
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || dev < 0 || dev >= 64) return e != cudaSuccess ? e : cudaErrorInvalidDevice;
    if (done[dev].load(std::memory_order_acquire)) return cudaSuccess;
    cudaError_t f = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (f == cudaSuccess && cluster > 8) f = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (f == cudaSuccess) done[dev].store(true, std::memory_order_release);
    return f;
}
// Whether the device has room for a cluster of 16 of the kernel's CTAs: a whole chip has, the share of one that a process may be given
// need not
template <typename K> bool holds_16(K kernel, size_t bytes, std::atomic<bool> (&known)[64]) {
    int dev = 0, clusters = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
    if (known[dev].load(std::memory_order_acquire)) return true;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = 16;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.gridDim = dim3(16);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    const bool held = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess &&
                      cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                      cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) == cudaSuccess && clusters > 0;
    if (held) known[dev].store(true, std::memory_order_release);
    else (void)cudaGetLastError();
    return held;
}
template <typename F> based_status with_parts(int parts, F f) {
    switch (parts) {
        case 1: return f(std::integral_constant<int, 1>{});
        case 2: return f(std::integral_constant<int, 2>{});
        case 4: return f(std::integral_constant<int, 4>{});
        case 8: return f(std::integral_constant<int, 8>{});
        default: return f(std::integral_constant<int, 16>{});
    }
}

template <typename T>
based_status forward_t(const Tokens& x, const Tokens& r, const Tokens& g, const float* rate, const float* state_in, void* out,
                       float* state_out, int B, int N, int C, cudaStream_t stream) {
    constexpr bool f32 = sizeof(T) == 4;
    const int slabs = slabs_of<T>(C);
    RecurrenceMaps maps;
    unsigned int* err = nullptr;
    constexpr int run = run_tokens<T, false>();
    if (!make_tokens_map(&maps.r, r, f32, B, N, C, slab_of<T>(), run) || !make_tokens_map(&maps.g, g, f32, B, N, C, slab_of<T>(), run) ||
        !make_tokens_map(&maps.x, x, f32, B, N, C, slab_of<T>(), run) || error_word_ptr(&err) != BASED_OK)
        return BASED_ERR_CUDA;
    maps.dout = maps.out = maps.x;
    constexpr size_t smem = Plan<T, false>::kStages * 3 * tile_bytes<T, false>();
    static std::atomic<bool> known16[64];
    int parts = parts_of<T, false>(B, N, C);
    if (parts == 16 && !holds_16(gated_recurrence_kernel<T, 16>, smem, known16)) parts = 8;
    return with_parts(parts, [&](auto tag) {
        constexpr int PARTS = decltype(tag)::value;
        static std::atomic<bool> ready[64];
        auto kernel = gated_recurrence_kernel<T, PARTS>;
        cudaError_t e = allow(kernel, smem, PARTS, ready);
        if (e == cudaSuccess)
            e = launch_ex(kernel, dim3((unsigned)((long long)B * slabs * PARTS)), dim3(kThreads), smem, PARTS, beside<false>((long long)B * slabs * PARTS, 0), stream, maps, rate,
                          state_in, static_cast<T*>(out), state_out, err, N, C, slabs);
        note_launch();
        const based_status st = check_launch("gated_recurrence_kernel");
        return e == cudaSuccess ? st : BASED_ERR_CUDA;
    });
}
template <typename T>
based_status backward_t(const Tokens& x, const Tokens& r, const Tokens& g, const float* rate, const float* state_in, const Tokens& out,
                        const Tokens& dout, const float* dstate_out, void* dx, void* dr, void* dg, float* drate, float* dstate_in, int B,
                        int N, int C, float* part, cudaStream_t stream) {
    constexpr bool f32 = sizeof(T) == 4;
    const int slabs = slabs_of<T>(C);
    RecurrenceMaps maps;
    unsigned int* err = nullptr;
    constexpr int run = run_tokens<T, true>();
    if (!make_tokens_map(&maps.r, r, f32, B, N, C, slab_of<T>(), run) || !make_tokens_map(&maps.g, g, f32, B, N, C, slab_of<T>(), run) ||
        !make_tokens_map(&maps.x, x, f32, B, N, C, slab_of<T>(), run) || !make_tokens_map(&maps.out, out, f32, B, N, C, slab_of<T>(), run) ||
        !make_tokens_map(&maps.dout, dout, f32, B, N, C, slab_of<T>(), run) || error_word_ptr(&err) != BASED_OK)
        return BASED_ERR_CUDA;
    constexpr size_t smem = Plan<T, true>::kStages * 5 * tile_bytes<T, true>();
    static std::atomic<bool> known16[64];
    int parts = parts_of<T, true>(B, N, C);                      // (the scratch is for that many, or more than needed)
    if (parts == 16 && !holds_16(gated_recurrence_backward_kernel<T, 16>, smem, known16)) parts = 8;
    const based_status st = with_parts(parts, [&](auto tag) {
        constexpr int PARTS = decltype(tag)::value;
        static std::atomic<bool> ready[64];
        auto kernel = gated_recurrence_backward_kernel<T, PARTS>;
        cudaError_t e = allow(kernel, smem, PARTS, ready);
        if (e == cudaSuccess)
            e = launch_ex(kernel, dim3((unsigned)((long long)B * slabs * PARTS)), dim3(kThreads), smem, PARTS,
                          beside<true>((long long)B * slabs * PARTS, ((long long)N + run * PARTS - 1) / (run * PARTS)), stream, maps, rate,
                          state_in, dstate_out, static_cast<T*>(dx), static_cast<T*>(dr), static_cast<T*>(dg), part, dstate_in, err, N, C,
                          slabs);
        note_launch();
        const based_status s = check_launch("gated_recurrence_backward_kernel");
        return e == cudaSuccess ? s : BASED_ERR_CUDA;
    });
    if (st != BASED_OK) return st;
    return launch_column_sums(part, (long long)B * parts, C, drate, C, nullptr, stream);
}
}  // namespace

long long gated_recurrence_blocks(int B, int C, based_dtype io) {
    return io == BASED_F32 ? (long long)B * slabs_of<float>(C) * 8 : (long long)B * slabs_of<__nv_bfloat16>(C) * 8;
}
size_t gated_recurrence_backward_bytes(int B, int N, int C, based_dtype io) {
    const int parts = io == BASED_F32 ? parts_of<float, true>(B, N, C) : parts_of<__nv_bfloat16, true>(B, N, C);
    return (size_t)B * parts * C * sizeof(float);
}

based_status launch_gated_recurrence(const Tokens& x, const Tokens& r, const Tokens& g, const float* rate, const float* state_in, void* out,
                                     float* state_out, int B, int N, int C, based_dtype io, cudaStream_t stream) {
    if (N > 1) {
        return io == BASED_F32 ? forward_t<float>(x, r, g, rate, state_in, out, state_out, B, N, C, stream)
                               : forward_t<__nv_bfloat16>(x, r, g, rate, state_in, out, state_out, B, N, C, stream);
    }
    auto step = [&](auto zero) {
        using T = decltype(zero);
        const int per_row = C / kV;
        const long long pieces = (long long)B * per_row;
        return launch_ex(gated_recurrence_step_kernel<T>, dim3((unsigned)((pieces + kThreads - 1) / kThreads)), dim3(kThreads), 0, 1,
                         true, stream, x, r, g, rate, state_in, static_cast<T*>(out), state_out, pieces, per_row);
    };
    const cudaError_t e = io == BASED_F32 ? step(0.f) : step(__nv_bfloat16{});
    note_launch();
    const based_status st = check_launch("gated_recurrence_step_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}

based_status launch_gated_recurrence_backward(const Tokens& x, const Tokens& r, const Tokens& g, const float* rate, const float* state_in,
                                              const Tokens& out, const Tokens& dout, const float* dstate_out, void* dx, void* dr, void* dg,
                                              float* drate, float* dstate_in, int B, int N, int C, float* part, based_dtype io,
                                              cudaStream_t stream) {
    return io == BASED_F32 ? backward_t<float>(x, r, g, rate, state_in, out, dout, dstate_out, dx, dr, dg, drate, dstate_in, B, N, C,
                                               part, stream)
                           : backward_t<__nv_bfloat16>(x, r, g, rate, state_in, out, dout, dstate_out, dx, dr, dg, drate, dstate_in, B,
                                                       N, C, part, stream);
}

}  // namespace based
