// based_qk_norm_rotate / _backward: what stands between a layer's projections and its attention: every head's query and key
// is normed over its d elements, weighted, and its first 2 n elements turn pairwise with the token's position,
//
//   y = w x / sqrt(mean(x^2) + eps);   pair j: (y_lo cos t - y_hi sin t, y_hi cos t + y_lo sin t), t = position freqs[j],
//
// pairs (j, n + j), or (2 j, 2 j + 1).  The projections hold the heads of a token side by side, [B,L,H,d] (with a token stride:
// they may be slices of one fused projection); the mixers take [B,H,L,d], which is how y is written, so the layout change costs
// no pass of its own.  Backward, from the gradient of y in the mixers' layout to that of x in the projections':
//
//   e = turned back dy,  dw = sum over rows of e x inv,  dx = inv (w e - x inv^2 mean(w e x)),   inv = 1 / sqrt(mean(x^2) + eps).
//
// One pass over rows of 32 bytes to 1 KB: bound by HBM bandwidth.  A row is shared by d / (2 V) threads, each with two 16-byte
// pieces (V values) that hold both elements of its pairs, so only the row's sums cross threads.  A CTA takes up to 32
// consecutive tokens and all their heads: a warp reads pieces of rows that lie a token stride apart and writes rows that lie
// side by side, and the angles of the tokens, the same for all heads, are taken once, into shared memory.  An angle is a
// product in fp64, reduced to a part of a turn there (a far position's angle in fp32 would be off by position x 6e-8), and only
// that part is rounded to fp32 for the sine and cosine.  What is left of HBM's rate goes to the start of each CTA, where it
// waits for the angles and its first rows: those rows are asked for before the angles, and a turn ahead after that.
//
// Measured: bf16, 2 x 32768 tokens, 16 + 16 heads of 64, rotating: 106 us (77 % of the copy rate; 115 with 8 tokens per CTA, 165
// with 4); fp32, 3 x 777 tokens, 16 + 4 heads of 128, 64 of them rotating: 8.6 us (85 %); backward, bf16, 4 x 2048 tokens of
// 16 + 16 heads of 64: 30 us (51 %: latency, 16 warps of 116 registers per SM).  A form with a TMA pipeline through shared memory (4 stages, results stored by TMA) took 117,
// 17 and 50: its rows pass through shared memory twice, and short grids fill no pipeline.
#include <type_traits>

#include "common.cuh"
#include "pairs.cuh"

namespace based {
using namespace pairs;

namespace {
constexpr int kThreads = 128;
constexpr double kTurnsPerRadian = 0.15915494309189533577;

__device__ __forceinline__ pair swap2(pair a) { return (a >> 32) | (a << 32); }

struct Grid {
    int T, TP;                     // threads that share a row, and the power of two they are spaced by
    int TB;                        // tokens per block, a power of two
    int NP;                        // the angles of a token are spaced by that many threads, a power of two
    int blocks;                    // blocks of tokens
};
// Sine and cosine of x half turns, |x| <= 1.  For bf16 io the fast ones (off by 2^-20.5, where the result is rounded by 2^-9 of it)
template <typename T> __device__ __forceinline__ float2 cos_sin(float x) {
    float2 r;
    if constexpr (sizeof(T) == 2) {
        const float a = x * 3.14159265f;
        asm("cos.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(a));
        asm("sin.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(a));
    } else {
        sincospif(x, &r.y, &r.x);
    }
    return r;
}
// The angles of TB tokens from token m0 of the batch on: cos and sin [TB][n] in shared memory
template <typename T> __device__ __forceinline__ void fill_angles(const NormRotate& a, const Grid& gr, int m0, float2* table) {
    const int j = threadIdx.x & (gr.NP - 1), step = kThreads / gr.NP;
    if (j >= a.n) return;
    const double freq = a.freqs[j] * kTurnsPerRadian;
    for (int tok = threadIdx.x / gr.NP; tok < gr.TB; tok += step) {
        const int m = m0 + tok;
        if (m >= a.B * a.L) return;
        double pos;
        if (a.positions && a.per_token) {
            pos = (double)a.positions[m];
        } else {
            const int b = m / a.L, t = m - b * a.L;
            pos = (a.positions ? (double)a.positions[b] : (double)a.start) + (double)t;
        }
        const double turns = pos * freq;
        table[tok * a.n + j] = cos_sin<T>((float)(2.0 * (turns - rint(turns))));
    }
}

// What a thread keeps of its place in a row: pieces va and vb, and its token's angles for them
template <typename T, bool PAIRS> struct Place {
    static constexpr int V = Piece<T>::V, P2 = V / 2;
    int va, vb;                    // pieces
    bool in, turns;                // the thread has pieces; they turn
    // halves: cos, sin of pairs of elements; PAIRS: of one pair each, piece a then b
    pair c[PAIRS ? 2 * P2 : P2], s[PAIRS ? 2 * P2 : P2];

    __device__ __forceinline__ void set(int j, int T_, int n) {
        const int half = n / V;
        in = j < T_;
        turns = j < half;
        va = turns ? j : 2 * half + 2 * (j - half);
        vb = turns ? half + j : va + 1;
    }
    __device__ __forceinline__ void angles(const float2* row) {
        if (!in || !turns) return;
        if constexpr (PAIRS) {
#pragma unroll
            for (int e = 0; e < P2; ++e) {
                const float2 fa = row[va * P2 + e], fb = row[vb * P2 + e];
                c[e] = both(fa.x);
                s[e] = make(-fa.y, fa.y);
                c[P2 + e] = both(fb.x);
                s[P2 + e] = make(-fb.y, fb.y);
            }
        } else {
#pragma unroll
            for (int e = 0; e < P2; ++e) {
                const float2 f0 = row[va * V + 2 * e], f1 = row[va * V + 2 * e + 1];
                c[e] = make(f0.x, f1.x);
                s[e] = make(f0.y, f1.y);
            }
        }
    }
    // BACK: by the opposite angle
    template <bool BACK> __device__ __forceinline__ void turn(pair (&a)[P2], pair (&b)[P2]) const {
        if (!turns) return;
#pragma unroll
        for (int e = 0; e < P2; ++e) {
            if constexpr (PAIRS) {
                const pair sa = BACK ? neg2(s[e]) : s[e], sb = BACK ? neg2(s[P2 + e]) : s[P2 + e];
                a[e] = fma2(a[e], c[e], mul2(swap2(a[e]), sa));
                b[e] = fma2(b[e], c[P2 + e], mul2(swap2(b[e]), sb));
            } else {
                const pair sn = BACK ? neg2(s[e]) : s[e];
                const pair lo = fma2(a[e], c[e], neg2(mul2(b[e], sn)));
                b[e] = fma2(b[e], c[e], mul2(a[e], sn));
                a[e] = lo;
            }
        }
    }
};
template <int P2> __device__ __forceinline__ float dot(const pair (&a)[P2], const pair (&b)[P2], const pair (&c)[P2], const pair (&d)[P2]) {
    pair t = mul2(a[0], c[0]);
#pragma unroll
    for (int e = 1; e < P2; ++e) t = fma2(a[e], c[e], t);
#pragma unroll
    for (int e = 0; e < P2; ++e) t = fma2(b[e], d[e], t);
    const float2 f = split(t);
    return f.x + f.y;
}
template <int P2> __device__ __forceinline__ void weights(const float* w, int va, int vb, bool in, pair (&a)[P2], pair (&b)[P2]) {
#pragma unroll
    for (int e = 0; e < P2; ++e) a[e] = b[e] = both(1.f);
    if (w && in) {
        load_f32<P2>(w + va * 2 * P2, a);
        load_f32<P2>(w + vb * 2 * P2, b);
    }
}
}  // namespace

// grid: blocks of TB tokens; queries and keys
template <typename T, bool PAIRS>
__global__ void __launch_bounds__(kThreads, 4) norm_rotate_kernel(const NormRotate a, const Grid gr, T* __restrict__ out_q, T* __restrict__ out_k) {
    constexpr int V = Piece<T>::V, P2 = V / 2, U = 2;
    extern __shared__ float2 table[];
    enter_dependent();
    const int tid = threadIdx.x, j = tid & (gr.TP - 1), slot = tid / gr.TP;
    const int tok = slot & (gr.TB - 1), h0 = slot / gr.TB, hs = kThreads / gr.TP / gr.TB;
    const int m0 = blockIdx.x * gr.TB, m = m0 + tok;             // (B L < 2^31 - 2^4)
    const bool keys = blockIdx.y != 0;
    const int H = keys ? a.Hk : a.Hq;
    Place<T, PAIRS> at;
    at.set(j, gr.T, a.n);
    const bool live = at.in && m < a.B * a.L;
    const int b = m / a.L, t = m - b * a.L;
    const float per_d = 1.f / (float)a.d;
    const T* row = static_cast<const T*>(keys ? a.k : a.q) + m * (keys ? a.k_stride : a.q_stride);
    T* to = (keys ? out_k : out_q) + ((size_t)b * H * a.L + t) * a.d;
    // rows of U heads at a time, those of the next turn under way while this one's are worked on; the first ones before the angles
    uint4 ua[U], ub[U];
    auto fetch = [&](int hb) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = hb + u * hs + h0;
            ua[u] = ub[u] = make_uint4(0, 0, 0, 0);
            if (live && h < H) {
                ua[u] = __ldcs(reinterpret_cast<const uint4*>(row + (size_t)h * a.d) + at.va);
                ub[u] = __ldcs(reinterpret_cast<const uint4*>(row + (size_t)h * a.d) + at.vb);
            }
        }
    };
    fetch(0);
    pair wa[P2], wb[P2];
    weights<P2>(keys ? a.wk : a.wq, at.va, at.vb, at.in, wa, wb);
    if (a.n) {
        fill_angles<T>(a, gr, m0, table);
        __syncthreads();
    }
    at.angles(table + tok * a.n);
    for (int hb = 0; hb < H; hb += U * hs) {                     // (every thread: the sums cross lanes)
        pair xa[U][P2], xb[U][P2];
        float ss[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Piece<T>::unpack(ua[u], xa[u]);
            Piece<T>::unpack(ub[u], xb[u]);
        }
        if (hb + U * hs < H) fetch(hb + U * hs);
#pragma unroll
        for (int u = 0; u < U; ++u) ss[u] = dot<P2>(xa[u], xb[u], xa[u], xb[u]);
        for (int d = gr.TP / 2; d > 0; d /= 2)
#pragma unroll
            for (int u = 0; u < U; ++u) ss[u] += __shfl_xor_sync(0xffffffffu, ss[u], d);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = hb + u * hs + h0;
            const pair inv = both(rsqrtf(fmaf(ss[u], per_d, a.eps)));
#pragma unroll
            for (int e = 0; e < P2; ++e) {
                xa[u][e] = mul2(mul2(xa[u][e], inv), wa[e]);
                xb[u][e] = mul2(mul2(xb[u][e], inv), wb[e]);
            }
            at.template turn<false>(xa[u], xb[u]);
            if (live && h < H) {
                uint4* dst = reinterpret_cast<uint4*>(to + (size_t)h * a.L * a.d);
                __stcs(dst + at.va, Piece<T>::pack(xa[u]));
                __stcs(dst + at.vb, Piece<T>::pack(xb[u]));
            }
        }
    }
}

// The same rows backward.  part: a row of 2 d sums per block, the queries' and the keys' (null: the weights' gradients are not wanted)
template <typename T, bool PAIRS>
__global__ void __launch_bounds__(kThreads, 4)
    norm_rotate_backward_kernel(const NormRotate a, const Grid gr, const T* __restrict__ gq, const T* __restrict__ gk, T* __restrict__ dq,
                                long long dq_stride, T* __restrict__ dk, long long dk_stride, float* __restrict__ part) {
    constexpr int V = Piece<T>::V, P2 = V / 2, U = 1;
    extern __shared__ float2 table[];
    __shared__ pair sums[kThreads / 32][2][P2][32];              // warp, piece, pair, thread of a row
    enter_dependent();
    const int tid = threadIdx.x, j = tid & (gr.TP - 1), slot = tid / gr.TP;
    const int tok = slot & (gr.TB - 1), h0 = slot / gr.TB, hs = kThreads / gr.TP / gr.TB;
    const bool keys = blockIdx.y != 0;
    const int H = keys ? a.Hk : a.Hq;
    const T *x = static_cast<const T*>(keys ? a.k : a.q), *g = keys ? gk : gq;
    T* dx = keys ? dk : dq;
    const long long stride = keys ? a.k_stride : a.q_stride, dx_stride = keys ? dk_stride : dq_stride;
    Place<T, PAIRS> at;
    at.set(j, gr.T, a.n);
    pair wa[P2], wb[P2], sa[P2], sb[P2];
    weights<P2>(keys ? a.wk : a.wq, at.va, at.vb, at.in, wa, wb);
    const float per_d = 1.f / (float)a.d;
#pragma unroll
    for (int e = 0; e < P2; ++e) sa[e] = sb[e] = 0;
    for (int blk = blockIdx.x; blk < gr.blocks; blk += gridDim.x) {
        const int m0 = blk * gr.TB, m = m0 + tok;
        const bool live = at.in && m < a.B * a.L;
        const int b = m / a.L, t = m - b * a.L;
        const T *row = x + m * stride, *from = g + ((size_t)b * H * a.L + t) * a.d;
        uint4 ux[U][2], ug[U][2];
        auto fetch = [&](int hb) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = hb + u * hs + h0;
                ux[u][0] = ux[u][1] = ug[u][0] = ug[u][1] = make_uint4(0, 0, 0, 0);
                if (live && h < H) {
                    const uint4 *px = reinterpret_cast<const uint4*>(row + (size_t)h * a.d),
                                *pg = reinterpret_cast<const uint4*>(from + (size_t)h * a.L * a.d);
                    ux[u][0] = __ldcs(px + at.va);
                    ux[u][1] = __ldcs(px + at.vb);
                    ug[u][0] = __ldcs(pg + at.va);
                    ug[u][1] = __ldcs(pg + at.vb);
                }
            }
        };
        fetch(0);
        if (a.n) {
            __syncthreads();
            fill_angles<T>(a, gr, m0, table);
            __syncthreads();
        }
        at.angles(table + tok * a.n);
        for (int hb = 0; hb < H; hb += U * hs) {
            pair xa[U][P2], xb[U][P2], ea[U][P2], eb[U][P2];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                Piece<T>::unpack(ux[u][0], xa[u]);
                Piece<T>::unpack(ux[u][1], xb[u]);
                Piece<T>::unpack(ug[u][0], ea[u]);
                Piece<T>::unpack(ug[u][1], eb[u]);
            }
            if (hb + U * hs < H) fetch(hb + U * hs);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = hb + u * hs + h0;
                pair na[P2], nb[P2];
                at.template turn<true>(ea[u], eb[u]);
#pragma unroll
                for (int e = 0; e < P2; ++e) {
                    na[e] = mul2(ea[u][e], wa[e]);
                    nb[e] = mul2(eb[u][e], wb[e]);
                }
                float ss = dot<P2>(xa[u], xb[u], xa[u], xb[u]), sd = dot<P2>(na, nb, xa[u], xb[u]);
                for (int d = gr.TP / 2; d > 0; d /= 2) {
                    ss += __shfl_xor_sync(0xffffffffu, ss, d);
                    sd += __shfl_xor_sync(0xffffffffu, sd, d);
                }
                if (!live || h >= H) continue;
                const float inv = rsqrtf(fmaf(ss, per_d, a.eps));
                const pair i2 = both(inv), c = both(-inv * inv * sd * per_d);
#pragma unroll
                for (int e = 0; e < P2; ++e) {
                    sa[e] = fma2(mul2(ea[u][e], i2), xa[u][e], sa[e]);
                    sb[e] = fma2(mul2(eb[u][e], i2), xb[u][e], sb[e]);
                    na[e] = mul2(i2, fma2(xa[u][e], c, na[e]));
                    nb[e] = mul2(i2, fma2(xb[u][e], c, nb[e]));
                }
                uint4* dst = reinterpret_cast<uint4*>(dx + m * dx_stride + (size_t)h * a.d);
                __stcs(dst + at.va, Piece<T>::pack(na));
                __stcs(dst + at.vb, Piece<T>::pack(nb));
            }
        }
    }
    if (!part) return;
    // over the rows of the warp, then over the warps: always in the same order
    const int lane = tid & 31;
#pragma unroll
    for (int i = 0; i < 2 * P2; ++i) {
        pair v = i < P2 ? sa[i] : sb[i - P2];
        for (int d = 16; d >= gr.TP; d /= 2) v = add2(v, __shfl_xor_sync(0xffffffffu, v, d));
        if (lane < gr.TP) (&sums[tid / 32][0][0][0])[i * 32 + lane] = v;
    }
    __syncthreads();
    for (int i = tid; i < 2 * P2 * gr.T; i += kThreads) {
        const int col = i % gr.T, e = i / gr.T;                  // e: (piece, pair)
        pair v = (&sums[0][0][0][0])[e * 32 + col];
#pragma unroll
        for (int w = 1; w < kThreads / 32; ++w) v = add2(v, (&sums[w][0][0][0])[e * 32 + col]);
        Place<T, PAIRS> pl;
        pl.set(col, gr.T, a.n);
        const float2 f = split(v);
        float* to = part + ((size_t)blockIdx.x * 2 + keys) * a.d + (e / P2 ? pl.vb : pl.va) * V + 2 * (e % P2);
        to[0] = f.x;
        to[1] = f.y;
    }
}

namespace {
Grid grid_for(int B, int L, int d, int n, based_dtype io) {
    Grid g;
    g.T = d / (io == BASED_F32 ? 8 : 16);
    g.TP = 1;
    while (g.TP < g.T) g.TP *= 2;
    g.NP = 1;
    while (g.NP < n) g.NP *= 2;
    const int rows = B * L;
    // up to 32 tokens per block, so that a head's rows are written in runs; fewer where there would not be two blocks of the
    // queries' and two of the keys' per SM (with twice that, the fp32 case above takes 10.4 us)
    g.TB = 32;
    while (g.TB > kThreads / g.TP) g.TB /= 2;
    while (g.TB > 1 && rows < (long long)g.TB * 2 * kSMs) g.TB /= 2;
    g.blocks = (int)(((long long)rows + g.TB - 1) / g.TB);
    return g;
}
// blocks along the tokens backward: as many as are resident at once, of the queries and of the keys
int backward_blocks(const Grid& g) { return g.blocks < 2 * kSMs ? g.blocks : 2 * kSMs; }

template <typename F> cudaError_t with_kinds(based_dtype io, int pairs, F f) {
    using Yes = std::true_type;
    using No = std::false_type;
    if (io == BASED_F32) return pairs ? f(0.f, Yes{}) : f(0.f, No{});
    return pairs ? f(__nv_bfloat16{}, Yes{}) : f(__nv_bfloat16{}, No{});
}
}  // namespace

size_t norm_rotate_backward_bytes(int B, int L, int d, based_dtype io) {
    return (size_t)backward_blocks(grid_for(B, L, d, 0, io)) * 2 * d * sizeof(float);
}

based_status launch_norm_rotate(const NormRotate& a, void* out_q, void* out_k, based_dtype io, cudaStream_t stream) {
    const Grid g = grid_for(a.B, a.L, a.d, a.n, io);
    const cudaError_t e = with_kinds(io, a.pairs, [&](auto zero, auto pairs) {
        using T = decltype(zero);
        return launch_ex(norm_rotate_kernel<T, decltype(pairs)::value>, dim3(g.blocks, 2), dim3(kThreads),
                         (size_t)g.TB * a.n * sizeof(float2), 1, true, stream, a, g, static_cast<T*>(out_q), static_cast<T*>(out_k));
    });
    note_launch();
    const based_status st = check_launch("norm_rotate_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}

based_status launch_norm_rotate_backward(const NormRotate& a, const void* gq, const void* gk, void* dq, long long dq_stride, void* dk,
                                         long long dk_stride, float* dwq, float* dwk, float* part, based_dtype io, cudaStream_t stream) {
    const Grid g = grid_for(a.B, a.L, a.d, a.n, io);
    const int blocks = backward_blocks(g);
    const cudaError_t e = with_kinds(io, a.pairs, [&](auto zero, auto pairs) {
        using T = decltype(zero);
        return launch_ex(norm_rotate_backward_kernel<T, decltype(pairs)::value>, dim3(blocks, 2), dim3(kThreads),
                         (size_t)g.TB * a.n * sizeof(float2), 1, true, stream, a, g, static_cast<const T*>(gq), static_cast<const T*>(gk),
                         static_cast<T*>(dq), dq_stride, static_cast<T*>(dk), dk_stride, dwq ? part : static_cast<float*>(nullptr));
    });
    note_launch();
    const based_status st = check_launch("norm_rotate_backward_kernel");
    if (e != cudaSuccess || st != BASED_OK) return st != BASED_OK ? st : BASED_ERR_CUDA;
    if (!dwq) return BASED_OK;
    return launch_column_sums(part, blocks, 2 * a.d, dwq, a.d, dwk, stream);
}

}  // namespace based
