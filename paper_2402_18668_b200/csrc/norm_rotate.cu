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
// One pass over rows of 32 to 512 bytes: bound by HBM bandwidth.  A row is shared by d / (2 V) threads, each with two 16-byte
// pieces (V values) that hold both elements of its pairs, so only the row's sums cross threads.  A CTA takes a few
// consecutive tokens and all their heads: a warp reads pieces of rows that lie a token stride apart and writes rows that lie
// side by side, and the angles of the tokens, the same for all heads, are taken once, into shared memory.  An angle is a
// product in fp64, reduced to a part of a turn there (a far position's angle in fp32 would be off by position x 6e-8), and only
// that part is rounded to fp32 for the sine and cosine.
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
    long long blocks;              // blocks of tokens
};

// The angles of TB tokens from m0 on: cos and sin [TB][n] in shared memory
__device__ __forceinline__ void fill_angles(const NormRotate& a, long long m0, int TB, float2* table) {
    const long long rows = (long long)a.B * a.L;
    for (int i = threadIdx.x; i < TB * a.n; i += kThreads) {
        const int tok = i / a.n, j = i - tok * a.n;
        const long long m = m0 + tok;
        float2 cs = make_float2(1.f, 0.f);
        if (m < rows) {
            const long long b = m / a.L, t = m - b * a.L;
            const long long pos = a.positions ? (a.per_token ? (long long)a.positions[m] : a.positions[b] + t) : a.start + t;
            const double turns = (double)pos * (a.freqs[j] * kTurnsPerRadian);
            float s, c;
            sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
            cs = make_float2(c, s);
        }
        table[i] = cs;
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

// a block: TB tokens and all their heads
template <typename T, bool PAIRS>
__global__ void __launch_bounds__(kThreads) norm_rotate_kernel(const NormRotate a, const Grid gr, T* __restrict__ out_q, T* __restrict__ out_k) {
    constexpr int V = Piece<T>::V, P2 = V / 2, U = 4;
    extern __shared__ float2 table[];
    enter_dependent();
    const int tid = threadIdx.x, j = tid & (gr.TP - 1), slot = tid / gr.TP;
    const int tok = slot & (gr.TB - 1), h0 = slot / gr.TB, hs = kThreads / gr.TP / gr.TB;
    const long long m = (long long)blockIdx.x * gr.TB + tok, rows = (long long)a.B * a.L;
    if (a.n) {
        fill_angles(a, (long long)blockIdx.x * gr.TB, gr.TB, table);
        __syncthreads();
    }
    Place<T, PAIRS> at;
    at.set(j, gr.T, a.n);
    at.angles(table + tok * a.n);
    const bool live = at.in && m < rows;
    const long long b = m / a.L, t = m - b * a.L;
    const float per_d = 1.f / (float)a.d;
    auto heads = [&](const T* x, long long stride, const float* w, T* y, int H) {
        pair wa[P2], wb[P2];
        weights<P2>(w, at.va, at.vb, at.in, wa, wb);
        const T* row = x + m * stride;
        T* to = y + (b * H * a.L + t) * a.d;
        for (int hb = 0; hb < H; hb += U * hs) {                 // (every thread: the sums cross lanes)
            uint4 ua[U], ub[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = hb + u * hs + h0;
                ua[u] = ub[u] = make_uint4(0, 0, 0, 0);
                if (live && h < H) {
                    ua[u] = __ldcs(reinterpret_cast<const uint4*>(row + (size_t)h * a.d) + at.va);
                    ub[u] = __ldcs(reinterpret_cast<const uint4*>(row + (size_t)h * a.d) + at.vb);
                }
            }
            float ss[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                pair xa[P2], xb[P2];
                Piece<T>::unpack(ua[u], xa);
                Piece<T>::unpack(ub[u], xb);
                ss[u] = dot<P2>(xa, xb, xa, xb);
            }
            for (int d = gr.TP / 2; d > 0; d /= 2)
#pragma unroll
                for (int u = 0; u < U; ++u) ss[u] += __shfl_xor_sync(0xffffffffu, ss[u], d);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = hb + u * hs + h0;
                if (!live || h >= H) continue;
                const pair inv = both(rsqrtf(fmaf(ss[u], per_d, a.eps)));
                pair xa[P2], xb[P2];
                Piece<T>::unpack(ua[u], xa);
                Piece<T>::unpack(ub[u], xb);
#pragma unroll
                for (int e = 0; e < P2; ++e) {
                    xa[e] = mul2(mul2(xa[e], inv), wa[e]);
                    xb[e] = mul2(mul2(xb[e], inv), wb[e]);
                }
                at.template turn<false>(xa, xb);
                uint4* dst = reinterpret_cast<uint4*>(to + (size_t)h * a.L * a.d);
                __stcs(dst + at.va, Piece<T>::pack(xa));
                __stcs(dst + at.vb, Piece<T>::pack(xb));
            }
        }
    };
    heads(static_cast<const T*>(a.q), a.q_stride, a.wq, out_q, a.Hq);
    heads(static_cast<const T*>(a.k), a.k_stride, a.wk, out_k, a.Hk);
}

// the same rows backward; part: a row of 2 d sums per CTA (null: the weights' gradients are not wanted)
template <typename T, bool PAIRS>
__global__ void __launch_bounds__(kThreads)
    norm_rotate_backward_kernel(const NormRotate a, const Grid gr, const T* __restrict__ gq, const T* __restrict__ gk, T* __restrict__ dq,
                                long long dq_stride, T* __restrict__ dk, long long dk_stride, float* __restrict__ part) {
    constexpr int V = Piece<T>::V, P2 = V / 2, U = 2;
    extern __shared__ float2 table[];
    __shared__ pair sums[kThreads / 32][2][2][P2][32];           // warp, query or key, piece, pair, thread of a row
    enter_dependent();
    const int tid = threadIdx.x, j = tid & (gr.TP - 1), slot = tid / gr.TP;
    const int tok = slot & (gr.TB - 1), h0 = slot / gr.TB, hs = kThreads / gr.TP / gr.TB;
    const long long rows = (long long)a.B * a.L;
    Place<T, PAIRS> at;
    at.set(j, gr.T, a.n);
    const float per_d = 1.f / (float)a.d;
    pair acc[2][2][P2];
#pragma unroll
    for (int i = 0; i < 4 * P2; ++i) (&acc[0][0][0])[i] = 0;
    for (long long blk = blockIdx.x; blk < gr.blocks; blk += gridDim.x) {
        const long long m = blk * gr.TB + tok;
        if (a.n) {
            __syncthreads();
            fill_angles(a, blk * gr.TB, gr.TB, table);
            __syncthreads();
        }
        at.angles(table + tok * a.n);
        const bool live = at.in && m < rows;
        const long long b = m / a.L, t = m - b * a.L;
        auto heads = [&](const T* x, long long stride, const float* w, const T* g, T* dx, long long dx_stride, int H, pair (&sa)[P2],
                         pair (&sb)[P2]) {
            pair wa[P2], wb[P2];
            weights<P2>(w, at.va, at.vb, at.in, wa, wb);
            const T* row = x + m * stride;
            const T* from = g + (b * H * a.L + t) * a.d;
            for (int hb = 0; hb < H; hb += U * hs) {
                uint4 ux[U][2], ug[U][2];
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
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int h = hb + u * hs + h0;
                    pair xa[P2], xb[P2], ea[P2], eb[P2], na[P2], nb[P2];
                    Piece<T>::unpack(ux[u][0], xa);
                    Piece<T>::unpack(ux[u][1], xb);
                    Piece<T>::unpack(ug[u][0], ea);
                    Piece<T>::unpack(ug[u][1], eb);
                    at.template turn<true>(ea, eb);
#pragma unroll
                    for (int e = 0; e < P2; ++e) {
                        na[e] = mul2(ea[e], wa[e]);
                        nb[e] = mul2(eb[e], wb[e]);
                    }
                    float ss = dot<P2>(xa, xb, xa, xb), sd = dot<P2>(na, nb, xa, xb);
                    for (int d = gr.TP / 2; d > 0; d /= 2) {
                        ss += __shfl_xor_sync(0xffffffffu, ss, d);
                        sd += __shfl_xor_sync(0xffffffffu, sd, d);
                    }
                    if (!live || h >= H) continue;
                    const float inv = rsqrtf(fmaf(ss, per_d, a.eps));
                    const pair i2 = both(inv), c = both(-inv * inv * sd * per_d);
#pragma unroll
                    for (int e = 0; e < P2; ++e) {
                        sa[e] = fma2(mul2(ea[e], i2), xa[e], sa[e]);
                        sb[e] = fma2(mul2(eb[e], i2), xb[e], sb[e]);
                        na[e] = mul2(i2, fma2(xa[e], c, na[e]));
                        nb[e] = mul2(i2, fma2(xb[e], c, nb[e]));
                    }
                    uint4* dst = reinterpret_cast<uint4*>(dx + m * dx_stride + (size_t)h * a.d);
                    __stcs(dst + at.va, Piece<T>::pack(na));
                    __stcs(dst + at.vb, Piece<T>::pack(nb));
                }
            }
        };
        heads(static_cast<const T*>(a.q), a.q_stride, a.wq, gq, dq, dq_stride, a.Hq, acc[0][0], acc[0][1]);
        heads(static_cast<const T*>(a.k), a.k_stride, a.wk, gk, dk, dk_stride, a.Hk, acc[1][0], acc[1][1]);
    }
    if (!part) return;
    // over the rows of the warp, then over the warps: always in the same order
    const int lane = tid & 31;
#pragma unroll
    for (int i = 0; i < 4 * P2; ++i) {
        pair v = (&acc[0][0][0])[i];
        for (int d = 16; d >= gr.TP; d /= 2) v = add2(v, __shfl_xor_sync(0xffffffffu, v, d));
        if (lane < gr.TP) (&sums[tid / 32][0][0][0][0])[i * 32 + lane] = v;
    }
    __syncthreads();
    for (int i = tid; i < 4 * P2 * gr.T; i += kThreads) {
        const int x = i % gr.T, e = i / gr.T;                    // e: (query or key, piece, pair)
        pair v = (&sums[0][0][0][0][0])[e * 32 + x];
#pragma unroll
        for (int w = 1; w < kThreads / 32; ++w) v = add2(v, (&sums[w][0][0][0][0])[e * 32 + x]);
        Place<T, PAIRS> pl;
        pl.set(x, gr.T, a.n);
        const int piece = (e / P2) & 1 ? pl.vb : pl.va;
        const float2 f = split(v);
        float* to = part + (size_t)blockIdx.x * 2 * a.d + (e / (2 * P2)) * a.d + piece * V + 2 * (e % P2);
        to[0] = f.x;
        to[1] = f.y;
    }
}

namespace {
Grid grid_for(int B, int L, int d, based_dtype io) {
    Grid g;
    g.T = d / (io == BASED_F32 ? 8 : 16);
    g.TP = 1;
    while (g.TP < g.T) g.TP *= 2;
    const long long rows = (long long)B * L;
    // up to 8 tokens per block, so that a head's rows are written in runs; fewer where the chip would not be filled
    g.TB = 8;
    while (g.TB > kThreads / g.TP) g.TB /= 2;
    while (g.TB > 1 && rows < (long long)g.TB * 4 * kSMs) g.TB /= 2;
    g.blocks = (rows + g.TB - 1) / g.TB;
    return g;
}
unsigned backward_blocks(const Grid& g) { return (unsigned)(g.blocks < 4 * kSMs ? g.blocks : 4 * kSMs); }

template <typename F> cudaError_t with_kinds(based_dtype io, int pairs, F f) {
    using Yes = std::true_type;
    using No = std::false_type;
    if (io == BASED_F32) return pairs ? f(0.f, Yes{}) : f(0.f, No{});
    return pairs ? f(__nv_bfloat16{}, Yes{}) : f(__nv_bfloat16{}, No{});
}
}  // namespace

size_t norm_rotate_backward_bytes(int B, int L, int d, based_dtype io) {
    return (size_t)backward_blocks(grid_for(B, L, d, io)) * 2 * d * sizeof(float);
}

based_status launch_norm_rotate(const NormRotate& a, void* out_q, void* out_k, based_dtype io, cudaStream_t stream) {
    const Grid g = grid_for(a.B, a.L, a.d, io);
    if (g.blocks > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    const cudaError_t e = with_kinds(io, a.pairs, [&](auto zero, auto pairs) {
        using T = decltype(zero);
        return launch_ex(norm_rotate_kernel<T, decltype(pairs)::value>, dim3((unsigned)g.blocks), dim3(kThreads),
                         (size_t)g.TB * a.n * sizeof(float2), 1, true, stream, a, g, static_cast<T*>(out_q), static_cast<T*>(out_k));
    });
    note_launch();
    const based_status st = check_launch("norm_rotate_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}

based_status launch_norm_rotate_backward(const NormRotate& a, const void* gq, const void* gk, void* dq, long long dq_stride, void* dk,
                                         long long dk_stride, float* dwq, float* dwk, float* part, based_dtype io, cudaStream_t stream) {
    const Grid g = grid_for(a.B, a.L, a.d, io);
    const unsigned blocks = backward_blocks(g);
    const cudaError_t e = with_kinds(io, a.pairs, [&](auto zero, auto pairs) {
        using T = decltype(zero);
        return launch_ex(norm_rotate_backward_kernel<T, decltype(pairs)::value>, dim3(blocks), dim3(kThreads),
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
