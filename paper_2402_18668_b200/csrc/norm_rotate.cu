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
// that part is rounded to fp32 for the sine and cosine.  Rows are asked for two steps ahead, the first ones before the angles, by
// asynchronous copies into places that each thread has to itself, which costs neither registers nor barriers.  Backward the tokens
// are shared out evenly among the CTAs that are resident at once, and a CTA's (head, token) rows go round its threads without gaps.
//
// Measured: bf16, 2 x 32768 tokens, 16 + 16 heads of 64, rotating: 94 us (87 % of the copy rate; 106 with the next step's rows in
// registers); fp32, 3 x 777 tokens, 16 + 4 heads of 128, 64 elements of them rotating: 8.4 us (87 %); backward, bf16, 4 x 2048 tokens of
// 16 + 16 heads of 64: 26 us (58 %; 3.6 of them the second launch, which joins the weights' gradients), 4 x 8192: 85 us (72 %);
// in fp32 45 us (68 %) and 165 (75 %).
#include <type_traits>

#include "common.cuh"
#include "pairs.cuh"

namespace based {
using namespace pairs;

namespace {
constexpr int kThreads = 128, kBlocks = 4;       // (blocks per SM)
constexpr int kHeads = 2, kAhead = 3, kAheadBack = 3;    // heads per step forward; steps that have a place in shared memory
constexpr double kTurnsPerRadian = 0.15915494309189533577;

__device__ __forceinline__ pair swap2(pair a) { return (a >> 32) | (a << 32); }

struct Grid {
    int T, TP;                     // threads that share a row, and the power of two they are spaced by
    int NP;                        // the angles of a token are spaced by that many threads, a power of two
    int AS;                        // a token's angles in shared memory, n cosines and n sines: floats from one to the next (4 more: other banks)
    int TB;                        // tokens per block, a power of two.  Backward: whose angles are there at once
    int blocks;                    // blocks of tokens.  Backward: even shares of them
};
// Sine and cosine of x half turns, |x| <= 1.  For bf16 io the fast ones (off by 2^-20.5, where the result is rounded by up to 2^-8 of it)
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
// The angles of tokens m0 .. m0 + count - 1 of the batch (those there are)
template <typename T> __device__ __forceinline__ void fill_angles(const NormRotate& a, const Grid& gr, int m0, int count, float* table) {
    const int j = threadIdx.x & (gr.NP - 1), step = kThreads / gr.NP;
    if (j >= a.n) return;
    const double freq = a.freqs[j] * kTurnsPerRadian;
    for (int tok = threadIdx.x / gr.NP; tok < count; tok += step) {
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
        const float2 f = cos_sin<T>((float)(2.0 * (turns - rint(turns))));
        table[tok * gr.AS + j] = f.x;
        table[tok * gr.AS + a.n + j] = f.y;
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
        va = turns ? j : half + j;                               // (neighbours side by side: behind the turning pieces too)
        vb = turns ? half + j : T_ + j;
    }
    __device__ __forceinline__ void angles(const float* row, int n) {
        if (!in || !turns) return;
        if constexpr (PAIRS) {
#pragma unroll
            for (int e = 0; e < P2; ++e) {
                const float sa = row[n + va * P2 + e], sb = row[n + vb * P2 + e];
                c[e] = both(row[va * P2 + e]);
                s[e] = make(-sa, sa);
                c[P2 + e] = both(row[vb * P2 + e]);
                s[P2 + e] = make(-sb, sb);
            }
        } else {
            load_f32<P2>(row + va * V, c);
            load_f32<P2>(row + n + va * V, s);
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
__global__ void __launch_bounds__(kThreads, kBlocks) norm_rotate_kernel(const NormRotate a, const Grid gr, T* __restrict__ out_q, T* __restrict__ out_k) {
    constexpr int V = Piece<T>::V, P2 = V / 2, U = kHeads, NS = kAhead;
    extern __shared__ __align__(16) float table[];
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
    // rows of U heads at a time, NS - 1 such steps ahead through places in shared memory that each thread has to itself; the first ones
    // before the angles
    uint4* ring = reinterpret_cast<uint4*>(table + gr.TB * gr.AS) + tid;
    const int its = (H + U * hs - 1) / (U * hs);
    int fetched = 0, place = 0;
    auto fetch = [&] {
        if (fetched < its) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = (fetched * U + u) * hs + h0;
                const bool in = live && h < H;
                const T* src = row + (in ? (size_t)h * a.d : 0);
                copy_async16(ring + (place + 2 * u) * kThreads, src + (in ? at.va * V : 0), in);
                copy_async16(ring + (place + 2 * u + 1) * kThreads, src + (in ? at.vb * V : 0), in);
            }
            ++fetched;
        }
        place = place == (NS - 1) * 2 * U ? 0 : place + 2 * U;
        copy_async_commit();
    };
#pragma unroll
    for (int i = 0; i < NS - 1; ++i) fetch();
    pair wa[P2], wb[P2];
    weights<P2>(keys ? a.wk : a.wq, at.va, at.vb, at.in, wa, wb);
    if (a.n) {
        fill_angles<T>(a, gr, m0, gr.TB, table);
        __syncthreads();
    }
    at.angles(table + tok * gr.AS, a.n);
    int from = 0;
    for (int hb = 0; hb < H; hb += U * hs) {                     // (every thread: the sums cross lanes)
        pair xa[U][P2], xb[U][P2];
        float ss[U];
        copy_async_wait<NS - 2>();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Piece<T>::unpack(ring[(from + 2 * u) * kThreads], xa[u]);
            Piece<T>::unpack(ring[(from + 2 * u + 1) * kThreads], xb[u]);
        }
        from = from == (NS - 1) * 2 * U ? 0 : from + 2 * U;
        fetch();                                                 // (into the place that the step before this one read)
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
__global__ void __launch_bounds__(kThreads, kBlocks)
    norm_rotate_backward_kernel(const NormRotate a, const Grid gr, const T* __restrict__ gq, const T* __restrict__ gk, T* __restrict__ dq,
                                long long dq_stride, T* __restrict__ dk, long long dk_stride, float* __restrict__ part) {
    constexpr int V = Piece<T>::V, P2 = V / 2, NS = kAheadBack;
    extern __shared__ __align__(16) float table[];
    __shared__ pair sums[kThreads / 32][2][P2][32];              // warp, piece, pair, thread of a row
    enter_dependent();
    const int tid = threadIdx.x, j = tid & (gr.TP - 1), slot = tid / gr.TP;
    const int groups = kThreads / gr.TP, rows = a.B * a.L;
    const int m_begin = (int)((long long)rows * blockIdx.x / gridDim.x), m_end = (int)((long long)rows * (blockIdx.x + 1) / gridDim.x);
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
    // A CTA's share of the tokens in pieces of up to TB, a piece's rows one per group and step, its tokens in a row for one head after
    // the other.  The rows come NS - 1 steps ahead through places in shared memory that each thread has to itself
    struct Cursor {
        int m0, count, left, tok, h, dt, dh;
    };
    auto start = [&](Cursor& c) {
        c.count = min(gr.TB, m_end - c.m0);
        c.left = (int)(((long long)c.count * H + groups - 1) / groups);       // (H up to 2^27)
        c.h = slot / c.count;
        c.tok = slot - c.h * c.count;
        c.dh = groups / c.count;
        c.dt = groups - c.dh * c.count;
    };
    auto step = [](Cursor& c) {
        --c.left;
        c.tok += c.dt;
        c.h += c.dh;
        if (c.tok >= c.count) {
            c.tok -= c.count;
            ++c.h;
        }
    };
    uint4* ring = reinterpret_cast<uint4*>(table + gr.TB * gr.AS) + tid;
    int place = 0, from = 0;
    Cursor ahead;
    ahead.m0 = m_begin;
    start(ahead);
    auto fetch = [&] {
        if (ahead.left) {
            const int m = ahead.m0 + ahead.tok, b = m / a.L, t = m - b * a.L;
            const bool in = at.in && ahead.h < H;
            const T *px = in ? x + m * stride + (size_t)ahead.h * a.d : x, *pg = in ? g + (((size_t)b * H + ahead.h) * a.L + t) * a.d : g;
            const int va = in ? at.va * V : 0, vb = in ? at.vb * V : 0;
            uint4* to = ring + place * kThreads;
            copy_async16(to, px + va, in);
            copy_async16(to + kThreads, px + vb, in);
            copy_async16(to + 2 * kThreads, pg + va, in);
            copy_async16(to + 3 * kThreads, pg + vb, in);
            step(ahead);
            if (!ahead.left && ahead.m0 + ahead.count < m_end) {
                ahead.m0 += ahead.count;
                start(ahead);
            }
        }
        place = place == (NS - 1) * 4 ? 0 : place + 4;
        copy_async_commit();
    };
#pragma unroll
    for (int i = 0; i < NS - 1; ++i) fetch();
    Cursor c;
    for (c.m0 = m_begin; c.m0 < m_end; c.m0 += gr.TB) {
        if (a.n) {
            __syncthreads();
            fill_angles<T>(a, gr, c.m0, min(gr.TB, m_end - c.m0), table);
            __syncthreads();
        }
        for (start(c); c.left; step(c)) {
            pair xa[P2], xb[P2], ea[P2], eb[P2], na[P2], nb[P2];
            copy_async_wait<NS - 2>();
            const uint4* own = ring + from * kThreads;
            Piece<T>::unpack(own[0], xa);
            Piece<T>::unpack(own[kThreads], xb);
            Piece<T>::unpack(own[2 * kThreads], ea);
            Piece<T>::unpack(own[3 * kThreads], eb);
            from = from == (NS - 1) * 4 ? 0 : from + 4;
            fetch();                                             // (into the place that the step before this one read)
            at.angles(table + c.tok * gr.AS, a.n);
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
            if (!at.in || c.h >= H) continue;
            const float inv = rsqrtf(fmaf(ss, per_d, a.eps));
            const pair i2 = both(inv), f = both(-inv * inv * sd * per_d);
#pragma unroll
            for (int e = 0; e < P2; ++e) {
                sa[e] = fma2(mul2(ea[e], i2), xa[e], sa[e]);
                sb[e] = fma2(mul2(eb[e], i2), xb[e], sb[e]);
                na[e] = mul2(i2, fma2(xa[e], f, na[e]));
                nb[e] = mul2(i2, fma2(xb[e], f, nb[e]));
            }
            uint4* dst = reinterpret_cast<uint4*>(dx + (c.m0 + c.tok) * dx_stride + (size_t)c.h * a.d);
            __stcs(dst + at.va, Piece<T>::pack(na));
            __stcs(dst + at.vb, Piece<T>::pack(nb));
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
Grid grid_for(int B, int L, int d, int n, based_dtype io, bool back) {
    Grid g;
    g.T = d / (io == BASED_F32 ? 8 : 16);
    g.TP = 1;
    while (g.TP < g.T) g.TP *= 2;
    g.NP = 1;
    while (g.NP < n) g.NP *= 2;
    g.AS = n ? 2 * n + 4 : 0;
    const int rows = B * L;
    g.TB = 32;
    if (back) {
        while (g.TB > 1 && g.TB * n > 1024) g.TB /= 2;           // (8 KB of angles)
        // as many as are resident at once, of the queries and of the keys (twice as many, of half the tokens: 33 us for the case's 26)
        g.blocks = rows < kBlocks * kSMs / 2 ? rows : kBlocks * kSMs / 2;
        return g;
    }
    // up to 32 tokens per block, so that a head's rows are written in runs; fewer where there would not be two blocks of the
    // queries' and two of the keys' per SM (with twice that, the fp32 case above takes 10.4 us)
    while (g.TB > kThreads / g.TP) g.TB /= 2;
    while (g.TB > 1 && rows < (long long)g.TB * kBlocks / 2 * kSMs) g.TB /= 2;
    g.blocks = (int)(((long long)rows + g.TB - 1) / g.TB);
    return g;
}

template <typename F> cudaError_t with_kinds(based_dtype io, int pairs, F f) {
    using Yes = std::true_type;
    using No = std::false_type;
    if (io == BASED_F32) return pairs ? f(0.f, Yes{}) : f(0.f, No{});
    return pairs ? f(__nv_bfloat16{}, Yes{}) : f(__nv_bfloat16{}, No{});
}
}  // namespace

size_t norm_rotate_backward_bytes(int B, int L, int d, based_dtype io) {
    return (size_t)grid_for(B, L, d, 0, io, true).blocks * 2 * d * sizeof(float);
}

based_status launch_norm_rotate(const NormRotate& a, void* out_q, void* out_k, based_dtype io, cudaStream_t stream) {
    const Grid g = grid_for(a.B, a.L, a.d, a.n, io, false);
    const cudaError_t e = with_kinds(io, a.pairs, [&](auto zero, auto pairs) {
        using T = decltype(zero);
        return launch_ex(norm_rotate_kernel<T, decltype(pairs)::value>, dim3(g.blocks, 2), dim3(kThreads),
                         (size_t)g.TB * g.AS * sizeof(float) + kAhead * 2 * kHeads * kThreads * 16, 1, true, stream, a, g, static_cast<T*>(out_q), static_cast<T*>(out_k));
    });
    note_launch();
    const based_status st = check_launch("norm_rotate_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}

based_status launch_norm_rotate_backward(const NormRotate& a, const void* gq, const void* gk, void* dq, long long dq_stride, void* dk,
                                         long long dk_stride, float* dwq, float* dwk, float* part, based_dtype io, cudaStream_t stream) {
    const Grid g = grid_for(a.B, a.L, a.d, a.n, io, true);
    const cudaError_t e = with_kinds(io, a.pairs, [&](auto zero, auto pairs) {
        using T = decltype(zero);
        return launch_ex(norm_rotate_backward_kernel<T, decltype(pairs)::value>, dim3(g.blocks, 2), dim3(kThreads),
                         (size_t)g.TB * g.AS * sizeof(float) + kAheadBack * 4 * kThreads * 16, 1, true, stream, a, g, static_cast<const T*>(gq), static_cast<const T*>(gk),
                         static_cast<T*>(dq), dq_stride, static_cast<T*>(dk), dk_stride, dwq ? part : static_cast<float*>(nullptr));
    });
    note_launch();
    const based_status st = check_launch("norm_rotate_backward_kernel");
    if (e != cudaSuccess || st != BASED_OK) return st != BASED_OK ? st : BASED_ERR_CUDA;
    if (!dwq) return BASED_OK;
    return launch_column_sums(part, g.blocks, 2 * a.d, dwq, a.d, dwk, stream);
}

}  // namespace based
