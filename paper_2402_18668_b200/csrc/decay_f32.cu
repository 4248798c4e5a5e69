// Decay attention, fp32 io, on multiply-adds: the passes of decay.cuh in blocks of 64 tokens.
//
// One CTA per pass, head, tile of 64 output columns and segment; three groups of 128 threads work on a block side by side:
//   pairs  P = x y^T, faded and masked (only columns that some row of 8 sees)
//   past   take (x S), left where x was
//   state  (give y)^T z; S <- f S + that, S in shared memory throughout
// and, once all are done, out = past + P z, a third of the rows each,
// while the next block's x, y, z come in by asynchronous copies (zeros where a token is padding).  A thread's tile is 8 x 4, lane bit 0 on its
// rows and the others on its columns: 12 loads of 16 bytes, two passes each, for 128 multiply-adds.  Where both operands lie along the
// sum's index (x y^T; x S, with S kept turned) two of its terms share an instruction; else two columns or rows do.
// Rows lie in shared memory in the order in which the pass goes through them, so that back passes are the same from there on.
// What bounds it: multiply-adds, 3.25 (wide heads 5.9) times 64^3 of them a block, at 4 cycles a pair where registers and shared memory are
// read for them too (2.5 without): a block takes 8 us.  256 threads that did all of it one after another on 4 x 4 tiles, two CTAs
// on an SM and the loads in between, took 1007 us for B8 H16 L4096 64/64 where this takes 501.
#include "decay.cuh"
#include "f32_tiles.cuh"
#include "pairs.cuh"

namespace based {

namespace {

using pairs::pair;
constexpr int kT = kDecayBlockF32, kTile = 64, kGroup = 128;
template <int DC, bool STATES> struct Cfg {
    static constexpr int kThreads = STATES ? 2 * kGroup : 3 * kGroup;
    static constexpr int kX = DC + 4, kZ = kTile + 4;          // floats per row
    static constexpr int offY = STATES ? 0 : kT * kX, offZ = offY + kT * kX, kStage = offZ + kT * kZ;
    static constexpr int offS = 2 * kStage, offP = offS + kTile * kX, offW = offP + (STATES ? 0 : kT * kZ);
    static constexpr size_t bytes = sizeof(float) * (offW + 4 * kT);
    static_assert(bytes <= 232448, "shared memory budget");
};

struct Args {
    DecayCall c;
    const uint32_t* places;
    float *states, *factors;
    int blocks, segments, tiles;
};

// the state in shared memory: a row per column of z, so that neighbouring threads, 4 columns each, read neighbouring rows
__device__ __forceinline__ int state_row(int e) { return (e & 3) * 16 + (e >> 2); }
// rows of a block of a [B,H,L,width] view into shared memory, `base` at its first token and column; zeros past the `width` columns and where
// a token is padding.  A thread stays with its column
template <int COLS, int THREADS>
__device__ __forceinline__ void load_rows(const float* base, long long stride, bool back, int width, const uint32_t* pl, float* dst) {
    constexpr int N = COLS / 4, R = THREADS / N;
    const int r0 = threadIdx.x / N, c = threadIdx.x % N * 4;
    const bool in = c < width;
    const float* src = base + (long long)(back ? kT - 1 - r0 : r0) * stride + c;
    const long long step = back ? -R * stride : R * stride;
#pragma unroll
    for (int k = 0; k < (kT + R - 1) / R; ++k, src += step) {
        const int r = r0 + k * R;
        if (kT % R == 0 || r < kT) {
            const bool there = in && !(pl[r] & kPadding);
            pairs::copy_async16(dst + r * (COLS + 4) + c, there ? src : base, there);
        }
    }
}
// acc[i][j] += x[8 i] . y[16 j] over K elements, rows of kX floats apart: sums of even and of odd elements.  HALF: only where 16 j <= 8 i + 7.
// With a state of 64 rows a row of x is read again as soon as its elements are used up (B8 H16 L4096 64/64 528 -> 506 us); with 128 there
// are no registers for it (B2 H16 L4096 128/128 574 -> 624).
template <int K, int kX, bool HALF>
__device__ __forceinline__ void dots(const float* x, const float* y, pair (&acc)[8][4]) {
    constexpr bool kAhead = K == 64;
    ulonglong2 a[8], b[4];
    if (kAhead) {
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = *reinterpret_cast<const ulonglong2*>(x + 8 * i * kX);
    }
#pragma unroll 1
    for (int k = 0; k < K; k += 4) {
        const int n = k + 4 < K ? k + 4 : 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = *reinterpret_cast<const ulonglong2*>(y + 16 * j * kX + k);
        if (!kAhead) {
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = *reinterpret_cast<const ulonglong2*>(x + 8 * i * kX + k);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (!HALF || 2 * j <= i) acc[i][j] = pairs::fma2(a[i].x, b[j].x, acc[i][j]);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (!HALF || 2 * j <= i) acc[i][j] = pairs::fma2(a[i].y, b[j].y, acc[i][j]);
            if (kAhead) a[i] = *reinterpret_cast<const ulonglong2*>(x + 8 * i * kX + n);
        }
    }
}
__device__ __forceinline__ float sum_of(pair x) {
    const float2 v = pairs::split(x);
    return v.x + v.y;
}

// Rows rg + 8 m of an output, m = group + 3 i: rows i from FROM on take columns k0 .. k1 of P times z
template <int FROM, int kZ>
__device__ __forceinline__ void rows_of(const float* const (&P)[3], const float* z, int k0, int k1, pair (&o)[3][2]) {
#pragma unroll 1
    for (int k = k0; k < k1; k += 4) {
        float4 x[3];
        ulonglong2 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const ulonglong2*>(z + (k + u) * kZ);
#pragma unroll
        for (int i = FROM; i < 3; ++i) x[i] = lds4(P[i] + k);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = FROM; i < 3; ++i) {
                const pair xs = pairs::both(u == 0 ? x[i].x : u == 1 ? x[i].y : u == 2 ? x[i].z : x[i].w);
                o[i][0] = pairs::fma2(xs, v[u].x, o[i][0]);
                o[i][1] = pairs::fma2(xs, v[u].y, o[i][1]);
            }
    }
}

template <int DC, bool STATES>
__global__ void __launch_bounds__(Cfg<DC, STATES>::kThreads, STATES && DC == 64 ? 2 : 1) decay_f32_kernel(const __grid_constant__ Args a) {
    using C = Cfg<DC, STATES>;
    constexpr int kX = C::kX, kZ = C::kZ, NH = DC / 64;
    extern __shared__ __align__(16) float sm[];
    float *sS = sm + C::offS, *sP = sm + C::offP, *give = sm + C::offW;
    uint32_t* ring = reinterpret_cast<uint32_t*>(give + kT);         // the places of three blocks
    const int tid = threadIdx.x, group = tid >> 7, gt = tid & 127, rg = (gt >> 5) * 2 + (gt & 1), cg = (gt & 31) >> 1;
    const DecayItem it(blockIdx.x, a.c.passes, a.tiles, STATES ? a.segments - 1 : a.segments);
    const DecayPass& p = a.c.pass[it.pass];
    const int e0 = it.tile * kTile, L = a.c.L;
    const bool back = p.back;
    enter_dependent();
    if (e0 >= p.de) return;
    const int b = (int)(it.head / a.c.H), h = (int)(it.head % a.c.H);
    const float rate2 = rate_of(a.c.rate[h]);
    const int g = back ? a.segments - 1 - it.segment : it.segment;
    const int first = decay_first(a.blocks, a.segments, g), count = decay_first(a.blocks, a.segments, g + 1) - first;
    auto block_of = [&](int i) { return back ? first + count - 1 - i : first + i; };
    auto word_of = [&](int i) -> uint32_t {                          // of this thread's row, in the pass's order
        const int n = block_of(i), r = back ? kT - 1 - tid : tid;
        return a.places ? a.places[((long long)b * a.blocks + n) * kT + r] : (uint32_t)min(r + 1, L - n * kT) | (r < L - n * kT ? 0u : kPadding);
    };
    auto base_of = [&](const based_heads& v) { return static_cast<const float*>(v.data) + b * v.batch_stride + h * v.head_stride; };
    const float *gx = base_of(p.x), *gy = base_of(p.y), *gz = base_of(p.z) + e0;
    auto load = [&](int i) {
        float* s = sm + (i & 1) * C::kStage;
        const uint32_t* pl = ring + i % 3 * kT;
        const long long t0 = (long long)block_of(i) * kT;
        if (!STATES) load_rows<DC, C::kThreads>(gx + t0 * p.x.token_stride, p.x.token_stride, back, p.dc, pl, s);
        load_rows<DC, C::kThreads>(gy + t0 * p.y.token_stride, p.y.token_stride, back, p.dc, pl, s + C::offY);
        load_rows<kTile, C::kThreads>(gz + t0 * p.z.token_stride, p.z.token_stride, back, p.de - e0, pl, s + C::offZ);
    };
    if (tid < kT) {
        ring[tid] = count > 0 ? word_of(0) : kPadding;
        ring[kT + tid] = count > 1 ? word_of(1) : kPadding;
    }
    __syncthreads();
    if (count > 0) load(0);
    pairs::copy_async_commit();

    // the state that the segment begins with
    if (!STATES) {
        for (int i = tid; i < DC * kTile; i += C::kThreads) {        // (neighbouring threads along the rows in memory, whichever way it lies)
            const int c = p.turned ? i % DC : i / kTile, e = p.turned ? i / DC : i % kTile;
            float s = 0.f;
            if (p.state_in && c < p.dc && e0 + e < p.de)
                s = p.in_factor * p.state_in[it.head * p.dc * p.de + (p.turned ? (long long)(e0 + e) * p.dc + c : (long long)c * p.de + e0 + e)];
            sS[state_row(e) * kX + c] = s;
        }
        if (it.segment > 0) {
            __syncthreads();
            constexpr int N = (DC * kTile / 4 + C::kThreads - 1) / C::kThreads;
            float4 s[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int i = tid + k * C::kThreads;
                s[k] = i < DC * kTile / 4 ? lds4(sS + i / (DC / 4) * kX + i % (DC / 4) * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            const long long slot = decay_slot(it.pass, a.c.passes, it.head, a.tiles, it.tile, a.segments, 0);
#pragma unroll 2
            for (int q = 0; q < it.segment; ++q) {
                const float f = a.factors[slot + q];
                const float4* from = reinterpret_cast<const float4*>(a.states + (slot + q) * kDecayMaxWidth * kTile);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const int i = tid + k * C::kThreads;
                    if (i < DC * kTile / 4) {
                        const float4 x = from[i];                    // (a factor of 0 drops what was before, whatever it holds)
                        s[k] = f == 0.f ? x : make_float4(fmaf(f, s[k].x, x.x), fmaf(f, s[k].y, x.y), fmaf(f, s[k].z, x.z), fmaf(f, s[k].w, x.w));
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int i = tid + k * C::kThreads;
                if (i < DC * kTile / 4) *reinterpret_cast<float4*>(sS + i / (DC / 4) * kX + i % (DC / 4) * 4) = s[k];
            }
        }
    }
    // factors of a row's columns in a block of one document without padding: 8 m + rg - cg steps (below 0: it does not see it)
    float plain_f[8];
#pragma unroll
    for (int m = 0; m < 8; ++m) plain_f[m] = !STATES && group == 0 && 8 * m + rg - cg >= 0 ? faded(rate2, 8 * m + rg - cg) : 0.f;

    float whole = 1.f;
    pair st[NH][4][4] = {};                                          // STATES: this group's share of the state, rows 8 rg + 64 n, columns 4 cg
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
        uint32_t ahead = kPadding;
        if (tid < kT && i + 2 < count) ahead = word_of(i + 2);
        pairs::copy_async_wait<0>();
        __syncthreads();                                             // block i is there, and nobody is at block i - 1 any more
        if (i + 1 < count) load(i + 1);
        pairs::copy_async_commit();
        float* sX = sm + (i & 1) * C::kStage;
        const float *sY = sX + C::offY, *sZ = sX + C::offZ;
        const uint32_t *pl = ring + i % 3 * kT, end = pl[back ? 0 : kT - 1];
        const int c1 = place_count(end), r1 = place_run(end), t0 = block_of(i) * kT;
        const bool empty = c1 == 0, plain = r1 == 0 && c1 == min(kT, L - t0);
        const float f = r1 == 0 ? faded(rate2, c1) : 0.f;
        if (!STATES && group == 0) {
            // ---- pairs
            pair acc[8][4] = {};
            if (!empty) dots<DC, kX, true>(sX + rg * kX, sY + cg * kX, acc);
            asm volatile("bar.arrive 2, 256;" ::: "memory");         // (x has been read)
            if (plain) {
#pragma unroll
                for (int m = 0; m < 8; ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int r = rg + 8 * m, q = cg + 16 * j;
                        sP[r * kZ + q] = 2 * j <= m && r >= q ? sum_of(acc[m][j]) * plain_f[2 * j <= m ? m - 2 * j : 0] : 0.f;
                    }
            } else {
                uint32_t wq[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) wq[j] = pl[cg + 16 * j];
#pragma unroll
                for (int m = 0; m < 8; ++m) {
                    const int r = rg + 8 * m;
                    const uint32_t wr = pl[r];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int q = cg + 16 * j;
                        float s = 0.f;
                        if (2 * j <= m) {
                            const bool seen = q <= r && !((wr | wq[j]) & kPadding) && place_run(wr) == place_run(wq[j]);
                            s = seen ? sum_of(acc[m][j]) * faded(rate2, abs(place_count(wr) - place_count(wq[j]))) : 0.f;
                        }
                        sP[r * kZ + q] = s;
                    }
                }
            }
        } else if (!STATES && group == 1) {
            // ---- past
            pair acc[8][4] = {};
            if (!empty) dots<DC, kX, false>(sX + rg * kX, sS + cg * kX, acc);
            asm volatile("bar.sync 2, 256;" ::: "memory");
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                const uint32_t w = pl[rg + 8 * m];
                const bool takes = !(w & kPadding) && place_run(w) == (back ? r1 : 0);
                const float t = takes ? faded(rate2, back ? c1 - place_count(w) : place_count(w)) : 0.f;
                *reinterpret_cast<float4*>(sX + (rg + 8 * m) * kX + 4 * cg) =
                    t == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f)       // (whatever the state holds)
                             : make_float4(sum_of(acc[m][0]) * t, sum_of(acc[m][1]) * t, sum_of(acc[m][2]) * t, sum_of(acc[m][3]) * t);
            }
        } else {
            // ---- state: rows 8 rg + 64 n, columns 4 cg ..; where only states are wanted, half of the tokens each group
            if (gt < kT) {
                const uint32_t w = pl[gt];
                const bool gives = !(w & kPadding) && place_run(w) == (back ? 0 : r1);
                if (!STATES || group == 0) give[gt] = gives ? faded(rate2, back ? place_count(w) : c1 - place_count(w)) : 0.f;
            }
            if (STATES) __syncthreads();
            else asm volatile("bar.sync 1, 128;" ::: "memory");
            if constexpr (STATES) {
                const pair ff = pairs::both(f);
#pragma unroll
                for (int n = 0; n < NH; ++n)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int u = 0; u < 4; ++u) st[n][k][u] = f == 0.f ? 0 : pairs::mul2(ff, st[n][k][u]);
            } else {
#pragma unroll
                for (int n = 0; n < NH; ++n)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int u = 0; u < 4; ++u) st[n][k][u] = 0;
            }
            if (!empty) {
                const int j0 = STATES ? group * (kT / 2) : 0;
#pragma unroll 2
                for (int j = j0; j < j0 + (STATES ? kT / 2 : kT); ++j) {
                    const float w = give[j];
                    const float4 z = lds4(sZ + j * kZ + 4 * cg);
                    const pair zs[4] = {pairs::both(z.x * w), pairs::both(z.y * w), pairs::both(z.z * w), pairs::both(z.w * w)};
#pragma unroll
                    for (int n = 0; n < NH; ++n) {
                        const ulonglong2 y0 = *reinterpret_cast<const ulonglong2*>(sY + j * kX + 64 * n + 8 * rg);
                        const ulonglong2 y1 = *reinterpret_cast<const ulonglong2*>(sY + j * kX + 64 * n + 8 * rg + 4);
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            st[n][0][u] = pairs::fma2(y0.x, zs[u], st[n][0][u]);
                            st[n][1][u] = pairs::fma2(y0.y, zs[u], st[n][1][u]);
                            st[n][2][u] = pairs::fma2(y1.x, zs[u], st[n][2][u]);
                            st[n][3][u] = pairs::fma2(y1.y, zs[u], st[n][3][u]);
                        }
                    }
                }
            }
        }
        if constexpr (!STATES) {
            __syncthreads();
            if (group == 2) {
                const pair ff = pairs::both(f);
#pragma unroll
                for (int n = 0; n < NH; ++n)
#pragma unroll
                    for (int u = 0; u < 4; ++u)
#pragma unroll
                        for (int k = 0; k < 4; k += 2) {
                            ulonglong2* s = reinterpret_cast<ulonglong2*>(sS + state_row(4 * cg + u) * kX + 64 * n + 8 * rg + 2 * k);
                            const ulonglong2 o = *s;                 // (a factor of 0 drops it, whatever it holds)
                            *s = f == 0.f ? make_ulonglong2(st[n][k][u], st[n][k + 1][u])
                                          : make_ulonglong2(pairs::fma2(ff, o.x, st[n][k][u]), pairs::fma2(ff, o.y, st[n][k + 1][u]));
                        }
            }
            // Rows rg + 8 m, m = group + 3 i: a row sees 8 m + 8 columns at most (the third group has two rows; its third one is the second)
            const int m2 = group == 2 ? 5 : group + 6;
            const float* const P[3] = {sP + (rg + 8 * group) * kZ, sP + (rg + 8 * group + 24) * kZ, sP + (rg + 8 * m2) * kZ};
            pair o[3][2] = {};
            if (!empty) {
                const float* z = sZ + 4 * cg;
                rows_of<0, kZ>(P, z, 0, 8 * group + 8, o);
                rows_of<1, kZ>(P, z, 8 * group + 8, 8 * group + 32, o);
                rows_of<2, kZ>(P, z, 8 * group + 32, group == 2 ? 0 : 8 * group + 56, o);
            }
            float* out = static_cast<float*>(const_cast<void*>(p.out.data)) + b * p.out.batch_stride + h * p.out.head_stride + e0 + 4 * cg;
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                const int r = rg + 8 * (group + 3 * k), t = t0 + (back ? kT - 1 - r : r);
                if (r < kT && t < L && e0 + 4 * cg < p.de) {
                    const float4 y = lds4(sX + r * kX + 4 * cg);
                    const float2 u = pairs::split(o[k][0]), v = pairs::split(o[k][1]);
                    *reinterpret_cast<float4*>(out + (long long)t * p.out.token_stride) =
                        make_float4((u.x + y.x) * a.c.factor, (u.y + y.y) * a.c.factor, (v.x + y.z) * a.c.factor, (v.y + y.w) * a.c.factor);
                }
            }
        }
        if (tid < kT) ring[(i + 2) % 3 * kT + tid] = ahead;
        whole *= f;
    }
    __syncthreads();
    if constexpr (STATES) {
        if (group == 1) {
#pragma unroll
            for (int n = 0; n < NH; ++n)
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int k = 0; k < 4; k += 2)
                        *reinterpret_cast<ulonglong2*>(sS + state_row(4 * cg + u) * kX + 64 * n + 8 * rg + 2 * k) = make_ulonglong2(st[n][k][u], st[n][k + 1][u]);
        }
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int n = 0; n < NH; ++n)
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int k = 0; k < 4; k += 2) {
                        ulonglong2* s = reinterpret_cast<ulonglong2*>(sS + state_row(4 * cg + u) * kX + 64 * n + 8 * rg + 2 * k);
                        const ulonglong2 o = *s;
                        *s = make_ulonglong2(pairs::add2(o.x, st[n][k][u]), pairs::add2(o.y, st[n][k + 1][u]));
                    }
        }
        __syncthreads();
        const long long slot = decay_slot(it.pass, a.c.passes, it.head, a.tiles, it.tile, a.segments, it.segment);
        float4* to = reinterpret_cast<float4*>(a.states + slot * kDecayMaxWidth * kTile);
        for (int i = tid; i < DC * kTile / 4; i += C::kThreads) to[i] = lds4(sS + i / (DC / 4) * kX + i % (DC / 4) * 4);
        if (tid == 0) a.factors[slot] = whole;
    } else {
        if (p.state_out && it.segment == a.segments - 1) {
            for (int i = tid; i < DC * kTile; i += C::kThreads) {
                const int c = p.turned ? i % DC : i / kTile, e = p.turned ? i / DC : i % kTile;
                if (c < p.dc && e0 + e < p.de)
                    p.state_out[it.head * p.dc * p.de + (p.turned ? (long long)(e0 + e) * p.dc + c : (long long)c * p.de + e0 + e)] =
                        p.out_factor * sS[state_row(e) * kX + c];
            }
        }
    }
}

template <int DC, bool STATES> based_status launch(const Args& a, long long ctas, bool behind, cudaStream_t stream) {
    if (cudaFuncSetAttribute(decay_f32_kernel<DC, STATES>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg<DC, STATES>::bytes) != cudaSuccess)
        return BASED_ERR_CUDA;
    const cudaError_t e = launch_ex(decay_f32_kernel<DC, STATES>, dim3((unsigned)ctas), dim3(Cfg<DC, STATES>::kThreads), Cfg<DC, STATES>::bytes, 1, behind, stream, a);
    note_launch();
    const based_status st = check_launch("decay_f32_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}

template <int DC> based_status launch_all(const Args& a, const DecayPlan& plan, cudaStream_t stream) {
    if (plan.segments > 1) {
        const based_status st = launch<DC, true>(a, plan.ctas / plan.segments * (plan.segments - 1), true, stream);
        if (st != BASED_OK) return st;
    }
    return launch<DC, false>(a, plan.ctas, true, stream);
}
bool wide(const DecayCall& c) {
    for (int i = 0; i < c.passes; ++i)
        if (c.pass[i].dc > 64) return true;
    return false;
}

}  // namespace

DecayPlan decay_plan_f32(const DecayCall& c) {
    int de = 0;
    for (int i = 0; i < c.passes; ++i) de = c.pass[i].de > de ? c.pass[i].de : de;
    return decay_plan(c.passes, de, c.B, c.H, c.L, c.documents != nullptr, kT, kTile, kSMs, {1.0, 0.3, 0.8, 0.1});
}

based_status launch_decay_f32(const DecayCall& c, const DecayPlan& plan, void* workspace, cudaStream_t stream) {
    char* ws = static_cast<char*>(workspace);
    uint32_t* places = c.documents ? reinterpret_cast<uint32_t*>(ws) : nullptr;
    if (places) {
        const based_status st = launch_decay_places(c.documents, places, c.B, c.L, kT, stream);
        if (st != BASED_OK) return st;
    }
    Args a{c, places, reinterpret_cast<float*>(ws + plan.places_bytes), reinterpret_cast<float*>(ws + plan.places_bytes + plan.states_bytes),
           plan.blocks, plan.segments, plan.tiles};
    return wide(c) ? launch_all<128>(a, plan, stream) : launch_all<64>(a, plan, stream);
}

}  // namespace based
