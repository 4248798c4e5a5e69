// Decay attention, fp32 io, on multiply-adds: the passes of decay.cuh in blocks of 64 tokens.
//
// One CTA of 256 threads per pass, head, tile of 64 output columns and segment.  Per block: scores x y^T (64 x 64), masked and faded into
// shared memory; out = take (x S) + P z; S <- f S + (give y)^T z, S in shared memory throughout.  A thread works on 4 x 4 outputs (its
// state rows: 4 columns x DC / 16), all operands 16 bytes at a time from rows padded by 4 floats, so that eight rows side by
// side fall into all 32 banks.
#include "decay.cuh"
#include "f32_tiles.cuh"

namespace based {

namespace {

constexpr int kT = kDecayBlockF32, kTile = 64, kThreads = 256;
template <int DC> struct Cfg {
    static constexpr int kX = DC + 4, kZ = kTile + 4;          // floats per row
    static constexpr int offY = kT * kX, offZ = 2 * kT * kX, offS = offZ + kT * kZ, offP = offS + DC * kZ, offW = offP + kT * kZ;
    static constexpr size_t bytes = sizeof(float) * (offW + 3 * kT);
};

struct Args {
    DecayCall c;
    const uint32_t* places;
    float *states, *factors;
    int blocks, segments, tiles;
};

// 4 values of a row, fp32
__device__ __forceinline__ float4 row4(const float* p) { return *reinterpret_cast<const float4*>(p); }

// rows t0 .. of a [B,H,L,width] view into shared memory: `cols` columns from `from` on; zeros outside and where a token is padding
template <int COLS>
__device__ __forceinline__ void load_rows(const based_heads& v, int b, int h, int t0, int L, int from, int width, const uint32_t* pl, float* dst) {
    const float* base = static_cast<const float*>(v.data) + b * v.batch_stride + h * v.head_stride;
#pragma unroll 4
    for (int i = threadIdx.x; i < kT * COLS / 4; i += kThreads) {
        const int r = i / (COLS / 4), c = i % (COLS / 4) * 4;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (!(pl[r] & kPadding) && from + c < width) x = row4(base + (long long)(t0 + r) * v.token_stride + from + c);
        *reinterpret_cast<float4*>(dst + r * (COLS + 4) + c) = x;
    }
}

template <int DC, bool STATES>
__global__ void __launch_bounds__(kThreads, DC == 64 ? 2 : 1) decay_f32_kernel(const __grid_constant__ Args a) {
    using C = Cfg<DC>;
    extern __shared__ __align__(16) float sm[];
    float *sX = sm, *sY = sm + C::offY, *sZ = sm + C::offZ, *sS = sm + C::offS, *sP = sm + C::offP;
    float *take = sm + C::offW, *give = take + kT;
    uint32_t* pl = reinterpret_cast<uint32_t*>(give + kT);
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const DecayItem it(blockIdx.x, a.c.passes, a.tiles, STATES ? a.segments - 1 : a.segments);
    const DecayPass& p = a.c.pass[it.pass];
    const int e0 = it.tile * kTile, L = a.c.L;
    enter_dependent();
    if (e0 >= p.de) return;
    const int b = (int)(it.head / a.c.H), h = (int)(it.head % a.c.H);
    const float rate2 = a.c.rate[h] * kLog2e;

    // the state that the segment begins with
    for (int i = tid; i < DC * kTile; i += kThreads) {
        const int c = i / kTile, e = i % kTile;
        float s = 0.f;
        if (!STATES) {
            if (p.state_in && c < p.dc && e0 + e < p.de)
                s = p.in_factor * p.state_in[it.head * p.dc * p.de + (p.turned ? (long long)(e0 + e) * p.dc + c : (long long)c * p.de + e0 + e)];
            for (int g = 0; g < it.segment; ++g) {
                const long long slot = decay_slot(it.pass, a.c.passes, it.head, a.tiles, it.tile, a.segments, g);
                // (a factor of 0 drops what was before, whatever it holds)
                const float f = a.factors[slot], x = a.states[slot * kDecayMaxWidth * kTile + i];
                s = f == 0.f ? x : fmaf(f, s, x);
            }
        }
        sS[c * C::kZ + e] = s;
    }
    const int g = p.back ? a.segments - 1 - it.segment : it.segment;
    const int first = decay_first(a.blocks, a.segments, g), count = decay_first(a.blocks, a.segments, g + 1) - first;
    float whole = 1.f;
    for (int i = 0; i < count; ++i) {
        const int n = p.back ? first + count - 1 - i : first + i, t0 = n * kT;
        if (tid < kT) pl[tid] = a.places ? a.places[((long long)b * a.blocks + n) * kT + tid]
                                         : (uint32_t)min(tid + 1, L - t0) | (tid < L - t0 ? 0u : kPadding);
        __syncthreads();
        const int c1 = place_count(pl[kT - 1]), r1 = place_run(pl[kT - 1]);
        if (c1 == 0) {                               // nothing but padding: zeros, and the state as it is
            if (!STATES)
                for (int j = tid; j < kT * kTile / 4; j += kThreads) {
                    const int t = t0 + j / (kTile / 4), e = e0 + j % (kTile / 4) * 4;
                    if (t < L && e < p.de)
                        *reinterpret_cast<float4*>(static_cast<float*>(const_cast<void*>(p.out.data)) + b * p.out.batch_stride + h * p.out.head_stride +
                                                   (long long)t * p.out.token_stride + e) = make_float4(0.f, 0.f, 0.f, 0.f);
                }
            __syncthreads();
            continue;
        }
        const float f = r1 == 0 ? faded(rate2, c1) : 0.f;
        if (tid < kT) {
            const uint32_t w = pl[tid];
            const bool pad = w & kPadding;
            const float up = !pad && place_run(w) == 0 ? faded(rate2, place_count(w)) : 0.f;
            const float down = !pad && place_run(w) == r1 ? faded(rate2, c1 - place_count(w)) : 0.f;
            take[tid] = p.back ? down : up;
            give[tid] = p.back ? up : down;
        }
        if (!STATES) load_rows<DC>(p.x, b, h, t0, L, 0, p.dc, pl, sX);
        load_rows<DC>(p.y, b, h, t0, L, 0, p.dc, pl, sY);
        load_rows<kTile>(p.z, b, h, t0, L, e0, p.de, pl, sZ);
        __syncthreads();
        if (!STATES) {
            {   // scores of rows ty + 16 i and columns tx + 16 j
                float2 acc[4][2] = {};
#pragma unroll 2
                for (int k = 0; k < DC; k += 4) {
                    float4 x[4], y[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = lds4(sX + (ty + 16 * i) * C::kX + k);
#pragma unroll
                    for (int j = 0; j < 4; ++j) y[j] = lds4(sY + (tx + 16 * j) * C::kX + k);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            fma_pair(acc[i][j], y[2 * j].x, y[2 * j + 1].x, x[i].x);
                            fma_pair(acc[i][j], y[2 * j].y, y[2 * j + 1].y, x[i].y);
                            fma_pair(acc[i][j], y[2 * j].z, y[2 * j + 1].z, x[i].z);
                            fma_pair(acc[i][j], y[2 * j].w, y[2 * j + 1].w, x[i].w);
                        }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int r = ty + 16 * i, q = tx + 16 * j;
                        const uint32_t wr = pl[r], wq = pl[q];
                        const int steps = p.back ? place_count(wq) - place_count(wr) : place_count(wr) - place_count(wq);
                        const bool seen = (p.back ? q >= r : q <= r) && !((wr | wq) & kPadding) && place_run(wr) == place_run(wq);
                        const float s = j & 1 ? acc[i][j >> 1].y : acc[i][j >> 1].x;
                        sP[r * C::kZ + q] = seen ? s * faded(rate2, steps) : 0.f;
                    }
            }
            __syncthreads();
            {   // out of rows ty + 16 i and columns 4 tx ..
                float2 acc[4][2] = {};
#pragma unroll 2
                for (int k = 0; k < DC; k += 4) {
                    float4 x[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = lds4(sX + (ty + 16 * i) * C::kX + k);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const float4 s = lds4(sS + (k + u) * C::kZ + 4 * tx);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float xs = u == 0 ? x[i].x : u == 1 ? x[i].y : u == 2 ? x[i].z : x[i].w;
                            fma_pair(acc[i][0], s.x, s.y, xs);
                            fma_pair(acc[i][1], s.z, s.w, xs);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float t = take[ty + 16 * i];
                    acc[i][0] = make_float2(t == 0.f ? 0.f : acc[i][0].x * t, t == 0.f ? 0.f : acc[i][0].y * t);
                    acc[i][1] = make_float2(t == 0.f ? 0.f : acc[i][1].x * t, t == 0.f ? 0.f : acc[i][1].y * t);
                }
#pragma unroll 2
                for (int k = 0; k < kT; k += 4) {
                    float4 x[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = lds4(sP + (ty + 16 * i) * C::kZ + k);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const float4 s = lds4(sZ + (k + u) * C::kZ + 4 * tx);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float xs = u == 0 ? x[i].x : u == 1 ? x[i].y : u == 2 ? x[i].z : x[i].w;
                            fma_pair(acc[i][0], s.x, s.y, xs);
                            fma_pair(acc[i][1], s.z, s.w, xs);
                        }
                    }
                }
                float* out = static_cast<float*>(const_cast<void*>(p.out.data)) + b * p.out.batch_stride + h * p.out.head_stride + e0 + 4 * tx;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = t0 + ty + 16 * i;
                    if (t < L && e0 + 4 * tx < p.de)
                        *reinterpret_cast<float4*>(out + (long long)t * p.out.token_stride) =
                            make_float4(acc[i][0].x * a.c.factor, acc[i][0].y * a.c.factor, acc[i][1].x * a.c.factor, acc[i][1].y * a.c.factor);
                }
            }
            __syncthreads();
        }
        {   // state rows ty DC / 16 .. and columns 4 tx ..
            constexpr int R = DC / 16;
            float2 acc[R][2] = {};
#pragma unroll 2
            for (int j = 0; j < kT; ++j) {
                const float w = give[j];
                float4 z = lds4(sZ + j * C::kZ + 4 * tx);
                z = make_float4(z.x * w, z.y * w, z.z * w, z.w * w);
#pragma unroll
                for (int r = 0; r < R; r += 4) {
                    const float4 y = lds4(sY + j * C::kX + ty * R + r);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const float ys = u == 0 ? y.x : u == 1 ? y.y : u == 2 ? y.z : y.w;
                        fma_pair(acc[r + u][0], z.x, z.y, ys);
                        fma_pair(acc[r + u][1], z.z, z.w, ys);
                    }
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float4* s = reinterpret_cast<float4*>(sS + (ty * R + r) * C::kZ + 4 * tx);
                const float4 o = f == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : *s;              // (0 drops it, whatever it holds)
                *s = make_float4(fmaf(f, o.x, acc[r][0].x), fmaf(f, o.y, acc[r][0].y), fmaf(f, o.z, acc[r][1].x), fmaf(f, o.w, acc[r][1].y));
            }
        }
        whole *= f;
        __syncthreads();
    }
    if (STATES) {
        const long long slot = decay_slot(it.pass, a.c.passes, it.head, a.tiles, it.tile, a.segments, it.segment);
        for (int i = tid; i < DC * kTile; i += kThreads)
            a.states[slot * kDecayMaxWidth * kTile + i] = sS[i / kTile * C::kZ + i % kTile];
        if (tid == 0) a.factors[slot] = whole;
    } else if (p.state_out && it.segment == a.segments - 1) {
        for (int i = tid; i < p.dc * kTile; i += kThreads) {
            // (neighbouring threads along the state's rows, whichever way it lies)
            const int c = p.turned ? i % p.dc : i / kTile, e = p.turned ? i / p.dc : i % kTile;
            if (e0 + e < p.de)
                p.state_out[it.head * p.dc * p.de + (p.turned ? (long long)(e0 + e) * p.dc + c : (long long)c * p.de + e0 + e)] =
                    p.out_factor * sS[c * C::kZ + e];
        }
    }
}

template <int DC, bool STATES> based_status launch(const Args& a, long long ctas, bool behind, cudaStream_t stream) {
    if (cudaFuncSetAttribute(decay_f32_kernel<DC, STATES>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg<DC>::bytes) != cudaSuccess)
        return BASED_ERR_CUDA;
    const cudaError_t e = launch_ex(decay_f32_kernel<DC, STATES>, dim3((unsigned)ctas), dim3(kThreads), Cfg<DC>::bytes, 1, behind, stream, a);
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
    return decay_plan(c.passes, de, c.B, c.H, c.L, c.documents != nullptr, kT, kTile, wide(c) ? kSMs : 2 * kSMs, {1.0, 0.4, 0.8, 0.1});
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
