// Softmax attention of one new token per sequence over a paged key-value cache.
//
//   s_j = cap tanh(scale q . k_j / cap) - slope (pos - j),   o = sum_j exp(s_j) v_j / sum_j exp(s_j),   j = max(0, pos - window + 1) .. pos
//
// Bound by HBM: every key and value is read once for all query heads that share it (Hq / Hk of them, the rows of a product), 2 d elements
// a token against 4 d Hq / Hk flop.  What has to be right is the division of the work: sequences have any lengths, known to the device alone.
//   - The unit is 64 tokens of one sequence and key head; all units lie in one row (sequence, head, tokens), and CTA i of G takes
//     units U i / G .. U (i + 1) / G: equal shares whatever the lengths, from one sequence of 131072 tokens to many short ones.
//   - A CTA's four warps take 16 tokens of a unit each, with rings of their own that copies (16 bytes a lane) fill two or three units ahead, and
//     a running maximum, sum and output of their own: no barrier but at the end of a (sequence, head).
//   - What a CTA has done whole it writes as output; the pieces at its range's ends go to the workspace, and a second, dependent launch
//     joins every output that was cut, its pieces in order.
// bf16: products on the tensor cores (m16n8k16: 16 query heads a row block, weights rounded to bf16 once, 2^-9 of each at most in the mean);
// fp32: multiply-adds, a lane per token and half a row for the scores, a lane per 2 or 4 columns for the output.
#include "paged.cuh"

#include "pairs.cuh"

namespace based {

namespace {

constexpr int kUnit = 64, kWarps = 4, kThreads = 128, kSub = 16;         // tokens of a unit, of a warp's share
constexpr unsigned kBadPage = 2u;                                        // in the error word
constexpr float kLog2e = 1.4426950408889634f;

// R: query heads at a time, 16 on tensor cores, else as many as share a key head (8 at most)
template <typename T, int DP, int R> struct Cfg {
    static constexpr bool kTc = sizeof(T) == 2;
    static constexpr int kRows = R;
    static constexpr int kRowBytes = DP * sizeof(T), kChunks = kRowBytes / 16;
    static constexpr int kStage = 2 * kSub * kRowBytes;                  // a warp's keys and values of a unit
    static constexpr int kStages = kStage >= 16384 ? 3 : kStage >= 8192 ? 3 : 4;
    static constexpr int kBytes = kWarps * kStages * kStage + kRows * DP * 4;      // and the queries, fp32
    static constexpr int kPerSm = kBytes > 113000 ? 1 : kBytes > 74000 ? 2 : 3;
    static constexpr int kPiece = kRows * (DP + 2);                      // floats of a piece: per row the maximum, the sum, the output
    static_assert(kStages * kStage >= kPiece * 4, "a warp's piece goes into its ring");
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// A sequence's keys: tokens lo .. pos, in units first .. first + count - 1 of 64 tokens from the start; none where it has no token, or one
// past what its pages can hold
struct Span {
    int pos, lo, first, count;
    __device__ __forceinline__ Span(const PagedCall& c, int b) {
        pos = c.pos[b];
        if (pos < 0 || pos >= c.max_pages * c.page_size) {
            lo = first = count = 0;
            return;
        }
        lo = c.window > 0 && pos >= c.window ? pos - c.window + 1 : 0;
        first = lo / kUnit;
        count = pos / kUnit - first + 1;
    }
};

// The units of all sequences in one row, cut into G shares that differ by one at most
struct Shares {
    long long total, base, more;                                         // the first `more` shares have base + 1 units
    int G;
    __device__ __forceinline__ Shares(long long total_, int G_) : total(total_), G(G_) {
        if (total >> 31 == 0) {
            base = (unsigned)total / (unsigned)G;
            more = (unsigned)total % (unsigned)G;
        } else {
            base = total / G;
            more = total % G;
        }
    }
    __device__ __forceinline__ long long begin(long long i) const { return i * base + (i < more ? i : more); }
    __device__ __forceinline__ long long of(long long x) const {
        const long long wide = more * (base + 1);
        if (total >> 31 == 0) return x < wide ? (unsigned)x / (unsigned)(base + 1) : more + (unsigned)(x - wide) / (unsigned)base;
        return x < wide ? x / (base + 1) : more + (x - wide) / base;
    }
};

struct Args {
    PagedCall c;
    float* pieces;                                                       // [2 G][rows][d + 2]
    unsigned int* err;
    int blocks;                                                          // row blocks of a key head's queries
    int shift;                                                           // page_size = 1 << shift, or -1
    bool whole;                                                          // 16 tokens from a multiple of 16 on lie in one page
};

template <typename T, int DP, int R>
__global__ void __launch_bounds__(kThreads, Cfg<T, DP, R>::kPerSm) paged_decode_kernel(const __grid_constant__ Args a) {
    using C = Cfg<T, DP, R>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long s_sum[4], s_from[2];
    const PagedCall& c = a.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint8_t* ring = smem + warp * C::kStages * C::kStage;
    float* sq = reinterpret_cast<float*>(smem + kWarps * C::kStages * C::kStage);
    const int group = c.Hq / c.Hk, heads = c.Hk * a.blocks;              // "heads": key heads and row blocks of their queries
    enter_dependent();

    // This CTA's units, and the sequence that they begin in: inclusive sums of the sequences' units, 128 a turn, by shuffles.  Twice where there are
    // more sequences than that (the first time for the total alone)
    long long total = 0, u = 0, end = 0, base = 0;                       // base: the units of the sequences before b
    int b = 0;
    for (int pass = c.B > kThreads ? 0 : 1; pass < 2; ++pass) {
        long long before = 0;
        for (int b0 = 0; b0 < c.B; b0 += kThreads) {
            const long long n = b0 + tid < c.B ? (long long)Span(c, b0 + tid).count * heads : 0;
            long long sum = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long x = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += x;
            }
            __syncthreads();
            if (lane == 31) s_sum[warp] = sum;
            __syncthreads();
            long long off = before;
            for (int w = 0; w < warp; ++w) off += s_sum[w];
            sum += off;
            before += s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
            if (pass == 1) {
                if (c.B <= kThreads) total = before;
                if (b0 == 0) {
                    const Shares sh(total, (int)gridDim.x);
                    u = sh.begin(blockIdx.x);
                    end = sh.begin(blockIdx.x + 1);
                    if (u >= end) return;
                }
                if (sum - n <= u && u < sum) {
                    s_from[0] = b0 + tid;
                    s_from[1] = sum - n;
                }
                if (before > u) break;
            }
        }
        if (pass == 0) total = before;
    }
    __syncthreads();
    b = (int)s_from[0];
    base = s_from[1];
    const long long range = u;

    for (; u < end; ) {
        Span sp(c, b);
        while ((long long)sp.count * heads <= u - base && b + 1 < c.B) { // on to the next sequence that has keys
            base += (long long)sp.count * heads;
            sp = Span(c, ++b);
        }
        if (sp.count == 0) return;
        const int hm = (int)((u - base) / sp.count), unit0 = (int)((u - base) % sp.count);
        const int units = (int)min((long long)(sp.count - unit0), end - u);
        const int hk = hm / a.blocks, row0 = (hm % a.blocks) * C::kRows, rows = min(C::kRows, group - row0);
        const int h0 = hk * group + row0;                                // the first query head
        const T* q = static_cast<const T*>(c.q) + ((long long)b * c.Hq + h0) * c.d;
        const T* knew = static_cast<const T*>(c.k) + ((long long)b * c.Hk + hk) * c.d;
        const T* vnew = static_cast<const T*>(c.v) + ((long long)b * c.Hk + hk) * c.d;
        T* kp = static_cast<T*>(c.k_pages) + hk * c.head_stride;
        T* vp = static_cast<T*>(c.v_pages) + hk * c.head_stride;
        const int* table = c.table + (long long)b * c.max_pages;

        // tokens j0 .. j0 + 15 of unit n are this warp's; lane < 16 (and its double) looks up the page of token j0 + lane a turn before it is needed:
        // what is checked is checked then, so that nothing waits for the table
        auto tokens = [&](int n) { return (sp.first + unit0 + n) * kUnit + warp * kSub; };
        auto page_of = [&](int j) { return a.shift >= 0 ? j >> a.shift : (int)((unsigned)j / (unsigned)c.page_size); };
        auto here = [&](int n, int j) { return n < units && j <= sp.pos && j >= sp.lo; };
        auto look = [&](int n) -> int {
            const int j = tokens(n) + (lane & 15);
            return here(n, j) ? table[page_of(j)] : 0;
        };
        // tokens strictly inside, whose page is one: nothing to check but that
        auto inside = [&](int n) { const int j0 = tokens(n); return n < units && j0 >= sp.lo && j0 + kSub <= sp.pos; };
        constexpr int V = 16 / (int)sizeof(T), kStep = 32 / C::kChunks > 0 ? 32 / C::kChunks : 1;          // values of a chunk, rows of a turn
        const int lrow = lane / C::kChunks, lch = lane % C::kChunks;     // (fp32, 128 wide: a row a turn)
        const bool lin = lch * V < c.d;
        const long long lane_at = lrow * c.token_stride + (lin ? lch * V : 0);
        auto load = [&](int n, int id) {
            uint8_t* st = ring + n % C::kStages * C::kStage;
            const int j0 = tokens(n), j = j0 + (lane & 15);
            if (a.whole && inside(n) && (unsigned)id < (unsigned)c.pages) {
                const long long at = id * c.page_stride + (long long)(j0 - page_of(j0) * c.page_size) * c.token_stride + lane_at;
                const T *ks = kp + at, *vs = vp + at;
                const long long step = kStep * c.token_stride;
#pragma unroll
                for (int i = 0; i < kSub / kStep; ++i) {
                    const int row = i * kStep + lrow;
                    uint8_t* to = st + row * C::kRowBytes + ((lch ^ (row & 7)) << 4);
                    pairs::copy_async16(to, ks, lin);
                    pairs::copy_async16(to + kSub * C::kRowBytes, vs, lin);
                    ks += step;
                    vs += step;
                }
                pairs::copy_async_commit();
                return;
            }
            long long at = -1;
            if (here(n, j)) {
                if ((unsigned)id < (unsigned)c.pages) at = id * c.page_stride + (long long)(j - page_of(j) * c.page_size) * c.token_stride;
                else atomicOr(a.err, kBadPage);
            }
#pragma unroll 1
            for (int i = 0; i < kSub / kStep; ++i) {
                const int row = i * kStep + lrow;
                const long long off = __shfl_sync(0xffffffffu, at, row);
                const bool fresh = j0 + row == sp.pos && n < units;      // the new token's, which may not be in its page yet
                const bool in = (off >= 0 || fresh) && lin;
                const T *ks = fresh ? knew : kp + (off >= 0 ? off : 0), *vs = fresh ? vnew : vp + (off >= 0 ? off : 0);
                uint8_t* to = st + row * C::kRowBytes + ((lch ^ (row & 7)) << 4);
                pairs::copy_async16(to, in ? ks + lch * V : c.q, in);
                pairs::copy_async16(to + kSub * C::kRowBytes, in ? vs + lch * V : c.q, in);
            }
            pairs::copy_async_commit();
        };

        __syncthreads();                                                 // (the rings and the queries are free)
        for (int i = tid; i < C::kRows * DP; i += kThreads) {
            const int r = i / DP, e = i % DP;
            sq[i] = r < rows && e < c.d ? to_f32(q[(long long)r * c.d + e]) : 0.f;
        }
        int next = look(0);
#pragma unroll
        for (int n = 0; n < C::kStages - 1; ++n) {
            const int id = next;
            next = look(n + 1);
            load(n, id);
        }
        __syncthreads();

        // running maximum (base 2), sum, output
        constexpr int kN = C::kTc ? DP / 8 : C::kRows;
        float m[C::kTc ? 2 : C::kRows], l[C::kTc ? 2 : C::kRows], acc[kN][C::kTc ? 4 : DP / 32];
#pragma unroll
        for (int i = 0; i < (C::kTc ? 2 : C::kRows); ++i) {
            m[i] = -INFINITY;
            l[i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < kN; ++i)
#pragma unroll
            for (int k = 0; k < (C::kTc ? 4 : DP / 32); ++k) acc[i][k] = 0.f;
        uint32_t qf[C::kTc ? DP / 16 : 1][4];
        float slope[C::kTc ? 2 : 1] = {};
        if constexpr (C::kTc) {
            const int r = lane >> 2, e = (lane & 3) * 2;
#pragma unroll
            for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float* s = sq + (r + (i & 1) * 8) * DP + 16 * k + e + (i >> 1) * 8;
                    qf[k][i] = pack2(s[0], s[1]);                        // (bf16 values: exact)
                }
            if (c.slopes) {
                slope[0] = r < rows ? c.slopes[h0 + r] : 0.f;
                slope[1] = r + 8 < rows ? c.slopes[h0 + r + 8] : 0.f;
            }
        }
        const bool modified = c.cap > 0.f || c.slopes;
        // a score as the softmax takes it, in base 2
        auto weigh = [&](float s, float sl, int j) -> float {
            if (j > sp.pos || j < sp.lo) return -INFINITY;
            s *= c.scale;
            if (c.cap > 0.f) s = c.cap * tanhf(s / c.cap);
            if (c.slopes) s -= sl * (float)(sp.pos - j);
            return s * kLog2e;
        };

        for (int n = 0; n < units; ++n) {
            {
                const int id = next;
                next = look(n + C::kStages);
                load(n + C::kStages - 1, id);
            }
            pairs::copy_async_wait<C::kStages - 1>();
            __syncwarp();
            const int j0 = tokens(n);
            uint8_t* st = ring + n % C::kStages * C::kStage;
            if (j0 <= sp.pos && j0 + kSub > sp.lo) {
                const uint32_t ks = static_cast<uint32_t>(__cvta_generic_to_shared(st)), vs = ks + kSub * C::kRowBytes;
                if constexpr (C::kTc) {
                    float s[2][4] = {};
                    const int mr = (lane & 7) + (lane >> 4) * 8, mc = lane >> 3 & 1;     // a lane's row and chunk of four 8 x 8 pieces
#pragma unroll
                    for (int k = 0; k < DP / 16; ++k) {
                        uint32_t f[4];
                        ldmatrix4(f, ks + mr * C::kRowBytes + (((2 * k + mc) ^ (mr & 7)) << 4));
                        mma16816(s[0], qf[k], f[0], f[1]);
                        mma16816(s[1], qf[k], f[2], f[3]);
                    }
                    float fade[2];
                    const bool plain = !modified && inside(n);           // the scores as they are, all of them
                    const float sc = plain ? c.scale * kLog2e : 1.f;
                    if (!plain) {
#pragma unroll
                        for (int t = 0; t < 2; ++t)
#pragma unroll
                            for (int x = 0; x < 4; ++x) s[t][x] = weigh(s[t][x], slope[x >> 1], j0 + 8 * t + (lane & 3) * 2 + (x & 1));
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {                        // rows lane / 4 and lane / 4 + 8
                        float top = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                        const float to = fmaxf(m[h], top * sc), z = to == -INFINITY ? 0.f : to;
                        fade[h] = ex2(m[h] - z);
                        m[h] = to;
                        float sum = 0.f;
#pragma unroll
                        for (int t = 0; t < 2; ++t)
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                s[t][2 * h + x] = ex2(fmaf(s[t][2 * h + x], sc, -z));
                                sum += s[t][2 * h + x];
                            }
                        l[h] = fmaf(l[h], fade[h], sum);
                    }
                    if (__any_sync(0xffffffffu, fade[0] != 1.f || fade[1] != 1.f)) {      // (seldom, once the largest score has come)
#pragma unroll
                        for (int k = 0; k < DP / 8; ++k) {
                            acc[k][0] *= fade[0];
                            acc[k][1] *= fade[0];
                            acc[k][2] *= fade[1];
                            acc[k][3] *= fade[1];
                        }
                    }
                    const uint32_t p[4] = {pack2(s[0][0], s[0][1]), pack2(s[0][2], s[0][3]), pack2(s[1][0], s[1][1]), pack2(s[1][2], s[1][3])};
                    const int vr = lane & 15, vc = lane >> 4;
#pragma unroll
                    for (int k = 0; k < DP / 16; ++k) {
                        uint32_t f[4];
                        ldmatrix4t(f, vs + vr * C::kRowBytes + (((2 * k + vc) ^ (vr & 7)) << 4));
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            mma16816(acc[2 * k + x], p, f[2 * x], f[2 * x + 1]);
                        }
                    }
                } else {
                    // scores: lane = token (lane & 15) and half of its row; every lane ends with the scores of its token
                    const int tok = lane & 15, half = lane >> 4;
                    float s[C::kRows] = {};
#pragma unroll 2
                    for (int k = 0; k < C::kChunks / 2; ++k) {
                        const int ch = half * (C::kChunks / 2) + k;
                        const float4 x = *reinterpret_cast<const float4*>(st + tok * C::kRowBytes + ((ch ^ (tok & 7)) << 4));
#pragma unroll
                        for (int r = 0; r < C::kRows; ++r) {             // (rows past the last: queries of zeros)
                            const float4 y = *reinterpret_cast<const float4*>(sq + r * DP + 4 * ch);
                            s[r] = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s[r]))));
                        }
                    }
                    const bool plain = !modified && inside(n);
#pragma unroll
                    for (int r = 0; r < C::kRows; ++r) {
                        s[r] += __shfl_xor_sync(0xffffffffu, s[r], 16);
                        s[r] = plain ? s[r] * (c.scale * kLog2e) : weigh(s[r], c.slopes && r < rows ? c.slopes[h0 + r] : 0.f, j0 + tok);
                        float top = s[r];
#pragma unroll
                        for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                        const float to = fmaxf(m[r], top), z = to == -INFINITY ? 0.f : to, fade = exp2f(m[r] - z);
                        m[r] = to;
                        s[r] = exp2f(s[r] - z);
                        l[r] = fmaf(l[r], fade, s[r]);                   // a lane's own tokens: joined at the end
#pragma unroll
                        for (int x = 0; x < DP / 32; ++x) acc[r][x] *= fade;
                    }
                    // output: lane = DP / 32 columns
#pragma unroll 4
                    for (int t = 0; t < kSub; ++t) {
                        const uint8_t* row = st + (kSub + t) * C::kRowBytes;
                        float x[DP / 32];
                        if constexpr (DP == 128) {
                            const float4 y = *reinterpret_cast<const float4*>(row + ((lane ^ (t & 7)) << 4));
                            x[0] = y.x; x[1] = y.y; x[2] = y.z; x[3] = y.w;
                        } else {
                            const float2 y = *reinterpret_cast<const float2*>(row + (((lane >> 1) ^ (t & 7)) << 4) + (lane & 1) * 8);
                            x[0] = y.x; x[1] = y.y;
                        }
#pragma unroll
                        for (int r = 0; r < C::kRows; ++r) {
                            const float w = __shfl_sync(0xffffffffu, s[r], t);
#pragma unroll
                            for (int k = 0; k < DP / 32; ++k) acc[r][k] = fmaf(w, x[k], acc[r][k]);
                        }
                    }
                }
                // the new token into its page, once for a key head
                if (row0 == 0 && j0 <= sp.pos && sp.pos < j0 + kSub) {
                    const int page = a.shift >= 0 ? sp.pos >> a.shift : (int)((unsigned)sp.pos / (unsigned)c.page_size), id = table[page];
                    if ((unsigned)id < (unsigned)c.pages) {
                        const long long at = id * c.page_stride + (long long)(sp.pos - page * c.page_size) * c.token_stride;
                        constexpr int V = 16 / sizeof(T);
                        for (int e = lane; e < 2 * (c.d / V); e += 32) {
                            const bool key = e < c.d / V;
                            const int x = (key ? e : e - c.d / V) * V;
                            *reinterpret_cast<uint4*>((key ? kp : vp) + at + x) = *reinterpret_cast<const uint4*>((key ? knew : vnew) + x);
                        }
                    }
                }
            }
            __syncwarp();                                                // (the stage is read; the next turn's load overwrites it)
        }
        pairs::copy_async_wait<0>();
        __syncwarp();

        // the warps' shares, then the four as one: a whole output, or a piece
        float* piece = reinterpret_cast<float*>(ring);
        if constexpr (C::kTc) {
            l[0] += __shfl_xor_sync(0xffffffffu, l[0], 1);
            l[0] += __shfl_xor_sync(0xffffffffu, l[0], 2);
            l[1] += __shfl_xor_sync(0xffffffffu, l[1], 1);
            l[1] += __shfl_xor_sync(0xffffffffu, l[1], 2);
            const int r = lane >> 2;
#pragma unroll
            for (int k = 0; k < DP / 8; ++k)
#pragma unroll
                for (int x = 0; x < 4; ++x) piece[(r + (x >> 1) * 8) * (DP + 2) + 2 + 8 * k + (lane & 3) * 2 + (x & 1)] = acc[k][x];
            if ((lane & 3) == 0) {
                piece[r * (DP + 2)] = m[0];
                piece[r * (DP + 2) + 1] = l[0];
                piece[(r + 8) * (DP + 2)] = m[1];
                piece[(r + 8) * (DP + 2) + 1] = l[1];
            }
        } else {
#pragma unroll
            for (int r = 0; r < C::kRows; ++r) {
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], o);
#pragma unroll
                for (int k = 0; k < DP / 32; ++k) piece[r * (DP + 2) + 2 + lane * (DP / 32) + k] = acc[r][k];
                if (lane == 0) {
                    piece[r * (DP + 2)] = m[r];
                    piece[r * (DP + 2) + 1] = l[r];
                }
            }
        }
        __syncthreads();
        const bool all = units == sp.count;
        float* to = a.pieces + (2 * (long long)blockIdx.x + (u != range)) * C::kPiece;
        for (int i = tid; i < rows * DP; i += kThreads) {
            const int r = i / DP, e = i % DP;
            float top = -INFINITY, sum = 0.f, o = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, reinterpret_cast<const float*>(smem + w * C::kStages * C::kStage)[r * (DP + 2)]);
            const float z = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float* x = reinterpret_cast<const float*>(smem + w * C::kStages * C::kStage) + r * (DP + 2);
                const float f = exp2f(x[0] - z);
                sum = fmaf(x[1], f, sum);
                o = fmaf(x[2 + e], f, o);
            }
            if (all) {
                if (e < c.d) static_cast<T*>(c.out)[((long long)b * c.Hq + h0 + r) * c.d + e] = from_f32<T>(o / sum);
            } else {
                to[r * (DP + 2) + 2 + e] = o;
                if (e == 0) {
                    to[r * (DP + 2)] = top;
                    to[r * (DP + 2) + 1] = sum;
                }
            }
        }
        u += units;
    }
}

// the outputs that were cut, from their pieces, and zeros where a sequence has no token; a CTA per sequence and "head"
template <typename T, int DP, int R> __global__ void __launch_bounds__(kThreads) paged_join_kernel(const __grid_constant__ Args a, int G) {
    using C = Cfg<T, DP, R>;
    __shared__ long long s_sum[8];
    const PagedCall& c = a.c;
    const int heads = c.Hk * a.blocks, group = c.Hq / c.Hk, b = blockIdx.x / heads, hm = blockIdx.x % heads;
    const int row0 = (hm % a.blocks) * C::kRows, rows = min(C::kRows, group - row0), h0 = (hm / a.blocks) * group + row0;
    enter_dependent();
    const Span sp(c, b);
    T* out = static_cast<T*>(c.out) + ((long long)b * c.Hq + h0) * c.d;
    if (sp.count == 0) {
        for (int i = threadIdx.x; i < rows * c.d; i += kThreads) out[i] = from_f32<T>(0.f);
        if (threadIdx.x == 0 && sp.pos >= 0) atomicOr(a.err, kBadPage);
        return;
    }
    long long mine[2] = {0, 0};                                          // the units before this sequence, and of all
    for (int k = threadIdx.x; k < c.B; k += kThreads) {
        const int n = Span(c, k).count;
        mine[0] += k < b ? n : 0;
        mine[1] += n;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        mine[0] += __shfl_xor_sync(0xffffffffu, mine[0], o);
        mine[1] += __shfl_xor_sync(0xffffffffu, mine[1], o);
    }
    if ((threadIdx.x & 31) == 0) {
        s_sum[threadIdx.x >> 5] = mine[0];
        s_sum[4 + (threadIdx.x >> 5)] = mine[1];
    }
    __syncthreads();
    const long long first = (s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3]) * heads + (long long)hm * sp.count, last = first + sp.count - 1;
    const Shares sh((s_sum[4] + s_sum[5] + s_sum[6] + s_sum[7]) * heads, G);
    const long long i0 = sh.of(first), i1 = sh.of(last);
    if (i0 == i1) return;
    const bool begun = sh.begin(i0) != first;                            // the first CTA had something else before it
    const int count = (int)(i1 - i0) + 1;
    const float* from = a.pieces + 2 * i0 * C::kPiece;
    for (int k = threadIdx.x; k < rows * DP; k += kThreads) {
        const int r = k / DP, e = k % DP;
        if (e >= c.d) continue;
        float top = -INFINITY, sum = 0.f, o = 0.f;
        for (int i = 0; i < count; i += 8) {                             // eight pieces' values asked for at once
            float x[8][3];
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const float* p = from + (2 * (long long)(i + s) + (i + s == 0 && begun)) * C::kPiece + r * (DP + 2);
                x[s][0] = i + s < count ? p[0] : -INFINITY;
                x[s][1] = i + s < count ? p[1] : 0.f;
                x[s][2] = i + s < count ? p[2 + e] : 0.f;
            }
            float to = top;
#pragma unroll
            for (int s = 0; s < 8; ++s) to = fmaxf(to, x[s][0]);
            const float z = to == -INFINITY ? 0.f : to, f = exp2f(top - z);
            sum *= f;
            o *= f;
            top = to;
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const float g = exp2f(x[s][0] - z);
                sum = fmaf(x[s][1], g, sum);
                o = fmaf(x[s][2], g, o);
            }
        }
        out[r * c.d + e] = from_f32<T>(o / sum);
    }
}

template <int R> int row_blocks(int Hq, int Hk) { return (Hq / Hk + R - 1) / R; }
// CTAs of a launch: what the device holds at a time, or one per unit where there cannot be as many
template <typename T, int DP, int R> int grid_of(int B, int Hq, int Hk, int page_size, int max_pages) {
    const long long units = (long long)B * Hk * row_blocks<R>(Hq, Hk) * (((long long)max_pages * page_size + kUnit - 1) / kUnit);
    const int most = kSMs * Cfg<T, DP, R>::kPerSm;
    return units < most ? (int)units : most;
}

template <typename T, int DP, int R> based_status launch(const PagedCall& c, void* workspace, cudaStream_t stream) {
    using C = Cfg<T, DP, R>;
    static std::atomic<bool> ready[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return BASED_ERR_CUDA;
    if (!ready[dev].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(paged_decode_kernel<T, DP, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kBytes) != cudaSuccess) return BASED_ERR_CUDA;
        ready[dev].store(true, std::memory_order_release);
    }
    Args a{c, static_cast<float*>(workspace), nullptr, row_blocks<R>(c.Hq, c.Hk), -1, c.page_size % kSub == 0};
    if (error_word_ptr(&a.err) != BASED_OK) return BASED_ERR_CUDA;
    for (int s = 0; s < 31; ++s)
        if (c.page_size == 1 << s) a.shift = s;
    const int G = grid_of<T, DP, R>(c.B, c.Hq, c.Hk, c.page_size, c.max_pages);
    cudaError_t e = launch_ex(paged_decode_kernel<T, DP, R>, dim3(G), dim3(kThreads), C::kBytes, 1, true, stream, a);
    note_launch();
    based_status st = check_launch("paged_decode_kernel");
    if (e != cudaSuccess || st != BASED_OK) return e != cudaSuccess ? BASED_ERR_CUDA : st;
    e = launch_ex(paged_join_kernel<T, DP, R>, dim3((unsigned)((long long)c.B * c.Hk * a.blocks)), dim3(kThreads), 0, 1, true, stream, a, G);
    note_launch();
    st = check_launch("paged_join_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}
// f with the kernel's type, width and rows for a call: f(T{}, width, rows) as types
template <int N> struct Num { static constexpr int value = N; };
template <typename F> auto for_call(based_dtype io, int d, int group, F f) {
    if (io == BASED_BF16) return d > 64 ? f(__nv_bfloat16(), Num<128>(), Num<16>()) : f(__nv_bfloat16(), Num<64>(), Num<16>());
    if (group == 1) return d > 64 ? f(0.f, Num<128>(), Num<1>()) : f(0.f, Num<64>(), Num<1>());
    if (group <= 4) return d > 64 ? f(0.f, Num<128>(), Num<4>()) : f(0.f, Num<64>(), Num<4>());
    return d > 64 ? f(0.f, Num<128>(), Num<8>()) : f(0.f, Num<64>(), Num<8>());
}

// ------------------------------------------------------------------------------------------------ a prompt into its pages
// 64 tokens of one head per CTA: the rows' loads do not wait for the table's
template <typename T>
__global__ void __launch_bounds__(256) paged_write_kernel(const __grid_constant__ PagedWrite c, unsigned int* err, int tiles) {
    enter_dependent();
    unsigned i = blockIdx.x;
    const int t0 = (int)(i % (unsigned)tiles) * 64;
    i /= (unsigned)tiles;
    const int h = (int)(i % (unsigned)c.H), b = (int)(i / (unsigned)c.H);
    const int pos = c.pos[b], count = c.counts ? min(c.counts[b], c.L) : c.L;
    if (pos < 0 || t0 >= count) return;
    constexpr int V = 16 / sizeof(T);
    const int chunks = c.d / V, n = min(64, count - t0) * chunks;
    const T* k = static_cast<const T*>(c.k.data) + b * c.k.batch_stride + h * c.k.head_stride;
    const T* v = static_cast<const T*>(c.v.data) + b * c.v.batch_stride + h * c.v.head_stride;
    T *kp = static_cast<T*>(c.k_pages) + h * c.head_stride, *vp = static_cast<T*>(c.v_pages) + h * c.head_stride;
    const int* table = c.table + (long long)b * c.max_pages;
    for (int x0 = threadIdx.x; x0 < n; x0 += 4 * 256) {
        uint4 kv[4], vv[4];
        long long to[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int x = x0 + s * 256;
            to[s] = -1;
            if (x < n) {
                const int t = t0 + x / chunks, e = x % chunks * V;
                kv[s] = *reinterpret_cast<const uint4*>(k + (long long)t * c.k.token_stride + e);
                vv[s] = *reinterpret_cast<const uint4*>(v + (long long)t * c.v.token_stride + e);
                const long long j = (long long)pos + t, page = j / c.page_size;
                const int id = page < c.max_pages ? table[page] : -1;
                if ((unsigned)id < (unsigned)c.pages) to[s] = id * c.page_stride + (j - page * c.page_size) * c.token_stride + e;
                else atomicOr(err, kBadPage);
            }
        }
#pragma unroll
        for (int s = 0; s < 4; ++s)
            if (to[s] >= 0) {
                *reinterpret_cast<uint4*>(kp + to[s]) = kv[s];
                *reinterpret_cast<uint4*>(vp + to[s]) = vv[s];
            }
    }
}

}  // namespace

size_t paged_decode_bytes(int B, int Hq, int Hk, int d, int page_size, int max_pages, based_dtype io) {
    return for_call(io, d, Hq / Hk, [&](auto t, auto width, auto rows) {
        using T = decltype(t);
        constexpr int W = decltype(width)::value, R = decltype(rows)::value;
        return (size_t)grid_of<T, W, R>(B, Hq, Hk, page_size, max_pages) * 2 * Cfg<T, W, R>::kPiece * sizeof(float);
    });
}

based_status launch_paged_decode(const PagedCall& c, void* workspace, based_dtype io, cudaStream_t stream) {
    return for_call(io, c.d, c.Hq / c.Hk, [&](auto t, auto width, auto rows) {
        return launch<decltype(t), decltype(width)::value, decltype(rows)::value>(c, workspace, stream);
    });
}

based_status launch_paged_write(const PagedWrite& c, based_dtype io, cudaStream_t stream) {
    unsigned int* err = nullptr;
    if (error_word_ptr(&err) != BASED_OK) return BASED_ERR_CUDA;
    const int tiles = (int)(((long long)c.L + 63) / 64);
    const dim3 grid((unsigned)((long long)tiles * c.B * c.H));
    const cudaError_t e = io == BASED_BF16 ? launch_ex(paged_write_kernel<__nv_bfloat16>, grid, dim3(256), 0, 1, true, stream, c, err, tiles)
                                           : launch_ex(paged_write_kernel<float>, grid, dim3(256), 0, 1, true, stream, c, err, tiles);
    note_launch();
    const based_status st = check_launch("paged_write_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}

}  // namespace based
