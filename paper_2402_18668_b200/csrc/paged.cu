// Softmax attention of one new token per sequence over a paged key-value cache.
//
//   s_j = cap tanh(scale q . k_j / cap) - slope (pos - j),   o = sum_j exp(s_j) v_j / sum_j exp(s_j),   j = max(0, pos - window + 1) .. pos
//
// Bound by HBM (131072 tokens, 16 heads of 64: 104 us, 5.2 TB/s): every key and value is read once for up to 16 (fp32 8) query heads that share it, the
// rows of a product (more are cut into blocks of so many, each of which reads it), 2 d elements a token against 4 d Hq / Hk flop.  What has to be right is the division of the work: sequences have any lengths, known to the device alone.
//   - The unit is 64 tokens of one sequence and key head; all units lie in one row (sequence, head, tokens), and every CTA takes an equal
//     share of it, whatever the lengths, from one sequence of 131072 tokens to many short ones.
//   - Each of a CTA's four warps takes 16 tokens of a unit, in a ring of its own that copies (16 bytes a lane) fill two or three units
//     ahead, with a running maximum, sum and output of its own: no barrier but at the end of a head, where the four are joined.
//     (Single warps as the workers of units of 16 tokens: 116.6 -> 118.9 us for 131072 tokens, 16 heads of 64; 53.5 -> 56.1 for 256
//     sequences of up to 100.)
//   - What a CTA has done whole it writes as output; the pieces at its share's ends go to the workspace, and a second, dependent launch
//     joins every output that was cut, its pieces in order.  Where no sequence can be long and there are heads enough, nothing is cut (uncut).
// bf16: products on the tensor cores (m16n8k16: 16 query heads a row block, weights rounded to bf16 once, 2^-9 of each at most in the mean);
// fp32: multiply-adds, a lane per token and half a row for the scores, a lane per 2 or 4 columns for the output.
#include "paged.cuh"

#include "pairs.cuh"

namespace based {

namespace {

constexpr int kSub = 16, kWarps = 4, kThreads = 128, kUnit = kSub * kWarps;  // tokens that a warp, a CTA takes at a time
// To begin with a head's tokens of a sequence and to join its warps takes about as long as 8 units do where HBM is shared by all CTAs: 256
// sequences of up to 1000 tokens (16 heads of 64, tables for 8192) took 196 us with shares of units alone, 171, 131, 121, 148 with 4, 6, 8, 12
constexpr int kBegin = 8;
constexpr unsigned kBadPage = 2u;                                        // in the error word
constexpr float kLog2e = 1.4426950408889634f;

template <int N> struct Num { static constexpr int value = N; };
// R: query heads at a time, 16 on tensor cores, else as many as share a key head (8 at most)
template <typename T, int DP, int R> struct Cfg {
    static constexpr bool kTc = sizeof(T) == 2;
    static constexpr int kRows = R;
    static constexpr int kRowBytes = DP * sizeof(T), kChunks = kRowBytes / 16;
    static constexpr int kStage = 2 * kSub * kRowBytes;                  // a warp's keys and values of a unit
    static constexpr int kStages = kStage >= 8192 ? 3 : 4;
    static constexpr int kWarp = kStages * kStage + (kTc ? 0 : kRows * DP * 4);    // a warp's ring, and its queries where they are fp32
    static constexpr int kBytes = kWarps * kWarp;
    static constexpr int kPerSm = kBytes > 113000 ? 1 : kBytes > 74000 ? 2 : 3;
    static constexpr int kPieceRow = DP + 2;                             // floats of a piece's row: the maximum, the sum, the output
    static_assert(kStages * kStage >= kRows * kPieceRow * 4, "a warp's piece goes into its ring");
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// tanh to some 4e-7 of itself: its power series up to x^9 below 1/3, (e^2x - 1) / (e^2x + 1) above (a third of tanhf's instructions; fp32 io takes
// that).  NaN takes the series, which keeps it (fminf does not)
__device__ __forceinline__ float tanh_short(float x) {
    const float z = x * x, t = ex2(fminf(fabsf(x), 15.f) * (2.f * kLog2e));
    const float series = x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
    return fabsf(x) >= 0.33f ? copysignf(__fdividef(t - 1.f, t + 1.f), x) : series;
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

// A sequence's keys: tokens lo .. pos, in units first .. first + count - 1 from the start; none where it has no token, or
// one past what its pages can hold
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
    // what it takes for one head, in units: to begin with it and to join its warps takes as long as some units
    __device__ __forceinline__ int cost() const { return count > 0 ? count + kBegin : 0; }
};
// the sum of a value over a CTA's threads; buf: a word per warp
__device__ __forceinline__ long long sum_all(long long x, long long* buf) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = x;
    __syncthreads();
    x = 0;
    for (int w = 0; w < (int)blockDim.x / 32; ++w) x += buf[w];
    return x;
}
// The sequence in which unit x of all sequences' (`heads` times over) lies, and the units ahead of that sequence: inclusive sums, one turn of
// the CTA's threads after the other.  buf: a word per warp and two more; for all threads
struct Found { int b; long long ahead; };
__device__ __forceinline__ Found find_unit(const PagedCall& c, int heads, long long x, long long* buf) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    long long before = 0;
    for (int b0 = 0; b0 < c.B && before <= x; b0 += blockDim.x) {
        const int b = b0 + (int)threadIdx.x;
        const long long n = b < c.B ? (long long)Span(c, b).cost() * heads : 0;
        long long sum = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += y;
        }
        __syncthreads();
        if (lane == 31) buf[warp] = sum;
        __syncthreads();
        sum += before;
        for (int w = 0; w < warps; ++w) {
            if (w < warp) sum += buf[w];
            before += buf[w];
        }
        if (sum - n <= x && x < sum) {
            buf[warps] = b;
            buf[warps + 1] = sum - n;
        }
    }
    __syncthreads();
    return {(int)buf[warps], buf[warps + 1]};
}
// x / y, whose quotient is an int; in 32 bits where that does
__device__ __forceinline__ int quotient(long long x, int y) { return x >> 31 == 0 ? (int)((unsigned)x / (unsigned)y) : (int)(x / y); }

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
    int piece;                                                           // floats of one
    unsigned int* err;
    int blocks;                                                          // row blocks of a key head's queries
    int shift;                                                           // page_size = 1 << shift, or -1
    bool whole;                                                          // 16 tokens from a multiple of 16 on lie in one page
    bool split;                                                          // false: a CTA per sequence and "head", and no join
};

template <typename T, int DP, int R>
__global__ void __launch_bounds__(kThreads, Cfg<T, DP, R>::kPerSm) paged_decode_kernel(const __grid_constant__ Args a) {
    using C = Cfg<T, DP, R>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long s_buf[kWarps + 2];
    const PagedCall& c = a.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint8_t* ring = smem + warp * C::kWarp;
    float* sq = reinterpret_cast<float*>(ring + C::kStages * C::kStage);
    const int group = c.Hq / c.Hk, heads = c.Hk * a.blocks;              // "heads": key heads and row blocks of their queries
    // (the join may come in once every CTA here is past the kernel ahead: what it reads before its own wait is there then)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // This CTA's units u .. end - 1, the sequence and the head that they begin in, and which of its units
    int b, hm, unit0 = 0;
    long long u = 0, end;
    if (!a.split) {
        b = blockIdx.x / heads;
        hm = blockIdx.x % heads;
        const Span sp(c, b);
        end = sp.count;
        if (end == 0) {
            const int h0 = hm / a.blocks * group + hm % a.blocks * C::kRows, n = min(C::kRows, group - hm % a.blocks * C::kRows) * c.d;
            T* out = static_cast<T*>(c.out) + ((long long)b * c.Hq + h0) * c.d;
            for (int i = tid; i < n; i += kThreads) out[i] = from_f32<T>(0.f);
            if (tid == 0 && sp.pos >= 0) atomicOr(a.err, kBadPage);
            return;
        }
    } else {
        for (int k = blockIdx.x; k < c.B; k += gridDim.x) {              // sequences without a token
            const Span sp(c, k);
            if (sp.count > 0) continue;
            T* out = static_cast<T*>(c.out) + (long long)k * c.Hq * c.d;
            for (int i = tid; i < c.Hq * c.d; i += kThreads) out[i] = from_f32<T>(0.f);
            if (tid == 0 && sp.pos >= 0) atomicOr(a.err, kBadPage);
        }
        long long all = 0;
        for (int k = tid; k < c.B; k += kThreads) all += Span(c, k).cost();
        const Shares sh(sum_all(all, s_buf) * heads, gridDim.x);
        u = sh.begin(blockIdx.x);
        end = sh.begin(blockIdx.x + 1);
        if (u >= end) return;
        const Found at = find_unit(c, heads, u, s_buf);
        b = at.b;
        const int cost = Span(c, b).cost();                              // (not 0)
        hm = quotient(u - at.ahead, cost);
        unit0 = (int)(u - at.ahead - (long long)hm * cost) - kBegin;
    }
    int later = 0;                                                       // (a share has pieces at its beginning and at its end)

    for (; u < end; ) {
        const Span sp(c, b);
        const int left = (int)min((long long)(sp.count - unit0), end - u);      // this share's part, from unit0 (below 0: its beginning) on
        const int units = left + min(unit0, 0);
        u += left;
        unit0 = max(unit0, 0);
        if (units <= 0) return;                                          // (the share ends with its beginning)
        const int hk = hm / a.blocks, row0 = (hm % a.blocks) * C::kRows, rows = min(C::kRows, group - row0);
        const int h0 = hk * group + row0;                                // the first query head
        const T* q = static_cast<const T*>(c.q) + ((long long)b * c.Hq + h0) * c.d;
        const T* knew = static_cast<const T*>(c.k) + ((long long)b * c.Hk + hk) * c.d;
        const T* vnew = static_cast<const T*>(c.v) + ((long long)b * c.Hk + hk) * c.d;
        T* kp = static_cast<T*>(c.k_pages) + hk * c.head_stride;
        T* vp = static_cast<T*>(c.v_pages) + hk * c.head_stride;
        const int* table = c.table + (long long)b * c.max_pages;

        // Lane < 16 (and its double) looks up the page of token j0 + lane of a unit a turn before it is needed: it is checked then, so that
        // nothing waits for the table
        // (units behind the last may begin past 2^31: their numbers wrap, and `here` goes by n first)
        auto tokens = [&](int n) { return (int)((unsigned)(sp.first + unit0 + n) * kUnit + warp * kSub); };
        auto page_of = [&](int j) { return a.shift >= 0 ? j >> a.shift : (int)((unsigned)j / (unsigned)c.page_size); };
        auto here = [&](int n, int j) { return n < units && j <= sp.pos && j >= sp.lo; };
        auto look = [&](int n) -> int {
            const int j = tokens(n) + (lane & 15);
            return here(n, j) ? table[page_of(j)] : 0;
        };
        constexpr int V = 16 / (int)sizeof(T), kStep = 32 / C::kChunks;  // values of a chunk, rows of a turn
        const int lrow = lane / C::kChunks, lch = lane % C::kChunks;
        const bool lin = lch * V < c.d;
        // units in0 .. in1 - 1: no token at the border of what is seen, and the new one not among them
        const int in0 = max(0, (sp.lo - tokens(0) + kUnit - 1) / kUnit), in1 = min(units, sp.pos - kSub >= tokens(0) ? (sp.pos - kSub - tokens(0)) / kUnit + 1 : 0);
        // rows of a unit whose tokens lie inside and in one page
        const long long lane_at = lrow * c.token_stride + (lin ? lch * V : 0), step = kStep * c.token_stride;
        auto load_inside = [&](int n, int id) {
            uint8_t* st = ring + n % C::kStages * C::kStage;
            const int j0 = tokens(n), page = page_of(j0);
            const bool good = (unsigned)id < (unsigned)c.pages;
            if (!good) atomicOr(a.err, kBadPage);
            const long long at = (good ? id * c.page_stride : 0) + (long long)(j0 - page * c.page_size) * c.token_stride + lane_at;
            const T *ks = kp + at, *vs = vp + at;
#pragma unroll
            for (int i = 0; i < kSub / kStep; ++i) {
                const int row = i * kStep + lrow;
                uint8_t* to = st + row * C::kRowBytes + ((lch ^ (row & 7)) << 4);
                pairs::copy_async16(to, ks, lin && good);
                pairs::copy_async16(to + kSub * C::kRowBytes, vs, lin && good);
                ks += step;
                vs += step;
            }
            pairs::copy_async_commit();
        };
        auto load = [&](int n, int id) {
            uint8_t* st = ring + n % C::kStages * C::kStage;
            const int j0 = tokens(n), j = j0 + (lane & 15);
            long long at = -1;
            if (here(n, j)) {
                if ((unsigned)id < (unsigned)c.pages) at = id * c.page_stride + (long long)(j - page_of(j) * c.page_size) * c.token_stride;
                else atomicOr(a.err, kBadPage);
            }
#pragma unroll 4
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

        int next = look(0);
        if constexpr (!C::kTc) {
            for (int i = lane; i < C::kRows * DP; i += 32) {
                const int r = i / DP, e = i % DP;
                sq[i] = r < rows && e < c.d ? to_f32(q[(long long)r * c.d + e]) : 0.f;
            }
        }
#pragma unroll 1
        for (int n = 0; n < C::kStages - 1; ++n) {
            const int id = next;
            next = look(n + 1);
            load(n, id);
        }

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
                    const int row = r + (i & 1) * 8, col = 16 * k + e + (i >> 1) * 8;
                    qf[k][i] = row < rows && col < c.d ? *reinterpret_cast<const uint32_t*>(q + (long long)row * c.d + col) : 0u;
                }
            if (c.slopes) {
                slope[0] = r < rows ? c.slopes[h0 + r] : 0.f;
                slope[1] = r + 8 < rows ? c.slopes[h0 + r + 8] : 0.f;
            }
        }
        const float inv_cap = 1.f / c.cap;
        // a score as the softmax takes it, in base 2; CHECK: whether the token is seen
        auto weigh = [&](float s, float sl, int j, bool check) -> float {
            s *= c.scale;
            if (c.cap > 0.f) s = c.cap * (C::kTc ? tanh_short(s * inv_cap) : tanhf(s * inv_cap));
            if (c.slopes) s -= sl * (float)(sp.pos - j);
            return check && (j > sp.pos || j < sp.lo) ? -INFINITY : s * kLog2e;
        };
        // unit n.  KIND 0: all its tokens are seen and the scores as they are; 1: all are seen; 2: any.  A loop for each, so that the one
        // that runs is short
        auto turn = [&](int n, auto kind) {
            constexpr int KIND = decltype(kind)::value;
            {
                const int id = next;
                next = look(n + C::kStages);
                if constexpr (KIND < 2) load_inside(n + C::kStages - 1, id);
                else load(n + C::kStages - 1, id);
            }
            pairs::copy_async_wait<C::kStages - 1>();
            __syncwarp();
            const int j0 = tokens(n);
            uint8_t* st = ring + n % C::kStages * C::kStage;
            if (KIND < 2 || (j0 <= sp.pos && sp.lo - j0 < kSub)) {        // (j0 + kSub may be 2^31)
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
                    const float sc = KIND == 0 ? c.scale * kLog2e : 1.f;
                    if constexpr (KIND > 0) {
#pragma unroll
                        for (int t = 0; t < 2; ++t)
#pragma unroll
                            for (int x = 0; x < 4; ++x)
                                if (x < 2 || rows > 8) s[t][x] = weigh(s[t][x], slope[x >> 1], j0 + 8 * t + (lane & 3) * 2 + (x & 1), KIND == 2);
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
#pragma unroll
                    for (int r = 0; r < C::kRows; ++r) {
                        s[r] += __shfl_xor_sync(0xffffffffu, s[r], 16);
                        s[r] = KIND == 0 ? s[r] * (c.scale * kLog2e) : weigh(s[r], c.slopes && r < rows ? c.slopes[h0 + r] : 0.f, j0 + tok, KIND == 2);
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
                if (KIND == 2 && row0 == 0 && j0 <= sp.pos && sp.pos - j0 < kSub) {
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
        };
        const bool plain = c.cap == 0.f && !c.slopes;
        const int last = a.whole ? in1 - (C::kStages - 1) : 0;           // (what is loaded meanwhile lies inside too)
#pragma unroll 1
        for (int n = 0; n < units; ) {
            if (n >= in0 && n < last) {
                if (plain) {
#pragma unroll 1
                    for (; n < last; ++n) turn(n, Num<0>());
                } else {
#pragma unroll 1
                    for (; n < last; ++n) turn(n, Num<1>());
                }
            } else {
                turn(n++, Num<2>());
            }
        }
        pairs::copy_async_wait<0>();
        __syncwarp();

        // the four warps' shares joined, by way of the rings: a whole output, or a piece
        const bool whole = units == sp.count;
        float* mine = reinterpret_cast<float*>(ring);
        if constexpr (C::kTc) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = (lane >> 2) + 8 * h;
                l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
                l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
                if (r >= rows) continue;
#pragma unroll
                for (int k = 0; k < DP / 8; ++k)
                    *reinterpret_cast<float2*>(mine + r * C::kPieceRow + 2 + 8 * k + (lane & 3) * 2) = make_float2(acc[k][2 * h], acc[k][2 * h + 1]);
                if ((lane & 3) == 0) *reinterpret_cast<float2*>(mine + r * C::kPieceRow) = make_float2(m[h], l[h]);
            }
        } else {
#pragma unroll
            for (int r = 0; r < C::kRows; ++r) {
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], o);
                if (r >= rows) continue;
#pragma unroll
                for (int k = 0; k < DP / 32; ++k) mine[r * C::kPieceRow + 2 + lane * (DP / 32) + k] = acc[r][k];
                if (lane == 0) *reinterpret_cast<float2*>(mine + r * C::kPieceRow) = make_float2(m[r], l[r]);
            }
        }
        __syncthreads();
        T* out = static_cast<T*>(c.out) + ((long long)b * c.Hq + h0) * c.d;
        float* to = a.pieces + (2 * (long long)blockIdx.x + later) * a.piece;
        for (int i = tid; i < rows * DP; i += kThreads) {
            const int r = i / DP, e = i % DP;
            auto of = [&](int w) { return reinterpret_cast<const float*>(smem + w * C::kWarp) + r * C::kPieceRow; };
            float top = -INFINITY, sum = 0.f, o = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, of(w)[0]);
            const float z = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = exp2f(of(w)[0] - z);
                sum = fmaf(of(w)[1], f, sum);
                o = fmaf(of(w)[2 + e], f, o);
            }
            if (whole) {
                if (e < c.d) out[r * c.d + e] = from_f32<T>(o / sum);
            } else {
                to[r * C::kPieceRow + 2 + e] = o;
                if (e == 0) *reinterpret_cast<float2*>(to + r * C::kPieceRow) = make_float2(top, sum);
            }
        }
        if (u >= end) return;
        unit0 = -kBegin;
        later = 1;
        __syncthreads();                                                 // (before the rings are filled again)
        if (++hm == heads) {                                             // on to the next sequence that has keys, 32 looked at a turn
            hm = 0;
            for (++b; ; b += 32) {
                const uint32_t some = __ballot_sync(0xffffffffu, b + lane < c.B && Span(c, b + lane).count > 0);
                if (some) {
                    b += __ffs(some) - 1;
                    break;
                }
                if (b + 32 >= c.B) return;
            }
        }
    }
}

// The outputs that were cut, from their pieces.  BY_CUT: a CTA per border of the shares, which sees to the output that is cut there first (with all its
// rows); else a CTA per sequence and query head.  Threads hold a column each and share the pieces out among kJoin / DP of them, whose
// results are joined in order.
constexpr int kJoin = 256;
template <typename T, int DP, int R, bool BY_CUT> __global__ void __launch_bounds__(kJoin) paged_join_kernel(const __grid_constant__ Args a, int ctas) {
    using C = Cfg<T, DP, R>;
    __shared__ long long s_buf[kJoin / 32 + 2];
    __shared__ float s_part[kJoin][3];
    const PagedCall& c = a.c;
    const int heads = c.Hk * a.blocks, group = c.Hq / c.Hk;
    int b = blockIdx.x / c.Hq, h = blockIdx.x % c.Hq, hm = h / group * a.blocks + h % group / C::kRows, r = h % group % C::kRows, rows = 1;
    long long all = 0, ahead = 0;
    for (int k = threadIdx.x; k < c.B; k += kJoin) {
        const int n = Span(c, k).cost();
        all += n;
        ahead += !BY_CUT && k < b ? n : 0;
    }
    const Shares sh(sum_all(all, s_buf) * heads, ctas);
    if constexpr (BY_CUT) {
        const long long x = sh.begin(blockIdx.x + 1);
        if (x >= sh.total) {
            enter_dependent();                                           // (what comes behind this launch relies on its wait)
            return;
        }
        const Found at = find_unit(c, heads, x, s_buf);
        b = at.b;
        ahead = at.ahead;
        hm = quotient(x - ahead, Span(c, b).cost());
        r = 0;
        rows = min(C::kRows, group - hm % a.blocks * C::kRows);
        h = hm / a.blocks * group + hm % a.blocks * C::kRows;
    } else {
        ahead = sum_all(ahead, s_buf) * heads;
    }
    const Span sp(c, b);
    enter_dependent();
    if (sp.count == 0) return;
    const long long first = ahead + (long long)hm * sp.cost() + kBegin;    // its first unit
    const long long i0 = sh.of(first), i1 = sh.of(first + sp.count - 1);
    if (i0 == i1 || (BY_CUT && i0 != blockIdx.x)) return;
    const bool begun = sh.begin(i0) < first - kBegin;                        // the first CTA had something else before it
    const int count = (int)(i1 - i0) + 1, part = threadIdx.x / DP, e = threadIdx.x % DP;
    constexpr int kParts = kJoin / DP;
#pragma unroll 1
    for (; rows > 0; --rows, ++r, ++h) {
        const float* from = a.pieces + 2 * i0 * a.piece + r * C::kPieceRow;
        float top = -INFINITY, sum = 0.f, o = 0.f;
        auto add = [&](float m, float l, float x) {
            const float to = fmaxf(top, m), z = to == -INFINITY ? 0.f : to, f = exp2f(top - z), g = exp2f(m - z);
            sum = fmaf(sum, f, l * g);
            o = fmaf(o, f, x * g);
            top = to;
        };
        for (int i = part; i < count; i += 8 * kParts) {                 // eight pieces' values asked for at once
            float x[8][3];
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const int k = i + s * kParts;
                const float* p = from + (2 * (long long)k + (k == 0 && begun)) * a.piece;
                x[s][0] = k < count ? p[0] : -INFINITY;
                x[s][1] = k < count ? p[1] : 0.f;
                x[s][2] = k < count ? p[2 + e] : 0.f;
            }
#pragma unroll
            for (int s = 0; s < 8; ++s) add(x[s][0], x[s][1], x[s][2]);
        }
        s_part[threadIdx.x][0] = top;
        s_part[threadIdx.x][1] = sum;
        s_part[threadIdx.x][2] = o;
        __syncthreads();
        if (part == 0 && e < c.d) {
#pragma unroll
            for (int k = 1; k < kParts; ++k) add(s_part[k * DP + e][0], s_part[k * DP + e][1], s_part[k * DP + e][2]);
            static_cast<T*>(c.out)[((long long)b * c.Hq + h) * c.d + e] = from_f32<T>(o / sum);
        }
        __syncthreads();
    }
}

template <int DP, int R> int piece_floats(int Hq, int Hk) { return (Hq / Hk < R ? Hq / Hk : R) * (DP + 2); }
template <int R> int row_blocks(int Hq, int Hk) { return (Hq / Hk + R - 1) / R; }
// CTAs of a launch: what the device holds at a time, or one per unit where there cannot be as many
template <typename T, int DP, int R> int grid_of(int B, int Hq, int Hk, int page_size, int max_pages) {
    const long long units = (long long)B * Hk * row_blocks<R>(Hq, Hk) * (((long long)max_pages * page_size + kUnit - 1) / kUnit);
    const int most = kSMs * Cfg<T, DP, R>::kPerSm;
    return units < most ? (int)units : most;
}

// Whether no output is cut: where the tables hold up to 256 tokens (250 tokens, 16 heads: 7.7 us for 13.2 cut), or up to 1024 and there are
// outputs (of a key head) for a quarter of the SMs (256 sequences of up to 1000 tokens: 110 us for 167; but 1000 tokens, 32 outputs: 18.2 for
// 15.1)
bool uncut(long long outputs, int page_size, int max_pages) {
    const long long most = (long long)page_size * max_pages;
    return most <= 256 || (most <= 1024 && 4 * outputs >= kSMs);
}

// More outputs than this: a join per cut (1024 sequences of up to 300 tokens, 16 query heads: 57 us for 120); fewer: one per output, whose
// query heads then need not wait for one another (20000 tokens, 32 query heads on 8: 27 us for 32)
constexpr int kManyOutputs = 1024;

template <typename T, int DP, int R> based_status launch(const PagedCall& c, void* workspace, cudaStream_t stream) {
    using C = Cfg<T, DP, R>;
    static std::atomic<bool> ready[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return BASED_ERR_CUDA;
    if (!ready[dev].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(paged_decode_kernel<T, DP, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kBytes) != cudaSuccess) return BASED_ERR_CUDA;
        ready[dev].store(true, std::memory_order_release);
    }
    Args a{c, static_cast<float*>(workspace), piece_floats<DP, R>(c.Hq, c.Hk), nullptr, row_blocks<R>(c.Hq, c.Hk), -1, c.page_size % kSub == 0, true};
    const int outputs = c.B * c.Hk * a.blocks;
    a.split = !uncut(outputs, c.page_size, c.max_pages);
    if (error_word_ptr(&a.err) != BASED_OK) return BASED_ERR_CUDA;
    for (int s = 0; s < 31; ++s)
        if (c.page_size == 1 << s) a.shift = s;
    const int G = a.split ? grid_of<T, DP, R>(c.B, c.Hq, c.Hk, c.page_size, c.max_pages) : outputs;
    cudaError_t e = launch_ex(paged_decode_kernel<T, DP, R>, dim3(G), dim3(kThreads), C::kBytes, 1, true, stream, a);
    note_launch();
    based_status st = check_launch("paged_decode_kernel");
    if (e != cudaSuccess || st != BASED_OK || !a.split) return e != cudaSuccess ? BASED_ERR_CUDA : st;
    if (G == 1) return BASED_OK;
    const bool by_cut = (long long)c.B * c.Hq > kManyOutputs;
    e = by_cut ? launch_ex(paged_join_kernel<T, DP, R, true>, dim3(G - 1), dim3(kJoin), 0, 1, true, stream, a, G)
               : launch_ex(paged_join_kernel<T, DP, R, false>, dim3(c.B * c.Hq), dim3(kJoin), 0, 1, true, stream, a, G);
    note_launch();
    st = check_launch("paged_join_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}
// f with the kernel's type, width and rows for a call: f(T{}, width, rows) as types
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
        if (uncut((long long)B * Hk * row_blocks<R>(Hq, Hk), page_size, max_pages)) return (size_t)0;
        return (size_t)grid_of<T, W, R>(B, Hq, Hk, page_size, max_pages) * 2 * piece_floats<W, R>(Hq, Hk) * sizeof(float);
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
