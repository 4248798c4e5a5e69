// Decay attention, bf16 io, on tensor cores (tcgen05 + TMEM + TMA): the passes of decay.cuh in blocks of 128 tokens.
//
// One CTA per pass, head, tile of E = 64 or 128 output columns and segment walks the blocks.  Per block, with x, y [128, DC], z [128, E]:
//   scores  X = x y^T          [128,128]   -> faded and masked by one thread per row, bf16, back over the scores (TMEM)
//   turn    Y = y^T            [DC,128]    by products with a 16 x 16 identity: a row per dimension, a column per token, in TMEM, where
//           one thread per row fades the columns and leaves them as bf16 parts that add up to 16 (24) bits
//   O = x S  [128, E], S rounded to bf16 in shared memory; then O <- take O by one thread per row, and O += P z
//   S += (give Y) z            [DC, E], fp32 in TMEM, after one thread per row has multiplied it by f and left it in bf16 for x S
//   out     O -> bf16 -> the place of z -> TMA store (the factor of the outputs lies in P and take)
// One bf16 part of the faded y would put a second rounding beside that of S into every output, and 2^-9 into a state that is
// returned: two parts where S is only an operand, three where the call returns a state.
//
// Why this way: HBM's share of an SM is some 23 bytes a cycle, 5500 cycles for the 128 KB of a block at DC = E = 128, so what counts is
// that loads are always under way.  x, y and z have rings of their own whose places are free as soon as the products have read
// them (y after the first third of a block), the output leaves through z's place, and nothing else of a block lies in shared memory but S.
// With give z written to shared memory in two parts (the first form of this kernel) there was room for two stages that a
// block held to its end: 224 us for B8 H16 L4096 128/128, which takes 97 now (5.5 TB/s; with documents 108, with a state returned 169, in twice
// as many tiles; in loops of seconds, under the power limit, up to 117); B8 H32 L4096 64/64 114 and 134.  There, with blocks of 64 KB, the chain of
// a block's steps bounds it: some 3300 cycles, 4000 with documents.
//
// Warps: 0-3 scores, 4-7 feed (fades Y), 8-11 state, 12-15 results, then one each for loads, products and stores.  The groups' work
// is counted in instructions and ways to tensor memory and back, 32 columns a time: with the state in registers, loads ahead of
// stores, or unrolled loops that the instruction caches do not hold, a block took up to twice as long.
#include <cuda_bf16.h>

#include "decay.cuh"
#include "pairs.cuh"
#include "sm100.cuh"

namespace based {

using namespace sm100;

namespace {

constexpr int kT = kDecayBlockTc, kThreads = 640;
constexpr int kWarpTma = 16, kWarpMma = 17, kWarpStore = 18;
constexpr uint32_t kPanel = kT * 128;                                // 128 tokens x 64 columns, bf16: 16 KB

template <int DC, int E, bool STATES> struct Cfg {
    static constexpr int kX = DC / 64, kZ = E / 64;                  // panels
    static constexpr int kStages = DC == 64 ? (E == 64 ? 4 : 3) : 2;
    static constexpr uint32_t offY = STATES ? 0 : kStages * kX * kPanel;
    static constexpr uint32_t offZ = offY + kStages * kX * kPanel;
    static constexpr uint32_t kSPanel = DC * 128;
    static constexpr uint32_t offS = offZ + kStages * kZ * kPanel;
    static constexpr uint32_t offUnit = offS + (STATES ? 0 : kZ * kSPanel);
    static constexpr uint32_t offBars = offUnit + 512;
    static constexpr uint32_t offPow = offBars + 352;                // a^0 .. a^128
    static constexpr uint32_t offGive = offPow + 528;
    static constexpr uint32_t offPlaces = offGive + 512;
    static constexpr uint32_t kBytes = offPlaces + kStages * kT * 4;
    static_assert(kBytes <= 232448, "shared memory budget");
};
// TMEM columns: scores, then P; the turned y; O; S; E = 64: a second turned y, or the third part of a faded one
constexpr uint32_t colX = 0, colY = 128, colO = 256;
// Where there is room, two turned y in turn (`two`); where only states are wanted, two third parts too
template <int E> __device__ __forceinline__ uint32_t col_y(bool two, int i) { return two && (i & 1) ? (E == 128 ? colO : 384u) : colY; }
// With three parts a block's own share of the state is summed apart and added by the state's group: the products' sums are cut off, not
// rounded (24 of them a block, 8 that count in a sum begun with the small parts: a state over 12000 tokens without decay 5e-7 off, over 1e-6
// with all of them in one sum)
template <bool STATES> constexpr uint32_t colD = STATES ? colO : 448;
template <bool STATES> __device__ __forceinline__ uint32_t col_third(int i) { return STATES ? colX + 64u * (i & 1) : 384u; }

// Rings: full and empty places of x, y, z, and the output in z's place.  One phase a block (bTurn, bFeed: of two in turn where there are two
// turned y): bTurn, bFeed y turned, faded; bX, bP scores there, P written; bClean padding out of y, z; bDS the state behind the
// block there; bS the state ahead of it in shared memory, and faded by the block in TMEM; bXS, bTake x S there, faded; bO, bOread all of O there, read.
enum Bar { bFullX = 0, bFullY = 4, bFullZ = 8, bEmptyX = 12, bEmptyY = 16, bEmptyZ = 20, bOut = 24, bTurn = 28, bFeed = 30, bX = 32, bP, bClean, bDS, bS, bXS, bTake, bO, bOread, bCount };
static_assert(bCount * 8 + 8 <= 352, "barrier area");

struct Words { uint32_t end, own; };
struct alignas(64) Maps { CUtensorMap m[3][4]; };                    // [pass] x, y, z, out
struct Args {
    DecayCall c;
    const uint32_t* places;
    float *states, *factors;
    unsigned int* err;
    int blocks, segments, tiles;
};

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ pairs::pair as_pair(uint32_t lo, uint32_t hi) { return pairs::make(__uint_as_float(lo), __uint_as_float(hi)); }
// A row of y^T (one dimension's 128 tokens) in TMEM, every token faded: near[k] a^steps inside 16 tokens and a power more for each 16, or
// `give` where the block is not a whole plain one; left as PARTS bf16 parts, 8 columns each behind one another (a third one at tx): all but the
// last cut off, that one rounded.  32 tokens a turn: what takes time is the way to tensor memory and back, not the arithmetic (loads
// ahead of the stores before them are no help: 680 cycles per 16 tokens for 370).
template <int PARTS, bool WHOLE>
__device__ __forceinline__ void feed_row(uint32_t ty, uint32_t tx, const pairs::pair (&near)[8], float rate2, bool back, const float* give) {
#pragma unroll 1
    for (int c = 0; c < 128; c += 32) {
        uint32_t x[32];
        tmem_ld32(ty + c, x);
        pairs::pair f2[2] = {0, 0};
        if (WHOLE) {
            f2[0] = pairs::both(exp2f(-rate2 * (float)(back ? c + 1 : 112 - c)));
            f2[1] = pairs::both(exp2f(-rate2 * (float)(back ? c + 17 : 96 - c)));
        }
        tmem_wait_ld();
        uint32_t out[32];                                            // (hi, lo) of 16 tokens, (hi, lo) of the next
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            pairs::pair q;
            if constexpr (WHOLE) q = pairs::mul2(f2[k >> 3], near[k & 7]);
            else q = *reinterpret_cast<const pairs::pair*>(give + c + 2 * k);
            const float2 v = pairs::split(pairs::mul2(pairs::make(__uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1])), q));
            const uint32_t a = __float_as_uint(v.x), b = __float_as_uint(v.y);
            const int at = (k >> 3) * 16 + (k & 7);
            out[at] = __byte_perm(a, b, 0x7632);
            const float y0 = v.x - __uint_as_float(a & 0xffff0000u), y1 = v.y - __uint_as_float(b & 0xffff0000u);
            if constexpr (PARTS == 2) {
                out[at + 8] = pack2(y0, y1);
            } else {
                const uint32_t l0 = __float_as_uint(y0), l1 = __float_as_uint(y1);
                out[at + 8] = __byte_perm(l0, l1, 0x7632);
                x[k] = pack2(y0 - __uint_as_float(l0 & 0xffff0000u), y1 - __uint_as_float(l1 & 0xffff0000u));
            }
        }
        tmem_st32(ty + c, out);
        if constexpr (PARTS == 3) {
            uint32_t third[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) third[k] = x[k];
            tmem_st16(tx + c / 2, third);
        }
    }
    tmem_wait_st();
}
// A row of scores in TMEM, faded and masked, over itself in bf16; row r = 32 w + lane.  KIND 0: one document, no padding; 1: several, no padding
// between their tokens (the row's own word tells where its document lies); 2: any (the words pl of all tokens, the powers pw).
// near[k]: a^steps from column k of 16 to the end that is nearer to rows outside; among[k]: factor a^steps to a row among the 16 (0: it does not see it).
// 32 columns a turn; a kind has a loop of its own, so that the one that runs stays in the instruction caches.
template <int KIND>
__device__ __forceinline__ void score_row(uint32_t tx, int w, int lane, bool back, float rate2, float factor, const pairs::pair (&near)[8],
                                          const pairs::pair (&among)[8], uint32_t own, const uint32_t* pl, const float* pw) {
    const int r = 32 * w + lane;
#pragma unroll 1
    for (int c = 0; c < 4; ++c) {
        uint32_t pk[16];
        if (back ? c < w : c > w) {
#pragma unroll
            for (int k = 0; k < 16; ++k) pk[k] = 0u;
        } else {
            uint32_t v[32];
            tmem_ld32(tx + 32 * c, v);
            if constexpr (KIND < 2) {
                const int steps = back ? 32 * c - r : r - 32 * c - 15;             // to the nearer end of the first 16 columns
                pairs::pair f0 = pairs::both(factor * exp2f(-rate2 * (float)steps)), f1 = pairs::both(factor * exp2f(-rate2 * (float)(back ? steps + 16 : steps - 16)));
                tmem_wait_ld();
                if (c != w) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const float2 y = pairs::split(pairs::mul2(as_pair(v[2 * k], v[2 * k + 1]), pairs::mul2(k < 8 ? f0 : f1, near[k & 7])));
                        pk[k] = pack2(y.x, y.y);
                    }
                } else {                                             // of either 16 the row is one, or it sees them all, or none
                    const bool high = lane >= 16;
                    if (back ? high : !high) f0 = f1 = 0;
                    if (back) f0 = 0;
                    else f1 = 0;
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const pairs::pair t = pairs::mul2(k < 8 ? f0 : f1, near[k & 7]);
                        const float2 y = pairs::split(pairs::mul2(as_pair(v[2 * k], v[2 * k + 1]), high == (k >= 8) ? among[k & 7] : t));
                        pk[k] = pack2(y.x, y.y);
                    }
                }
                if constexpr (KIND == 1) {                           // the row's document alone: columns lo .. hi of these 32, two a register
                    const int lo = own & kPadding ? 32 : (back ? 0 : max(place_from(own) - 32 * c, 0)), hi = back ? min(place_to(own) - 32 * c, 31) : 31;
                    const uint32_t m = lo > hi ? 0u : (0xffffffffu >> (31 - hi)) & (0xffffffffu << lo);
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        if (!((m >> (2 * k)) & 1u)) pk[k] &= 0xffff0000u;
                        if (!((m >> (2 * k + 1)) & 1u)) pk[k] &= 0x0000ffffu;
                    }
                }
            } else {
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 32; ++k) {
                    const uint32_t q = pl[32 * c + k];
                    const int steps = back ? place_count(q) - place_count(own) : place_count(own) - place_count(q);
                    const bool seen = ((q ^ own) & 0xff00u) == 0 && !((q | own) & kPadding) && (c != w || (back ? k >= lane : k <= lane));
                    const float f = pw[max(steps, 0)] * factor;
                    v[k] = seen ? __float_as_uint(__uint_as_float(v[k]) * f) : 0u;
                }
#pragma unroll
                for (int k = 0; k < 16; ++k) pk[k] = pack2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1]));
            }
        }
        tmem_st16(tx + 16 * c, pk);                                  // (over columns that this row has read, or does not need)
    }
    tmem_wait_st();
}
// mbar_wait in few instructions: every one that a block's way leads through has to fit into the instruction caches with all the others (88 KB
// of code, of which a block runs some 30; B8 H32 L4096 64/64 with documents took 220 us with the timed wait at each place, 195 with this).
// Parked for up to 20 us a turn, given up after kTurns of them.
constexpr int kTurns = 1 << 20;
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, volatile uint32_t* abort_flag) {
#pragma unroll 1
    for (int n = 0; !mbar_try_wait_hint(bar, parity, 20000u); ++n) {
        if (n == kTurns) *abort_flag = 1;
        if (*abort_flag) return false;
    }
    return true;
}
// Two at once: asked for side by side, since one answer takes some 150 cycles (in the products' warp: B2 H16 L32768 64/64 187 -> 178 us)
__device__ __forceinline__ bool wait_for_both(uint64_t* x, uint32_t px, uint64_t* y, uint32_t py, volatile uint32_t* abort_flag) {
    uint32_t there;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 q, [%3], %4;\n\t"
        "and.pred p, p, q;\n\t"
        "selp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(there)
        : "r"(smem_u32(x)), "r"(px), "r"(smem_u32(y)), "r"(py)
        : "memory");
    return there || (wait_for(x, px, abort_flag) && wait_for(y, py, abort_flag));
}
// barrier of a group of 128 threads that also tells whether all of them say yes
__device__ __forceinline__ bool group_all(int id, bool pred) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %1, 0;\n\t"
        "bar.red.and.pred q, %2, 128, p;\n\t"
        "selp.b32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)pred), "r"(id)
        : "memory");
    return r != 0;
}

}  // namespace

// PARTS: of the faded y.  (A kernel for each number, though tiles of 128 columns have two only: with code for both, which the instruction caches
// hold beside what runs, B8 H32 L4096 64/64 with documents took 148 us for 137, B2 H16 L32768 218 for 195)
template <int DC, int E, bool STATES, bool DOCS, int PARTS>
__global__ void __launch_bounds__(kThreads, 1) decay_tc_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Args a) {
    using C = Cfg<DC, E, STATES>;
    constexpr int NS = C::kStages;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::offBars);
    uint32_t* tmem_base_s = reinterpret_cast<uint32_t*>(bars + bCount);
    volatile uint32_t* abort_flag = tmem_base_s + 1;
    float* pw = reinterpret_cast<float*>(smem + C::offPow);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    DecayItem it(blockIdx.x, a.c.passes, a.tiles, STATES ? a.segments - 1 : a.segments);
    it.pass = __reduce_min_sync(0xffffffffu, it.pass);               // (uniform, as below)
    const DecayPass& p = a.c.pass[it.pass];
    const int e0 = it.tile * E, L = a.c.L;
    if (e0 >= p.de) return;
    if (smem_u32(smem) & 1023u) {                                    // (the tiles' swizzle goes by their addresses)
        if (tid == 0) atomicOr(a.err, 1u);
        return;
    }
    const int b = (int)(it.head / a.c.H), h = (int)(it.head % a.c.H);
    const bool back = p.back;
    constexpr bool two = STATES || (E == 64 && PARTS == 2);

    if (tid == 0) {
        for (int s = 0; s < bCount; ++s) {
            const bool group = s == bP || s == bClean || (s >= bFeed && s < bFeed + 2) || s == bS || s == bTake || s == bOread || (s >= bOut && s < bOut + 4);
            mbar_init(&bars[s], group ? 128 : 1);
        }
        *abort_flag = 0;
        fence_mbar_init();
        for (int i = 0; i < 4; ++i) prefetch_tensormap(&maps.m[it.pass][i]);
    }
    if (tid < 32) {                                                  // the identity, [16][16] as a K-major operand, rows of 32 bytes swizzled
        const int r = tid >> 1, half = tid & 1;
        uint32_t v[4] = {0, 0, 0, 0};
        if (r >> 3 == half) v[(r & 7) >> 1] = r & 1 ? 0x3f800000u : 0x3f80u;
        *reinterpret_cast<uint4*>(smem + C::offUnit + r * 32 + ((half ^ (r >> 2 & 1)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
    }
    fence_proxy_async_smem();
    if (warp == kWarpMma) { tmem_alloc(tmem_base_s, 512); tmem_relinquish(); }
    enter_dependent();
    const float rate2 = rate_of(a.c.rate[h]);
    if (tid <= kT) pw[tid] = faded(rate2, tid);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tb = *tmem_base_s;
    bool ok = true;

    const int g = back ? a.segments - 1 - it.segment : it.segment;
    int first = decay_first(a.blocks, a.segments, g), count = decay_first(a.blocks, a.segments, g + 1) - first;
    auto places_of = [&](int n) { return a.places + ((long long)b * a.blocks + n) * kT; };
    // the last token's place in block n: how many count, how many documents begin
    auto end_of = [&](int n) -> uint32_t { return DOCS ? places_of(n)[kT - 1] : (uint32_t)min(kT, L - n * kT); };
    // one document reaches over the whole block, and nothing in it is padding: as without documents
    auto plain = [&](uint32_t end, int n) { return !DOCS || (end & 0xffffu) == (uint32_t)min(kT, L - n * kT); };
    bool cut = false;
    if (STATES) {
        // Of a segment's own state only the blocks are worth reading behind which nothing fades to 0: those from the last one on in which a
        // document begins, or from which on the powers of a do not underflow
        int from = 0;
        if (DOCS) {
            for (int i = count; i > 0 && from == 0; i -= 32) {       // (every warp for itself)
                const int j = i - 1 - lane;
                const uint32_t m = __ballot_sync(0xffffffffu, j > 0 && place_run(end_of(back ? first + count - 1 - j : first + j)) != 0);
                if (m) from = i - 1 - (__ffs(m) - 1);
            }
        } else {
            const float keep = 150.f / (rate2 * kT);                 // (inf or NaN for a rate of 0: all)
            if (keep >= 0.f && keep < (float)(count - 2)) from = count - 2 - (int)keep;
        }
        cut = from > 0;
        if (!back) first += from;
        count -= from;
    }
    // Blocks of padding alone at either end: nothing but zeros to write
    int lead_in = 0, lead_out = 0;                                   // so many from `first` on, so many behind
    if (DOCS) {
        for (int i = 0; i < count; i += 32) {
            const uint32_t m = __ballot_sync(0xffffffffu, i + lane < count && place_count(end_of(first + i + lane)) != 0);
            if (m) {
                lead_in = i + __ffs(m) - 1;
                break;
            }
            lead_in = count;
        }
        for (int i = count; i > lead_in; i -= 32) {
            const uint32_t m = __ballot_sync(0xffffffffu, i - 1 - lane >= lead_in && place_count(end_of(first + i - 1 - lane)) != 0);
            if (m) {
                lead_out = count - (i - (__ffs(m) - 1));
                break;
            }
        }
        first += lead_in;
        count -= lead_in + lead_out;
        if (!STATES && lead_in + lead_out > 0 && warp >= 12 && warp < 16) {
            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(const_cast<void*>(p.out.data)) + b * p.out.batch_stride + h * p.out.head_stride + e0;
            const int chunks = min(E, p.de - e0) / 8;
            for (int part = 0; part < 2; ++part) {
                const int t0 = (part ? first + count : first - lead_in) * kT, t1 = min(t0 + (part ? lead_out : lead_in) * kT, L);
                for (long long k = tid & 127; k < (long long)(t1 - t0) * chunks; k += 128)
                    *reinterpret_cast<uint4*>(out + (t0 + k / chunks) * p.out.token_stride + k % chunks * 8) = make_uint4(0, 0, 0, 0);
            }
        }
    }
    // (the same in every lane, and known to be: the products' addresses stay in uniform registers.  B8 H32 L4096 64/64 with documents
    // took 185 us without, 159 with)
    first = __reduce_min_sync(0xffffffffu, first);
    count = __reduce_min_sync(0xffffffffu, count);
    auto block_of = [&](int i) { return back ? first + count - 1 - i : first + i; };
    auto wait = [&](int bar, int phase) -> bool { return __all_sync(0xffffffffu, wait_for(&bars[bar], phase & 1, abort_flag)); };
    auto wait2 = [&](int x, int px, int y, int py) -> bool {
        return __all_sync(0xffffffffu, wait_for_both(&bars[x], px & 1, &bars[y], py & 1, abort_flag));
    };
    // what block i leaves of the state ahead of it, from its last token's place
    auto fade_of = [&](uint32_t end) -> float { return place_run(end) == 0 ? pw[place_count(end)] : 0.f; };
    // N columns from e on of row c of the state: to shared memory in bf16, and to TMEM faded by the next block (0: dropped, whatever it holds)
    auto pass_on = [&](int c, int e, auto& x, float f) {
        constexpr int N = sizeof(x) / 4;
        if (!STATES) {
            uint8_t* row = smem + C::offS + (e >> 6) * C::kSPanel + c * 128;
            const uint32_t sw = c & 7;
#pragma unroll
            for (int j = 0; j < N / 8; ++j) {
                uint32_t v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = pack2(__uint_as_float(x[8 * j + 2 * k]), __uint_as_float(x[8 * j + 2 * k + 1]));
                *reinterpret_cast<uint4*>(row + (((uint32_t)((e & 63) / 8 + j) ^ sw) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
            }
        }
        if (f == 0.f) {
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = 0u;
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) * f);
        }
        const uint32_t at = tmem_addr(tb, (uint32_t)(c & ~31), colO + E + e);
        if constexpr (N == 32) tmem_st32(at, x);
        else tmem_st16(at, x);
    };
    // A block's last place and a token's own, asked for a block ahead of their use
    auto words_of = [&](int i, int r) -> Words {
        if (i >= count) return {0u, 0u};
        const int n = block_of(i);
        return {end_of(n), DOCS ? places_of(n)[r] : 0u};
    };
    // The state ahead of the first block, by all four groups, a quarter of its columns each: what was given, and the segments before
    // this one
    if (warp < 16 && (warp & 3) * 32 < DC) {
        constexpr int N = E / 4;
        const int c = 32 * (warp & 3) + lane, e = (warp >> 2) * N;
        uint32_t x[N];
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = 0u;
        if (!STATES) {
            if (p.state_in && c < p.dc) {
                const float* in = p.state_in + it.head * p.dc * p.de;
#pragma unroll
                for (int k = 0; k < N; k += 4)
                    if (e0 + e + k < p.de) {                         // (widths are multiples of 8)
                        float4 y;
                        if (p.turned) {
                            const float* col = in + (long long)(e0 + e + k) * p.dc + c;
                            y = make_float4(col[0], col[p.dc], col[2 * p.dc], col[3 * p.dc]);
                        } else {
                            y = *reinterpret_cast<const float4*>(in + (long long)c * p.de + e0 + e + k);
                        }
                        x[k] = __float_as_uint(p.in_factor * y.x);
                        x[k + 1] = __float_as_uint(p.in_factor * y.y);
                        x[k + 2] = __float_as_uint(p.in_factor * y.z);
                        x[k + 3] = __float_as_uint(p.in_factor * y.w);
                    }
            }
#pragma unroll 2
            for (int q = 0; q < it.segment; ++q) {
                const long long slot = decay_slot(it.pass, a.c.passes, it.head, a.tiles, it.tile, a.segments, q);
                const float g = a.factors[slot];
                const float4* from = reinterpret_cast<const float4*>(a.states + (slot * kDecayMaxWidth + c) * E + e);
#pragma unroll
                for (int k = 0; k < N; k += 4) {
                    const float4 y = from[k / 4];
                    const float ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[k + j] = __float_as_uint(g == 0.f ? ys[j] : fmaf(g, __uint_as_float(x[k + j]), ys[j]));
                }
            }
        }
        pass_on(c, e, x, count > 0 && PARTS == 2 ? fade_of(end_of(block_of(0))) : 1.f);
        tmem_wait_st();
        fence_proxy_async_smem();
    }
    tc_fence_before();
    if (warp != kWarpTma && warp < kWarpStore) asm volatile("bar.sync 2, 544;" ::: "memory");      // (the loads are under way meanwhile)
    tc_fence_after();

    if (warp == kWarpTma) {
        if (lane == 0) {
            for (int i = 0; i < count; ++i) {
                const int s = i % NS, n = block_of(i), t0 = n * kT, turn = i / NS - 1;
                if (i >= NS) ok = wait_for(&bars[bEmptyY + s], turn & 1, abort_flag);
                if (!ok) break;
                mbar_arrive_expect_tx(&bars[bFullY + s], C::kX * kPanel);
#pragma unroll
                for (int j = 0; j < C::kX; ++j)
                    tma_load_4d(smem + C::offY + (s * C::kX + j) * kPanel, &maps.m[it.pass][1], &bars[bFullY + s], 64 * j, t0, h, b);
                if (!STATES) {
                    if (i >= NS) ok = wait_for(&bars[bEmptyX + s], turn & 1, abort_flag);
                    if (!ok) break;
                    mbar_arrive_expect_tx(&bars[bFullX + s], C::kX * kPanel);
#pragma unroll
                    for (int j = 0; j < C::kX; ++j)
                        tma_load_4d(smem + (s * C::kX + j) * kPanel, &maps.m[it.pass][0], &bars[bFullX + s], 64 * j, t0, h, b);
                }
                if (i >= NS) ok = wait_for(&bars[bEmptyZ + s], turn & 1, abort_flag);
                if (!ok) break;
                mbar_arrive_expect_tx(&bars[bFullZ + s], C::kZ * kPanel + (DOCS ? kT * 4 : 0));
                if (DOCS) bulk_load_1d(smem + C::offPlaces + s * kT * 4, places_of(n), kT * 4, &bars[bFullZ + s]);
#pragma unroll
                for (int j = 0; j < C::kZ; ++j)
                    tma_load_4d(smem + C::offZ + (s * C::kZ + j) * kPanel, &maps.m[it.pass][2], &bars[bFullZ + s], e0 + 64 * j, t0, h, b);
            }
        }
    } else if (warp == kWarpStore) {
        if (!STATES && lane == 0) {
            for (int i = 0; i < count; ++i) {
                const int s = i % NS;
                ok = wait_for(&bars[bOut + s], (i / NS) & 1, abort_flag);
                if (!ok) break;
#pragma unroll
                for (int j = 0; j < C::kZ; ++j)
                    if (e0 + 64 * j < p.de)
                        tma_store_4d(&maps.m[it.pass][3], smem + C::offZ + (s * C::kZ + j) * kPanel, e0 + 64 * j, block_of(i) * kT, h, b);
                tma_store_commit();
                tma_store_wait_read<0>();
                mbar_arrive(&bars[bEmptyZ + s]);
            }
            tma_store_wait<0>();
        }
    } else if (warp == kWarpMma) {
        // the whole warp runs this block and one elected lane issues (see mma_ss_w)
        const uint32_t lead = elect_one();
        constexpr uint64_t dK = make_smem_desc_base(16, 1024, kSwizzle128B);             // K-major rows, or one MN-major block of 64
        constexpr uint64_t dZ = make_smem_desc_base(kPanel, 1024, kSwizzle128B);         // MN-major, blocks of 64 a panel apart
        constexpr uint64_t dS = make_smem_desc_base(C::kSPanel, 1024, kSwizzle128B);
        constexpr uint64_t dU = make_smem_desc_base(16, 256, kSwizzle32B);               // K-major [16][16]
        constexpr uint32_t iX = make_idesc_bf16(128, 128, 0, 0), iT = make_idesc_bf16(128, 16, 1, 0), iO = make_idesc_bf16(128, E, 0, 1);
        constexpr uint32_t colS = colO + E;
        const uint32_t sm = smem_u32(smem);
        auto lo = [](uint64_t base, uint32_t addr) { return desc_lo(base) + (addr >> 4); };
        // (rolled where the documents' code crowds the caches: B8 H16 L4096 128/128 119 -> 108 us there; B8 H32 64/64 without 124 -> 130)
        auto x_of = [&](int i) { return lo(dK, sm + (i % NS) * C::kX * kPanel); };
        auto y_of = [&](int i) { return sm + C::offY + (i % NS) * C::kX * kPanel; };
        auto z_of = [&](int i) { return lo(dZ, sm + C::offZ + (i % NS) * C::kZ * kPanel); };
        // y^T; products have 128 rows: those past the dimensions of a narrow y hold what lies behind it, and nobody reads them
        auto turn = [&](int i) -> bool {
            if (!(DOCS ? wait2(bFullY + i % NS, i / NS, bClean, i) : wait(bFullY + i % NS, i / NS))) return false;
            tc_fence_after();
            const uint32_t lt = lo(dZ, y_of(i)), lu = lo(dU, sm + C::offUnit), d = tb + col_y<E>(two, i);
#pragma unroll (DOCS ? 2 : 8)
            for (int k = 0; k < kT / 16; ++k) mma_ss_w<false>(lead, d + 16 * k, lt + k * 128, desc_hi(dZ), lu, desc_hi(dU), iT);
            mma_commit_w(lead, &bars[bTurn + (two ? i & 1 : 0)]);
            if (STATES) mma_commit_w(lead, &bars[bEmptyY + i % NS]);
            return true;
        };
        auto delta = [&](int i) -> bool {
            // (x S has waited for the state ahead)
            if (!wait2(bFullZ + i % NS, i / NS, bFeed + (two ? i & 1 : 0), two ? i >> 1 : i) || (STATES && i > 0 && !wait(bS, i - 1))) return false;
            tc_fence_after();
            const uint32_t lz = z_of(i), ty = tb + col_y<E>(two, i);
            if constexpr (PARTS == 3) {                              // the small parts first, into a sum of their own (see colD)
                const uint32_t t3 = tb + col_third<STATES>(i), d = tb + colD<STATES>;
#pragma unroll 2
                for (int k = 0; k < kT / 16; ++k) {
                    if (k == 0) mma_ts_w<false>(lead, d, t3, lz, desc_hi(dZ), iO);
                    else mma_ts_w<true>(lead, d, t3 + 8 * k, lz + k * 128, desc_hi(dZ), iO);
                }
#pragma unroll 2
                for (int k = 0; k < kT / 16; ++k) mma_ts_w<true>(lead, d, ty + 16 * k + 8, lz + k * 128, desc_hi(dZ), iO);
#pragma unroll 2
                for (int k = 0; k < kT / 16; ++k) mma_ts_w<true>(lead, d, ty + 16 * k, lz + k * 128, desc_hi(dZ), iO);
            } else {
#pragma unroll (DOCS ? 2 : 8)
                for (int k = 0; k < kT / 16; ++k) {
                    const uint32_t at = ty + 16 * k;
                    mma_ts_w<true>(lead, tb + colS, at, lz + k * 128, desc_hi(dZ), iO);
                    mma_ts_w<true>(lead, tb + colS, at + 8, lz + k * 128, desc_hi(dZ), iO);
                }
            }
            mma_commit_w(lead, &bars[bDS]);
            if (STATES) mma_commit_w(lead, &bars[bEmptyZ + i % NS]);
            return true;
        };
        auto scores = [&](int i) -> bool {
            if (!wait(bFullX + i % NS, i / NS)) return false;
            tc_fence_after();
            const uint32_t lx = x_of(i), ly = lo(dK, y_of(i));
#pragma unroll
            for (int k = 0; k < DC / 16; ++k) {
                const uint32_t at = (k >> 2) * (kPanel >> 4) + (k & 3) * 2;
                if (k == 0) mma_ss_w<false>(lead, tb + colX, lx, desc_hi(dK), ly, desc_hi(dK), iX);
                else mma_ss_w<true>(lead, tb + colX, lx + at, desc_hi(dK), ly + at, desc_hi(dK), iX);
            }
            mma_commit_w(lead, &bars[bX]);
            mma_commit_w(lead, &bars[bEmptyY + i % NS]);
            return true;
        };
        auto before = [&](int i) -> bool {
            if (i > 0 && !wait2(bS, i - 1, bOread, i - 1)) return false;
            tc_fence_after();
            const uint32_t lx = x_of(i), ls = lo(dS, sm + C::offS);
#pragma unroll
            for (int k = 0; k < DC / 16; ++k) {
                const uint32_t at = (k >> 2) * (kPanel >> 4) + (k & 3) * 2;
                if (k == 0) mma_ss_w<false>(lead, tb + colO, lx, desc_hi(dK), ls, desc_hi(dS), iO);
                else mma_ss_w<true>(lead, tb + colO, lx + at, desc_hi(dK), ls + k * 128, desc_hi(dS), iO);
            }
            mma_commit_w(lead, &bars[bXS]);
            mma_commit_w(lead, &bars[bEmptyX + i % NS]);
            return true;
        };
        auto inside = [&](int i) -> bool {
            if (!wait2(bP, i, bTake, i)) return false;
            tc_fence_after();
            const uint32_t lz = z_of(i);
#pragma unroll (DOCS ? 2 : 8)
            for (int k = 0; k < kT / 16; ++k) mma_ts_w<true>(lead, tb + colO, tb + colX + k * 8, lz + k * 128, desc_hi(dZ), iO);
            mma_commit_w(lead, &bars[bO]);
            return true;
        };
        // Products of one accumulator and shape run in the order of their issue; of others PTX promises no order.  So one that overwrites what
        // another reads waits for that one's end: the scores for P z (bO), the turned y for the product that reads the one ahead (bDS; of
        // two in turn the one before, whose end lies behind the wait for S: but where only states are wanted there is none).  B2 H16
        // L32768 64/64: 171 -> 175 us, with documents 184 -> 189, its backward pass 493 -> 518; B8 H16 L4096 128/128 with a state returned 165 -> 169,
        // without 97 either way.
        if (count == 0) {
        } else if constexpr (STATES) {
            ok = turn(0);
#pragma unroll 1
            for (int i = 0; i < count && ok; ++i) ok = (i == 0 || wait(bDS, i - 1)) && (i + 1 == count || turn(i + 1)) && delta(i);
        } else {
            ok = turn(0) && scores(0) && before(0);
#pragma unroll 1
            for (int i = 0; i < count && ok; ++i) {
                const bool more = i + 1 < count;
                if (two) ok = (!more || turn(i + 1)) && delta(i) && inside(i);
                else ok = delta(i) && (!more || (wait(bDS, i) && turn(i + 1))) && inside(i);
                if (more && ok) ok = wait(bO, i) && scores(i + 1) && before(i + 1);
            }
        }
    } else if (warp < 4) {
        // ---- scores: thread = row of the block, TMEM lane
        if constexpr (!STATES) {
            const int w = warp, r = tid;
            const uint32_t tl = tmem_addr(tb, (uint32_t)w * 32u, 0);
            const float factor = a.c.factor;
            // a^steps from column k of 16 to the end that is nearer to rows outside, and factor a^steps to a row among the 16 (0: the row does
            // not see it), in registers: a load from shared memory takes long while the products read it all the time
            pairs::pair near[8], among[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int l = lane & 15, j = 2 * k, s0 = back ? j - l : l - j, s1 = back ? j + 1 - l : l - j - 1;
                near[k] = pairs::make(faded(rate2, back ? j : 15 - j), faded(rate2, back ? j + 1 : 14 - j));
                among[k] = pairs::make(s0 >= 0 ? factor * faded(rate2, s0) : 0.f, s1 >= 0 ? factor * faded(rate2, s1) : 0.f);
            }
            Words next = words_of(0, r);
            for (int i = 0; i < count; ++i) {
                const int n = block_of(i), s = i % NS;
                const uint32_t end = next.end, own = next.own;
                next = words_of(i + 1, r);
                const bool simple = plain(end, n);
                const uint32_t* pl = reinterpret_cast<const uint32_t*>(smem + C::offPlaces + s * kT * 4);
                ok = wait(bX, i) && (simple || (end & kCompact) || wait(bFullZ + s, i / NS));      // (the places come with z)
                if (!ok) break;
                tc_fence_after();
                if (!DOCS || simple) score_row<0>(tl + colX, w, lane, back, rate2, factor, near, among, own, pl, pw);
                else if (end & kCompact) score_row<1>(tl + colX, w, lane, back, rate2, factor, near, among, own, pl, pw);
                else score_row<2>(tl + colX, w, lane, back, rate2, factor, near, among, own, pl, pw);
                tc_fence_before();
                mbar_arrive(&bars[bP]);
            }
        }
    } else if (warp >= 8 && warp < 12) {
        // ---- state: thread = row of the state, TMEM lane
        const int w = warp & 3, c = 32 * w + lane;
        const bool rows = w * 32 < DC;                               // (the whole warp's)
        const uint32_t ts = tmem_addr(tb, (uint32_t)w * 32u, colO + E);
        float whole = cut ? 0.f : 1.f, f = count > 0 ? fade_of(end_of(block_of(0))) : 1.f;
        for (int i = 0; i < count; ++i) {
            whole *= f;
            const float here = f;
            if (i + 1 < count) f = fade_of(end_of(block_of(i + 1)));
            ok = wait(bDS, i);
            if (!ok) break;
            tc_fence_after();
            if constexpr (PARTS == 3) {
                if (rows) {
#pragma unroll 1
                    for (int e = 0; e < E; e += 16) {
                        uint32_t x[16], y[16];
                        tmem_ld16(ts + e, x);
                        tmem_ld16(ts - (colO + E) + colD<STATES> + e, y);
                        tmem_wait_ld();
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            x[k] = here == 0.f ? y[k] : __float_as_uint(fmaf(here, __uint_as_float(x[k]), __uint_as_float(y[k])));
                        pass_on(c, e, x, 1.f);
                    }
                    tmem_wait_st();
                    fence_proxy_async_smem();
                }
                tc_fence_before();
                if (i + 1 < count) mbar_arrive(&bars[bS]);
                continue;
            }
            if (i + 1 < count) {                                     // (what commits this product waits for x S as well: the state ahead has been read)
                if (rows) {
#pragma unroll 1
                    for (int e = 0; e < E; e += 32) {
                        uint32_t x[32];
                        tmem_ld32(ts + e, x);
                        tmem_wait_ld();
                        pass_on(c, e, x, f);
                    }
                    tmem_wait_st();
                    fence_proxy_async_smem();
                }
                tc_fence_before();
                mbar_arrive(&bars[bS]);
            }
        }
        if ((STATES || PARTS == 3) && ok && rows && (STATES || (p.state_out && it.segment == a.segments - 1))) {
            const long long slot = STATES ? decay_slot(it.pass, a.c.passes, it.head, a.tiles, it.tile, a.segments, it.segment) : 0;
#pragma unroll 1
            for (int e = 0; e < E; e += 32) {
                uint32_t x[32];
                tmem_ld32(ts + e, x);
                tmem_wait_ld();
                if (STATES) {
                    uint4* to = reinterpret_cast<uint4*>(a.states + (slot * kDecayMaxWidth + c) * E + e);
#pragma unroll
                    for (int k = 0; k < 8; ++k) to[k] = make_uint4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
                } else if (c < p.dc) {
                    float* out = p.state_out + it.head * p.dc * p.de;
#pragma unroll
                    for (int k = 0; k < 32; k += 4)
                        if (e0 + e + k < p.de) {
                            float4 y = make_float4(__uint_as_float(x[k]), __uint_as_float(x[k + 1]), __uint_as_float(x[k + 2]), __uint_as_float(x[k + 3]));
                            y = make_float4(p.out_factor * y.x, p.out_factor * y.y, p.out_factor * y.z, p.out_factor * y.w);
                            if (p.turned) {
                                float* col = out + (long long)(e0 + e + k) * p.dc + c;
                                col[0] = y.x; col[p.dc] = y.y; col[2 * p.dc] = y.z; col[3 * p.dc] = y.w;
                            } else {
                                *reinterpret_cast<float4*>(out + (long long)c * p.de + e0 + e + k) = y;
                            }
                        }
                }
            }
            if (STATES && c == 0) a.factors[slot] = whole;
        }
    } else if (warp >= 12 && warp < 16) {
        // ---- results: thread = row of the block, TMEM lane
        if constexpr (!STATES) {
            const int w = warp & 3, r = 32 * w + lane;
            const uint32_t to = tmem_addr(tb, (uint32_t)w * 32u, colO), sw = r & 7;
            Words next = words_of(0, r);
            for (int i = 0; i < count; ++i) {
                const int n = block_of(i), s = i % NS;
                const uint32_t end = next.end, own = next.own;
                next = words_of(i + 1, r);
                float take;
                if (plain(end, n)) {
                    take = pw[back ? max(place_count(end) - 1 - r, 0) : r + 1];
                } else {
                    take = own & kPadding ? 0.f
                           : back         ? (place_run(own) == place_run(end) ? pw[place_count(end) - place_count(own)] : 0.f)
                                          : (place_run(own) == 0 ? pw[place_count(own)] : 0.f);
                }
                const bool all = __all_sync(0xffffffffu, take != 0.f);
                take *= a.c.factor;
                ok = wait(bXS, i);
                if (!ok) break;
                tc_fence_after();
#pragma unroll 1
                for (int e = 0; e < E; e += 32) {
                    uint32_t x[32];
                    tmem_ld32(to + e, x);
                    tmem_wait_ld();
                    if (all) {
#pragma unroll
                        for (int k = 0; k < 32; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) * take);
                    } else {                                         // (no product with a weight of 0: there the state's share need not be finite)
#pragma unroll
                        for (int k = 0; k < 32; ++k) x[k] = take == 0.f ? 0u : __float_as_uint(__uint_as_float(x[k]) * take);
                    }
                    tmem_st32(to + e, x);
                }
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(&bars[bTake]);
                ok = wait(bO, i);
                if (!ok) break;
                tc_fence_after();
                uint8_t* row = smem + C::offZ + s * C::kZ * kPanel + r * 128;
                // all of it out of tensor memory first: the next block's products wait for that
                uint32_t v[E / 2];
#pragma unroll
                for (int e = 0; e < E; e += 16) {
                    uint32_t x[16];
                    tmem_ld16(to + e, x);
                    tmem_wait_ld();
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[e / 2 + k] = pack2(__uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1]));
                }
                tc_fence_before();
                mbar_arrive(&bars[bOread]);
#pragma unroll
                for (int j = 0; j < E / 8; ++j)
                    *reinterpret_cast<uint4*>(row + (j >> 3) * kPanel + (((uint32_t)(j & 7) ^ sw) << 4)) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                fence_proxy_async_smem();
                mbar_arrive(&bars[bOut + s]);
            }
        }
    } else if (warp >= 4 && warp < 8) {
        // ---- feed: thread = dimension of y, TMEM lane; its tokens faded, in bf16 parts over themselves
        const int w = warp & 3, u = tid & 127;
        const bool rows = w * 32 < DC;                               // (the whole warp's)
        const uint32_t tl = tmem_addr(tb, (uint32_t)w * 32u, 0);
        float* give = reinterpret_cast<float*>(smem + C::offGive);
        // rows of padding out of y and z
        auto clean = [&](int i, uint32_t end) -> bool {
            const int n = block_of(i), s = i % NS;
            if (place_count(end) < min(kT, L - n * kT)) {
                if (!wait(bFullY + s, i / NS) || !wait(bFullZ + s, i / NS)) return false;
                const uint32_t* pl = reinterpret_cast<const uint32_t*>(smem + C::offPlaces + s * kT * 4);
                const uint4 zero = make_uint4(0, 0, 0, 0);
                for (int j = 0; j < 8; ++j) {
                    const int row = (u >> 3) + 16 * j;
                    if (!(pl[row] & kPadding)) continue;
                    const uint32_t to = row * 128 + (u & 7) * 16;
#pragma unroll
                    for (int k = 0; k < C::kX; ++k) *reinterpret_cast<uint4*>(smem + C::offY + (s * C::kX + k) * kPanel + to) = zero;
#pragma unroll
                    for (int k = 0; k < C::kZ; ++k) *reinterpret_cast<uint4*>(smem + C::offZ + (s * C::kZ + k) * kPanel + to) = zero;
                }
                fence_proxy_async_smem();
            }
            mbar_arrive(&bars[bClean]);
            return true;
        };
        Words next = words_of(0, u);
        pairs::pair near[8];                                         // a^steps from token k of 16 to the end that is nearer to where the state goes
#pragma unroll
        for (int k = 0; k < 8; ++k) near[k] = pairs::make(faded(rate2, back ? 2 * k : 15 - 2 * k), faded(rate2, back ? 2 * k + 1 : 14 - 2 * k));
        Words here{0u, 0u};
        for (int i = DOCS ? -1 : 0; i < count; ++i) {
            if (i >= 0) {
                here = next;
                next = words_of(i + 1, u);
                ok = group_all(1, ok && wait_for(&bars[bTurn + (two ? i & 1 : 0)], (two ? i >> 1 : i) & 1, abort_flag));
                if (!ok) break;
            }
            // (the next block's, once the products are past the wait for this one's)
            if (DOCS && i + 1 < count) {
                ok = group_all(1, clean(i + 1, next.end));
                if (!ok) break;
            }
            if (DOCS && i < 0) continue;
            const uint32_t end = here.end, own = here.own;
            const int c1 = place_count(end);
            const bool simple = plain(end, block_of(i)), whole = simple && c1 == kT;
            if (!whole) {
                float x;
                if (simple) {
                    x = u < c1 ? pw[back ? u + 1 : c1 - 1 - u] : 0.f;
                } else {
                    x = own & kPadding ? 0.f
                        : back         ? (place_run(own) == 0 ? pw[place_count(own)] : 0.f)
                                       : (place_run(own) == place_run(end) ? pw[c1 - place_count(own)] : 0.f);
                }
                give[u] = x;
                group_all(1, true);
            }
            tc_fence_after();
            if (rows) {
                const uint32_t ty = tl + col_y<E>(two, i), tx = tl + col_third<STATES>(i);
                if (whole) feed_row<PARTS, true>(ty, tx, near, rate2, back, give);
                else feed_row<PARTS, false>(ty, tx, near, rate2, back, give);
            }
            tc_fence_before();
            mbar_arrive(&bars[bFeed + (two ? i & 1 : 0)]);
        }
    }

    if (!ok && lane == 0) atomicOr(a.err, 1u);
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        for (int i = 0; i < 200; ++i) __nanosleep(1000);
    }
    __syncthreads();
    if (warp == kWarpMma) tmem_dealloc(tb, 512);
}

namespace {

template <int DC, int E, bool STATES, bool DOCS, int PARTS> based_status launch(const Maps& maps, const Args& a, long long ctas, cudaStream_t stream) {
    using C = Cfg<DC, E, STATES>;
    auto kern = decay_tc_kernel<DC, E, STATES, DOCS, PARTS>;
    static std::atomic<bool> ready[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return BASED_ERR_CUDA;
    if (!ready[dev].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kBytes) != cudaSuccess) return BASED_ERR_CUDA;
        ready[dev].store(true, std::memory_order_release);
    }
    const cudaError_t e = launch_ex(kern, dim3((unsigned)ctas), dim3(kThreads), C::kBytes, 1, true, stream, maps, a);
    note_launch();
    const based_status st = check_launch("decay_tc_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}
template <int DC, int E, bool DOCS, int PARTS> based_status launch_both(const Maps& maps, const Args& a, const DecayPlan& plan, cudaStream_t stream) {
    if (plan.segments > 1) {
        const based_status st = launch<DC, E, true, DOCS, PARTS>(maps, a, plan.ctas / plan.segments * (plan.segments - 1), stream);
        if (st != BASED_OK) return st;
    }
    return launch<DC, E, false, DOCS, PARTS>(maps, a, plan.ctas, stream);
}
template <int DC, int E, int PARTS> based_status launch_docs(const Maps& maps, const Args& a, const DecayPlan& plan, cudaStream_t stream) {
    return a.places ? launch_both<DC, E, true, PARTS>(maps, a, plan, stream) : launch_both<DC, E, false, PARTS>(maps, a, plan, stream);
}

}  // namespace

static bool state_wanted(const DecayCall& c) {
    for (int i = 0; i < c.passes; ++i)
        if (c.pass[i].state_out) return true;
    return false;
}
DecayPlan decay_plan_tc(const DecayCall& c) {
    int de = 0;
    for (int i = 0; i < c.passes; ++i) de = c.pass[i].de > de ? c.pass[i].de : de;
    const DecayPlan narrow = decay_plan(c.passes, de, c.B, c.H, c.L, c.documents != nullptr, kT, 64, kSMs, {1.0, 0.7, 2.5, 0.15});
    // (three parts of the faded y have no place beside tiles of 128)
    if (de <= 64 || state_wanted(c)) return narrow;
    // tiles of 128 columns read x and y once: worth it unless there are so few heads that half as many CTAs leave SMs idle
    const DecayPlan wide = decay_plan(c.passes, de, c.B, c.H, c.L, c.documents != nullptr, kT, 128, kSMs, {1.5, 0.7, 2.5, 0.15});
    return wide.time <= narrow.time ? wide : narrow;
}

based_status launch_decay_tc(const DecayCall& c, const DecayPlan& plan, void* workspace, cudaStream_t stream) {
    char* ws = static_cast<char*>(workspace);
    uint32_t* places = c.documents ? reinterpret_cast<uint32_t*>(ws) : nullptr;
    Maps maps;
    bool wide = false;
    for (int i = 0; i < c.passes; ++i) {
        const DecayPass& p = c.pass[i];
        if (!make_heads_map_bf16(&maps.m[i][0], p.x, c.B, c.H, c.L, p.dc, kT) || !make_heads_map_bf16(&maps.m[i][1], p.y, c.B, c.H, c.L, p.dc, kT) ||
            !make_heads_map_bf16(&maps.m[i][2], p.z, c.B, c.H, c.L, p.de, kT) || !make_heads_map_bf16(&maps.m[i][3], p.out, c.B, c.H, c.L, p.de, kT))
            return BASED_ERR_CUDA;
        wide = wide || p.dc > 64;
    }
    Args a{c, places, reinterpret_cast<float*>(ws + plan.places_bytes), reinterpret_cast<float*>(ws + plan.places_bytes + plan.states_bytes),
           nullptr, plan.blocks, plan.segments, plan.tiles};
    if (error_word_ptr(&a.err) != BASED_OK) return BASED_ERR_CUDA;
    if (places) {
        const based_status st = launch_decay_places(c.documents, places, c.B, c.L, kT, stream);
        if (st != BASED_OK) return st;
    }
    if (state_wanted(c)) return wide ? launch_docs<128, 64, 3>(maps, a, plan, stream) : launch_docs<64, 64, 3>(maps, a, plan, stream);
    if (plan.width == 64) return wide ? launch_docs<128, 64, 2>(maps, a, plan, stream) : launch_docs<64, 64, 2>(maps, a, plan, stream);
    return wide ? launch_docs<128, 128, 2>(maps, a, plan, stream) : launch_docs<64, 128, 2>(maps, a, plan, stream);
}

}  // namespace based
