// Decay attention, bf16 io, on tensor cores (tcgen05 + TMEM + TMA): the passes of decay.cuh in blocks of 128 tokens.
//
// One CTA per pass, head, tile of E = 64 or 128 output columns and segment walks the blocks.  Per block, with x, y [128, DC], z [128, E]:
//   scores  X = x y^T          [128,128]   -> faded and masked by one thread per row, bf16, back over the scores (TMEM)
//   turn    Y = y^T            [DC,128]    by products with a 16 x 16 identity: a row per dimension, a column per token, in TMEM, where
//           one thread per row fades the columns and leaves them as bf16 parts that add up to 16 (24) bits
//   O = x S  [128, E], S rounded to bf16 in shared memory; then O <- take O by one thread per row, and O += P z
//   dS = (give Y) z            [DC, E], fp32; the state S <- f S + dS is held in registers, a row per thread, so that no
//           block's products wait for the block before it
//   out     factor O -> bf16 -> the place of z -> TMA store
// One bf16 part of the faded y would put a second rounding beside that of S into every output, and 2^-9 into a state that is
// returned: two parts where S is only an operand, three where the call returns a state.
//
// Why this way: HBM's share of an SM is some 23 bytes a cycle, 5500 cycles for the 128 KB of a block at DC = E = 128, so what counts is
// that loads are always under way.  x, y and z have rings of their own whose places are free as soon as the products have read
// them (y after the first third of a block), the output leaves through z's place, and nothing else of a block lies in shared memory but S.
// With give z written to shared memory in two parts (the first form of this kernel) there was room for two stages that a
// block held to its end: 224 us for B8 H16 L4096 128/128.
//
// Warps: 0-3 scores (E = 128: and results), 4-7 feed (fades Y), 8-11 state, 12-15 results (E = 128: the state's columns 64 ..), 16 loads,
// 17 products, 18 stores.
#include <cuda_bf16.h>

#include "decay.cuh"
#include "sm100.cuh"

namespace based {

using namespace sm100;

namespace {

constexpr int kT = kDecayBlockTc, kThreads = 608;
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
    static constexpr uint32_t offPow = offBars + 320;                // a^0 .. a^128
    static constexpr uint32_t offGive = offPow + 528;
    static constexpr uint32_t offNear = offGive + 512;               // a^(steps to the near end of 32 columns)
    static constexpr uint32_t offPlaces = offNear + 128;
    static constexpr uint32_t kBytes = offPlaces + kStages * kT * 4;
    static_assert(kBytes <= 232448, "shared memory budget");
};
// TMEM columns: scores (P, and the third part of the faded y behind it), the turned y, O, dS
constexpr uint32_t colX = 0, colY = 128, colO = 256;

// Rings: full and empty places of x, y, z.  One phase a block: bX, bP scores there, P written; bClean padding out of y, z; bTurn, bFeed y
// turned, faded; bDS, bDSread; bS the state ahead of the block in shared memory; bXS, bTake x S there, faded; bO, bOread all of O
// there, read; bOut the output in z's place.
enum Bar { bFullX = 0, bFullY = 4, bFullZ = 8, bEmptyX = 12, bEmptyY = 16, bEmptyZ = 20, bX = 24, bP, bClean, bTurn, bFeed, bDS, bDSread, bS, bXS, bTake, bO, bOread, bOut, bCount };
static_assert(bCount * 8 + 8 <= 320, "barrier area");

struct alignas(64) Maps { CUtensorMap m[3][4]; };                    // [pass] x, y, z, out
struct Args {
    DecayCall c;
    const uint32_t* places;
    float *states, *factors;
    unsigned int* err;
    int blocks, segments, tiles;
    int parts;                                                       // of the faded y: 2 or 3
};

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ float lo_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f32(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
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

template <int DC, int E, bool STATES, bool DOCS>
__global__ void __launch_bounds__(kThreads, 1) decay_tc_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Args a) {
    using C = Cfg<DC, E, STATES>;
    constexpr int NS = C::kStages;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::offBars);
    uint32_t* tmem_base_s = reinterpret_cast<uint32_t*>(bars + bCount);
    volatile uint32_t* abort_flag = tmem_base_s + 1;
    float* pw = reinterpret_cast<float*>(smem + C::offPow);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const DecayItem it(blockIdx.x, a.c.passes, a.tiles, STATES ? a.segments - 1 : a.segments);
    const DecayPass& p = a.c.pass[it.pass];
    const int e0 = it.tile * E, L = a.c.L;
    if (e0 >= p.de) return;
    if (smem_u32(smem) & 1023u) {                                    // (the tiles' swizzle goes by their addresses)
        if (tid == 0) atomicOr(a.err, 1u);
        return;
    }
    const int b = (int)(it.head / a.c.H), h = (int)(it.head % a.c.H);
    const bool back = p.back;

    if (tid == 0) {
        for (int s = 0; s < bCount; ++s) {
            const bool groups = s == bDSread || s == bS;             // as many groups as the state has
            const bool group = s == bP || s == bClean || s == bFeed || s == bTake || s == bOread || s == bOut;
            mbar_init(&bars[s], groups ? 128 * C::kZ : group ? 128 : 1);
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
    const float rate2 = a.c.rate[h] * kLog2e;
    if (tid <= kT) pw[tid] = faded(rate2, tid);
    if (tid < 32) reinterpret_cast<float*>(smem + C::offNear)[tid] = faded(rate2, back ? tid : 31 - tid);
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
    auto block_of = [&](int i) { return back ? first + count - 1 - i : first + i; };
    auto wait = [&](int bar, int phase) -> bool { return __all_sync(0xffffffffu, mbar_wait(&bars[bar], phase & 1, abort_flag)); };

    if (warp == kWarpTma) {
        if (lane == 0) {
            for (int i = 0; i < count; ++i) {
                const int s = i % NS, n = block_of(i), t0 = n * kT, turn = i / NS - 1;
                if (i >= NS) ok = mbar_wait(&bars[bEmptyY + s], turn & 1, abort_flag);
                if (!ok) break;
                mbar_arrive_expect_tx(&bars[bFullY + s], C::kX * kPanel);
#pragma unroll
                for (int j = 0; j < C::kX; ++j)
                    tma_load_4d(smem + C::offY + (s * C::kX + j) * kPanel, &maps.m[it.pass][1], &bars[bFullY + s], 64 * j, t0, h, b);
                if (!STATES) {
                    if (i >= NS) ok = mbar_wait(&bars[bEmptyX + s], turn & 1, abort_flag);
                    if (!ok) break;
                    mbar_arrive_expect_tx(&bars[bFullX + s], C::kX * kPanel);
#pragma unroll
                    for (int j = 0; j < C::kX; ++j)
                        tma_load_4d(smem + (s * C::kX + j) * kPanel, &maps.m[it.pass][0], &bars[bFullX + s], 64 * j, t0, h, b);
                }
                if (i >= NS) ok = mbar_wait(&bars[bEmptyZ + s], turn & 1, abort_flag);
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
                ok = mbar_wait(&bars[bOut], i & 1, abort_flag);
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
        constexpr uint32_t colDS = colO + E;
        const uint32_t sm = smem_u32(smem);
        auto lo = [](uint64_t base, uint32_t addr) { return desc_lo(base) + (addr >> 4); };
#pragma unroll 1
        for (int i = 0; i < count && ok; ++i) {
            const int s = i % NS, turn = i / NS;
            const uint32_t y = sm + C::offY + s * C::kX * kPanel;
            const uint32_t lx = lo(dK, sm + s * C::kX * kPanel), ly = lo(dK, y), lz = lo(dZ, sm + C::offZ + s * C::kZ * kPanel);
            ok = wait(bFullY + s, turn) && (STATES || wait(bFullX + s, turn));
            if (!ok) break;
            tc_fence_after();
            if (!STATES) {
#pragma unroll
                for (int k = 0; k < DC / 16; ++k) {
                    const uint32_t at = (k >> 2) * (kPanel >> 4) + (k & 3) * 2;
                    if (k == 0) mma_ss_w<false>(lead, tb + colX, lx, desc_hi(dK), ly, desc_hi(dK), iX);
                    else mma_ss_w<true>(lead, tb + colX, lx + at, desc_hi(dK), ly + at, desc_hi(dK), iX);
                }
                mma_commit_w(lead, &bars[bX]);
            }
            if (DOCS) {
                ok = wait(bClean, i);
                if (!ok) break;
                tc_fence_after();
            }
            {   // (products have 128 rows: those past the dimensions of a narrow y hold what lies behind it, and nobody reads them)
                const uint32_t lt = lo(dZ, y);
                const uint32_t lu = lo(dU, sm + C::offUnit);
#pragma unroll
                for (int k = 0; k < kT / 16; ++k) mma_ss_w<false>(lead, tb + colY + 16 * k, lt + k * 128, desc_hi(dZ), lu, desc_hi(dU), iT);
                mma_commit_w(lead, &bars[bTurn]);
                mma_commit_w(lead, &bars[bEmptyY + s]);
            }
            if (!STATES) {
                ok = wait(bS, i) && (i == 0 || wait(bOread, i - 1));
                if (!ok) break;
                tc_fence_after();
                const uint32_t ls = lo(dS, sm + C::offS);
#pragma unroll
                for (int k = 0; k < DC / 16; ++k) {
                    const uint32_t at = (k >> 2) * (kPanel >> 4) + (k & 3) * 2;
                    if (k == 0) mma_ss_w<false>(lead, tb + colO, lx, desc_hi(dK), ls, desc_hi(dS), iO);
                    else mma_ss_w<true>(lead, tb + colO, lx + at, desc_hi(dK), ls + k * 128, desc_hi(dS), iO);
                }
                mma_commit_w(lead, &bars[bXS]);
                mma_commit_w(lead, &bars[bEmptyX + s]);
            }
            ok = wait(bFullZ + s, turn) && wait(bFeed, i) && (i == 0 || wait(bDSread, i - 1));
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < kT / 16; ++k) {
                const uint32_t at = colY + 32 * (k >> 1) + 8 * (k & 1);
                if (k == 0) mma_ts_w<false>(lead, tb + colDS, tb + at, lz, desc_hi(dZ), iO);
                else mma_ts_w<true>(lead, tb + colDS, tb + at, lz + k * 128, desc_hi(dZ), iO);
                mma_ts_w<true>(lead, tb + colDS, tb + at + 16, lz + k * 128, desc_hi(dZ), iO);
            }
            if (a.parts == 3) {
#pragma unroll
                for (int k = 0; k < kT / 16; ++k) mma_ts_w<true>(lead, tb + colDS, tb + colX + 64 + 8 * k, lz + k * 128, desc_hi(dZ), iO);
            }
            mma_commit_w(lead, &bars[bDS]);
            if (STATES) {
                mma_commit_w(lead, &bars[bEmptyZ + s]);
            } else {
                ok = wait(bP, i) && wait(bTake, i);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < kT / 16; ++k) mma_ts_w<true>(lead, tb + colO, tb + colX + k * 8, lz + k * 128, desc_hi(dZ), iO);
                mma_commit_w(lead, &bars[bO]);
            }
        }
    } else if (warp < 4 || (E == 64 && warp >= 12 && warp < 16)) {
        // ---- scores and results: thread = row of the block, TMEM lane; two groups where there is one to spare
        if constexpr (!STATES) {
            const bool do_scores = warp < 4, do_results = E == 128 || warp >= 12;
            const int w = warp & 3, r = 32 * w + lane;
            const uint32_t tl = tmem_addr(tb, (uint32_t)w * 32u, 0);
            const float* near = reinterpret_cast<const float*>(smem + C::offNear);
            const uint32_t sw = r & 7;
            const float factor = a.c.factor;
            for (int i = 0; i < count; ++i) {
                const int n = block_of(i), s = i % NS;
                const uint32_t end = end_of(n);
                const bool simple = plain(end, n);
                const uint32_t own = DOCS && !simple ? places_of(n)[r] : 0u;
                if (do_scores) {
                    const uint32_t* pl = reinterpret_cast<const uint32_t*>(smem + C::offPlaces + s * kT * 4);
                    ok = wait(bX, i) && (simple || wait(bFullZ + s, i / NS));      // (the places come with z)
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < 4; ++c) {                    // 32 columns a time
                        uint32_t pk[16];
                        if (back ? c < w : c > w) {
#pragma unroll
                            for (int k = 0; k < 16; ++k) pk[k] = 0u;
                        } else {
                            uint32_t x[32];
                            tmem_ld32(tl + colX + 32 * c, x);
                            tmem_wait_ld();
                            if (simple) {
                                if (c == w) {
#pragma unroll
                                    for (int k = 0; k < 32; ++k) {
                                        const int steps = back ? k - lane : lane - k;
                                        x[k] = steps >= 0 ? __float_as_uint(__uint_as_float(x[k]) * pw[steps]) : 0u;
                                    }
                                } else {                             // steps from the row to the nearer end of the columns, and on from there
                                    const float f = pw[back ? 32 * c - r : r - 32 * c - 31];
#pragma unroll
                                    for (int k = 0; k < 32; k += 4) {
                                        const float4 q = *reinterpret_cast<const float4*>(near + k);
                                        x[k] = __float_as_uint(__uint_as_float(x[k]) * f * q.x);
                                        x[k + 1] = __float_as_uint(__uint_as_float(x[k + 1]) * f * q.y);
                                        x[k + 2] = __float_as_uint(__uint_as_float(x[k + 2]) * f * q.z);
                                        x[k + 3] = __float_as_uint(__uint_as_float(x[k + 3]) * f * q.w);
                                    }
                                }
                            } else {
#pragma unroll
                                for (int k = 0; k < 32; ++k) {
                                    const uint32_t q = pl[32 * c + k];
                                    const int steps = back ? place_count(q) - place_count(own) : place_count(own) - place_count(q);
                                    const bool seen = ((q ^ own) & (kPadding | 0xff00u)) == 0 && !(own & kPadding) && (c != w || (back ? k >= lane : k <= lane));
                                    x[k] = seen ? __float_as_uint(__uint_as_float(x[k]) * pw[max(steps, 0)]) : 0u;
                                }
                            }
#pragma unroll
                            for (int k = 0; k < 16; ++k) pk[k] = pack2(__uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1]));
                        }
                        tmem_st16(tl + colX + 16 * c, pk);           // (over columns that this row has read, or does not need)
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(&bars[bP]);
                }
                if (do_results) {
                    float take;
                    if (simple) take = back ? pw[max(place_count(end) - 1 - r, 0)] : pw[r + 1];
                    else
                        take = own & kPadding ? 0.f
                               : back         ? (place_run(own) == place_run(end) ? pw[place_count(end) - place_count(own)] : 0.f)
                                              : (place_run(own) == 0 ? pw[place_count(own)] : 0.f);
                    ok = wait(bXS, i);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < E; c += 32) {
                        uint32_t x[32];
                        tmem_ld32(tl + colO + c, x);
                        tmem_wait_ld();
                        // (no product with a weight of 0: there the state's share need not be finite)
#pragma unroll
                        for (int k = 0; k < 32; ++k) x[k] = take == 0.f ? 0u : __float_as_uint(__uint_as_float(x[k]) * take);
                        tmem_st32(tl + colO + c, x);
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(&bars[bTake]);
                    ok = wait(bO, i);
                    if (!ok) break;
                    tc_fence_after();
                    uint8_t* row = smem + C::offZ + s * C::kZ * kPanel + r * 128;
#pragma unroll 1
                    for (int c = 0; c < E; c += 32) {
                        uint32_t x[32];
                        tmem_ld32(tl + colO + c, x);
                        tmem_wait_ld();
                        if (c + 32 == E) {
                            tc_fence_before();
                            mbar_arrive(&bars[bOread]);
                        }
                        uint8_t* panel = row + (c >> 6) * kPanel;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            uint32_t v[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) v[k] = pack2(__uint_as_float(x[8 * j + 2 * k]) * factor, __uint_as_float(x[8 * j + 2 * k + 1]) * factor);
                            *reinterpret_cast<uint4*>(panel + (((uint32_t)((c & 32) / 8 + j) ^ sw) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
                        }
                    }
                    fence_proxy_async_smem();
                    mbar_arrive(&bars[bOut]);
                }
            }
        }
    } else if (warp >= 8 && warp < 16) {
        // ---- state: thread = row of the state, TMEM lane, 64 of its columns
        const int w = warp & 3, c = 32 * w + lane, at = warp < 12 ? 0 : 64, e1 = e0 + at;
        const bool rows = w * 32 < DC;                               // (the whole warp's)
        float s[64];
#pragma unroll
        for (int e = 0; e < 64; ++e) s[e] = 0.f;
        if (!STATES && rows) {
            if (p.state_in && c < p.dc) {
                const float* in = p.state_in + it.head * p.dc * p.de;
#pragma unroll
                for (int e = 0; e < 64; ++e)
                    if (e1 + e < p.de) s[e] = p.in_factor * in[p.turned ? (long long)(e1 + e) * p.dc + c : (long long)c * p.de + e1 + e];
            }
            for (int k = 0; k < it.segment; ++k) {
                const long long slot = decay_slot(it.pass, a.c.passes, it.head, a.tiles, it.tile, a.segments, k);
                const float f = a.factors[slot];
                const float4* from = reinterpret_cast<const float4*>(a.states + (slot * kDecayMaxWidth + c) * E + at);
#pragma unroll
                for (int e = 0; e < 64; e += 4) {
                    const float4 x = from[e / 4];
                    s[e] = fmaf(f, s[e], x.x);
                    s[e + 1] = fmaf(f, s[e + 1], x.y);
                    s[e + 2] = fmaf(f, s[e + 2], x.z);
                    s[e + 3] = fmaf(f, s[e + 3], x.w);
                }
            }
        }
        auto to_shared = [&] {
            if (rows) {
                uint8_t* row = smem + C::offS + (at >> 6) * C::kSPanel + c * 128;
                const uint32_t sw = c & 7;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    *reinterpret_cast<uint4*>(row + (((uint32_t)j ^ sw) << 4)) =
                        make_uint4(pack2(s[8 * j], s[8 * j + 1]), pack2(s[8 * j + 2], s[8 * j + 3]), pack2(s[8 * j + 4], s[8 * j + 5]),
                                   pack2(s[8 * j + 6], s[8 * j + 7]));
                fence_proxy_async_smem();
            }
            mbar_arrive(&bars[bS]);
        };
        if (!STATES) to_shared();
        float whole = cut ? 0.f : 1.f;
        for (int i = 0; i < count; ++i) {
            const uint32_t end = end_of(block_of(i));
            const float f = place_run(end) == 0 ? pw[place_count(end)] : 0.f;
            ok = wait(bDS, i);
            if (!ok) break;
            tc_fence_after();
            if (rows) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t x[16];
                    tmem_ld16(tmem_addr(tb, (uint32_t)w * 32u, colO + E + at + 16 * q), x);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[16 * q + e] = fmaf(f, s[16 * q + e], __uint_as_float(x[e]));
                }
            }
            whole *= f;
            tc_fence_before();
            mbar_arrive(&bars[bDSread]);
            if (!STATES && i + 1 < count) to_shared();               // (dS comes behind x S in order: the state before has been read)
        }
        if (ok && rows) {
            if (STATES) {
                const long long slot = decay_slot(it.pass, a.c.passes, it.head, a.tiles, it.tile, a.segments, it.segment);
                float4* to = reinterpret_cast<float4*>(a.states + (slot * kDecayMaxWidth + c) * E + at);
#pragma unroll
                for (int e = 0; e < 64; e += 4) to[e / 4] = make_float4(s[e], s[e + 1], s[e + 2], s[e + 3]);
                if (c == 0 && at == 0) a.factors[slot] = whole;
            } else if (p.state_out && it.segment == a.segments - 1 && c < p.dc) {
                float* to = p.state_out + it.head * p.dc * p.de;
#pragma unroll
                for (int e = 0; e < 64; ++e)
                    if (e1 + e < p.de) to[p.turned ? (long long)(e1 + e) * p.dc + c : (long long)c * p.de + e1 + e] = p.out_factor * s[e];
            }
        }
    } else if (warp >= 4 && warp < 8) {
        // ---- feed: thread = dimension of y, TMEM lane; its tokens faded, in bf16 parts over themselves
        const int w = warp & 3, u = tid & 127;
        const bool rows = w * 32 < DC;                               // (the whole warp's)
        const uint32_t ty = tmem_addr(tb, (uint32_t)w * 32u, colY), tx = tmem_addr(tb, (uint32_t)w * 32u, colX + 64);
        float* give = reinterpret_cast<float*>(smem + C::offGive);
        // rows of padding out of y and z
        auto clean = [&](int i) -> bool {
            const int n = block_of(i), s = i % NS;
            if (place_count(end_of(n)) < min(kT, L - n * kT)) {
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
        if (DOCS) ok = clean(0);
        int held = 0;                                                // what `give` holds: 1 a whole plain block's weights
        for (int i = 0; i < count; ++i) {
            const int n = block_of(i);
            const uint32_t end = end_of(n);
            const int c1 = place_count(end);
            const bool simple = plain(end, n), whole = simple && c1 == kT;
            // (the third part goes where scores were that P does not need)
            ok = ok && mbar_wait(&bars[bTurn], i & 1, abort_flag);
            if (!STATES && a.parts == 3) ok = ok && mbar_wait(&bars[bP], i & 1, abort_flag);
            ok = group_all(1, ok);
            if (!ok) break;
            if (!whole || !held) {
                float x;
                if (simple) {
                    x = u < c1 ? pw[back ? u + 1 : c1 - 1 - u] : 0.f;
                } else {
                    const uint32_t q = places_of(n)[u];
                    x = q & kPadding ? 0.f
                        : back       ? (place_run(q) == 0 ? pw[place_count(q)] : 0.f)
                                     : (place_run(q) == place_run(end) ? pw[c1 - place_count(q)] : 0.f);
                }
                give[u] = x;
                held = whole;
                group_all(1, true);
            }
            tc_fence_after();
            if (rows) {
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {                        // 32 tokens a time
                    uint32_t x[32], hi[16], lo[16];
                    tmem_ld32(ty + 32 * c, x);
                    tmem_wait_ld();
#pragma unroll
                    for (int k = 0; k < 32; k += 4) {
                        const float4 q = *reinterpret_cast<const float4*>(give + 32 * c + k);
                        const float x0 = __uint_as_float(x[k]) * q.x, x1 = __uint_as_float(x[k + 1]) * q.y, x2 = __uint_as_float(x[k + 2]) * q.z,
                                    x3 = __uint_as_float(x[k + 3]) * q.w;
                        hi[k / 2] = pack2(x0, x1);
                        hi[k / 2 + 1] = pack2(x2, x3);
                        const float y0 = x0 - lo_f32(hi[k / 2]), y1 = x1 - hi_f32(hi[k / 2]), y2 = x2 - lo_f32(hi[k / 2 + 1]), y3 = x3 - hi_f32(hi[k / 2 + 1]);
                        lo[k / 2] = pack2(y0, y1);
                        lo[k / 2 + 1] = pack2(y2, y3);
                        x[k / 2] = pack2(y0 - lo_f32(lo[k / 2]), y1 - hi_f32(lo[k / 2]));
                        x[k / 2 + 1] = pack2(y2 - lo_f32(lo[k / 2 + 1]), y3 - hi_f32(lo[k / 2 + 1]));
                    }
                    tmem_st16(ty + 32 * c, hi);
                    tmem_st16(ty + 32 * c + 16, lo);
                    if (a.parts == 3) {
                        uint32_t third[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) third[k] = x[k];
                        tmem_st16(tx + 16 * c, third);
                    }
                }
                tmem_wait_st();
            }
            tc_fence_before();
            mbar_arrive(&bars[bFeed]);
            if (DOCS && i + 1 < count) ok = clean(i + 1);
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

template <int DC, int E, bool STATES, bool DOCS> based_status launch(const Maps& maps, const Args& a, long long ctas, cudaStream_t stream) {
    using C = Cfg<DC, E, STATES>;
    auto kern = decay_tc_kernel<DC, E, STATES, DOCS>;
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
template <int DC, int E, bool DOCS> based_status launch_both(const Maps& maps, const Args& a, const DecayPlan& plan, cudaStream_t stream) {
    if (plan.segments > 1) {
        const based_status st = launch<DC, E, true, DOCS>(maps, a, plan.ctas / plan.segments * (plan.segments - 1), stream);
        if (st != BASED_OK) return st;
    }
    return launch<DC, E, false, DOCS>(maps, a, plan.ctas, stream);
}
template <int DC, int E> based_status launch_docs(const Maps& maps, const Args& a, const DecayPlan& plan, cudaStream_t stream) {
    return a.places ? launch_both<DC, E, true>(maps, a, plan, stream) : launch_both<DC, E, false>(maps, a, plan, stream);
}

}  // namespace

DecayPlan decay_plan_tc(const DecayCall& c) {
    int de = 0;
    for (int i = 0; i < c.passes; ++i) de = c.pass[i].de > de ? c.pass[i].de : de;
    const DecayPlan narrow = decay_plan(c.passes, de, c.B, c.H, c.L, c.documents != nullptr, kT, 64, kSMs, 1.0);
    if (de <= 64) return narrow;
    // tiles of 128 columns read x and y once: worth it unless there are so few heads that half as many CTAs leave SMs idle
    const DecayPlan wide = decay_plan(c.passes, de, c.B, c.H, c.L, c.documents != nullptr, kT, 128, kSMs, 1.5);
    return wide.time <= narrow.time ? wide : narrow;
}

based_status launch_decay_tc(const DecayCall& c, const DecayPlan& plan, void* workspace, cudaStream_t stream) {
    char* ws = static_cast<char*>(workspace);
    uint32_t* places = c.documents ? reinterpret_cast<uint32_t*>(ws) : nullptr;
    Maps maps;
    bool wide = false, wanted = false;
    for (int i = 0; i < c.passes; ++i) {
        const DecayPass& p = c.pass[i];
        if (!make_heads_map_bf16(&maps.m[i][0], p.x, c.B, c.H, c.L, p.dc, kT) || !make_heads_map_bf16(&maps.m[i][1], p.y, c.B, c.H, c.L, p.dc, kT) ||
            !make_heads_map_bf16(&maps.m[i][2], p.z, c.B, c.H, c.L, p.de, kT) || !make_heads_map_bf16(&maps.m[i][3], p.out, c.B, c.H, c.L, p.de, kT))
            return BASED_ERR_CUDA;
        wide = wide || p.dc > 64;
        wanted = wanted || p.state_out;
    }
    Args a{c, places, reinterpret_cast<float*>(ws + plan.places_bytes), reinterpret_cast<float*>(ws + plan.places_bytes + plan.states_bytes),
           nullptr, plan.blocks, plan.segments, plan.tiles, wanted ? 3 : 2};
    if (error_word_ptr(&a.err) != BASED_OK) return BASED_ERR_CUDA;
    if (places) {
        const based_status st = launch_decay_places(c.documents, places, c.B, c.L, kT, stream);
        if (st != BASED_OK) return st;
    }
    if (plan.width == 64) return wide ? launch_docs<128, 64>(maps, a, plan, stream) : launch_docs<64, 64>(maps, a, plan, stream);
    return wide ? launch_docs<128, 128>(maps, a, plan, stream) : launch_docs<64, 128>(maps, a, plan, stream);
}

}  // namespace based
