// Decay attention, bf16 io, on tensor cores (tcgen05 + TMEM + TMA): the passes of decay.cuh in blocks of 128 tokens.
//
// One CTA per pass, head, tile of 64 output columns and segment walks the blocks.  Per block, with x, y [128, DC], z [128, 64] by TMA:
//   scores  x y^T [128,128]                    -> faded and masked by one thread per row, bf16, back over the scores (TMEM)
//   dS      y^T [give z, in two bf16 parts]    [DC, 64 + 64], fp32; the state itself, S <- f S + both halves, is held in
//           registers, one row a thread, so that no block's products wait for the block before it
//   Oa      P z,   Ob  x S [128, 64 each]      S rounded to bf16 in shared memory
//   out     factor (Oa + take Ob) -> bf16 -> TMA store
// give z in one bf16 part would put a second rounding beside that of S into every output, and 2^-9 into the state that a call returns;
// the two parts hold 16 bits and cost one product of N = 128 for one of N = 64, which shared memory bounds anyway.
//
// Groups of four warps: scores (P), state (S), feed (give z), results (O); one warp issues the loads, one the products, in the order
// scores n, dS n, Oa n-1, Ob n-1, so that every group has a block's products of time for its part.
#include <cuda_bf16.h>

#include "decay.cuh"
#include "sm100.cuh"

namespace based {

using namespace sm100;

namespace {

constexpr int kT = kDecayBlockTc, kThreads = 576;
constexpr int kWarpTma = 16, kWarpMma = 17;
constexpr uint32_t kPanel = kT * 128;                                // 128 tokens x 64 columns, bf16: 16 KB

template <int DC, bool STATES> struct Cfg {
    static constexpr int kPanels = DC / 64;
    static constexpr uint32_t offY = STATES ? 0 : kPanels * kPanel;  // in a stage: x, y, z
    static constexpr uint32_t offZ = offY + kPanels * kPanel;
    static constexpr uint32_t kStage = offZ + kPanel;
    static constexpr int kStages = DC == 128 ? (STATES ? 3 : 2) : (STATES ? 4 : 3);
    static constexpr uint32_t offZero = kStages * kStage;            // DC = 64: y's columns 64 .. 127
    static constexpr uint32_t offFeed = offZero + (DC == 64 ? kPanel : 0);
    static constexpr uint32_t offS = offFeed + 2 * kPanel;
    static constexpr uint32_t offOut = offS + (STATES ? 0 : DC * 128);
    static constexpr uint32_t offBars = offOut + (STATES ? 0 : kPanel);
    static constexpr uint32_t offPow = offBars + 256;                // a^0 .. a^128
    static constexpr uint32_t offPlaces = offPow + 528;
    static constexpr uint32_t kBytes = offPlaces + kStages * kT * 4 + 1024;
    static_assert(kBytes <= 232448, "shared memory budget");
};
// TMEM columns: two scores, Oa, Ob, dS
constexpr uint32_t colX = 0, colOa = 256, colOb = 320, colDS = 384;

// full, empty: a stage each.  bX, bP: scores there, P written, for two blocks in turn.  One phase a block: bFeed the feed written, bDS
// dS there, bDSread, bS the state before the block in shared memory, bO the block's results there, bOread.
enum Bar { bFull = 0, bEmpty = 4, bX = 8, bP = 10, bFeed = 12, bDS, bDSread, bS, bO, bOread, bCount };
static_assert(bCount * 8 + 8 <= 256, "barrier area");

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

template <int DC, bool STATES, bool DOCS>
__global__ void __launch_bounds__(kThreads, 1) decay_tc_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Args a) {
    using C = Cfg<DC, STATES>;
    constexpr int NS = C::kStages;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::offBars);
    uint32_t* tmem_base_s = reinterpret_cast<uint32_t*>(bars + bCount);
    volatile uint32_t* abort_flag = tmem_base_s + 1;
    float* pw = reinterpret_cast<float*>(smem + C::offPow);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const DecayItem it(blockIdx.x, a.c.passes, a.tiles, STATES ? a.segments - 1 : a.segments);
    const DecayPass& p = a.c.pass[it.pass];
    const int e0 = it.tile * kDecayTile, L = a.c.L;
    if (e0 >= p.de) return;
    const int b = (int)(it.head / a.c.H), h = (int)(it.head % a.c.H);
    const bool back = p.back;

    if (tid == 0) {
        for (int s = 0; s < bCount; ++s)
            mbar_init(&bars[s], s == bP || s == bP + 1 || s == bFeed || s == bDSread || s == bS || s == bOread ? 128 : 1);
        *abort_flag = 0;
        fence_mbar_init();
        for (int i = 0; i < 4; ++i) prefetch_tensormap(&maps.m[it.pass][i]);
    }
    if (DC == 64) {
        for (uint32_t i = tid * 16; i < kPanel; i += kThreads * 16) *reinterpret_cast<uint4*>(smem + C::offZero + i) = make_uint4(0, 0, 0, 0);
        fence_proxy_async_smem();
    }
    if (warp == kWarpMma) { tmem_alloc(tmem_base_s, 512); tmem_relinquish(); }
    enter_dependent();
    if (tid <= kT) pw[tid] = faded(a.c.rate[h] * kLog2e, tid);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tb = *tmem_base_s;
    bool ok = true;

    const int g = back ? a.segments - 1 - it.segment : it.segment;
    const int first = decay_first(a.blocks, a.segments, g), count = decay_first(a.blocks, a.segments, g + 1) - first;
    auto block_of = [&](int i) { return back ? first + count - 1 - i : first + i; };
    auto wait = [&](int bar, int phase) -> bool { return __all_sync(0xffffffffu, mbar_wait(&bars[bar], phase & 1, abort_flag)); };
    auto places_of = [&](int n) { return a.places + ((long long)b * a.blocks + n) * kT; };
    // the last token's place in block n: how many count, how many documents begin
    auto end_of = [&](int n) -> uint32_t { return DOCS ? places_of(n)[kT - 1] : (uint32_t)min(kT, L - n * kT); };
    // one document reaches over the whole block, and nothing in it is padding: as without documents
    auto plain = [&](uint32_t end, int n) { return !DOCS || (end & 0xffffu) == (uint32_t)min(kT, L - n * kT); };

    if (warp == kWarpTma) {
        if (lane == 0) {
            for (int i = 0; i < count; ++i) {
                const int s = i % NS, n = block_of(i), t0 = n * kT;
                if (i >= NS) ok = mbar_wait(&bars[bEmpty + s], (i / NS - 1) & 1, abort_flag);
                if (!ok) break;
                uint8_t* st = smem + s * C::kStage;
                uint64_t* full = &bars[bFull + s];
                mbar_arrive_expect_tx(full, C::kStage + (DOCS ? kT * 4 : 0));
#pragma unroll
                for (int j = 0; j < C::kPanels; ++j) {
                    if (!STATES) tma_load_4d(st + j * kPanel, &maps.m[it.pass][0], full, 64 * j, t0, h, b);
                    tma_load_4d(st + C::offY + j * kPanel, &maps.m[it.pass][1], full, 64 * j, t0, h, b);
                }
                tma_load_4d(st + C::offZ, &maps.m[it.pass][2], full, e0, t0, h, b);
                if (DOCS) bulk_load_1d(smem + C::offPlaces + s * kT * 4, places_of(n), kT * 4, full);
            }
        }
    } else if (warp == kWarpMma) {
        // the whole warp runs this block and one elected lane issues (see mma_ss_w)
        const uint32_t lead = elect_one();
        constexpr uint64_t dK = make_smem_desc_base(16, 1024, kSwizzle128B);             // K-major rows, or one MN-major block of 64
        constexpr uint64_t dN = make_smem_desc_base(kPanel, 1024, kSwizzle128B);         // MN-major, two blocks of 64 a panel apart
        constexpr uint32_t iX = make_idesc_bf16(128, 128, 0, 0), iO = make_idesc_bf16(128, 64, 0, 1), iD = make_idesc_bf16(128, 128, 1, 1);
        const uint32_t sm = smem_u32(smem);
        auto lo = [](uint64_t base, uint32_t addr) { return desc_lo(base) + (addr >> 4); };
        auto scores = [&](int i) {
            const uint32_t st = sm + (i % NS) * C::kStage, d = tb + colX + (i & 1) * 128;
            const uint32_t lx = lo(dK, st), ly = lo(dK, st + C::offY);
#pragma unroll
            for (int k = 0; k < DC / 16; ++k) {
                const uint32_t at = (k >> 2) * (kPanel >> 4) + (k & 3) * 2;
                if (k == 0) mma_ss_w<false>(lead, d, lx, desc_hi(dK), ly, desc_hi(dK), iX);
                else mma_ss_w<true>(lead, d, lx + at, desc_hi(dK), ly + at, desc_hi(dK), iX);
            }
            mma_commit_w(lead, &bars[bX + (i & 1)]);
        };
        auto delta = [&](int i) {
            const uint32_t y = sm + (i % NS) * C::kStage + C::offY, d = tb + colDS;
            const uint64_t dY = make_smem_desc_base(DC == 128 ? kPanel : sm + C::offZero - y, 1024, kSwizzle128B);
            const uint32_t ly = lo(dY, y), lf = lo(dN, sm + C::offFeed);
#pragma unroll
            for (int k = 0; k < kT / 16; ++k) {
                if (k == 0) mma_ss_w<false>(lead, d, ly, desc_hi(dN), lf, desc_hi(dN), iD);
                else mma_ss_w<true>(lead, d, ly + k * 128, desc_hi(dN), lf + k * 128, desc_hi(dN), iD);
            }
            mma_commit_w(lead, &bars[bDS]);
        };
        auto results = [&](int i) -> bool {
            if (!wait(bP + (i & 1), i >> 1)) return false;
            if (i > 0 && !wait(bOread, i - 1)) return false;
            tc_fence_after();
            const uint32_t st = sm + (i % NS) * C::kStage, px = tb + colX + (i & 1) * 128;
            const uint32_t lz = lo(dK, st + C::offZ), lx = lo(dK, st), ls = lo(dK, sm + C::offS);
#pragma unroll
            for (int k = 0; k < kT / 16; ++k) {
                if (k == 0) mma_ts_w<false>(lead, tb + colOa, px, lz, desc_hi(dK), iO);
                else mma_ts_w<true>(lead, tb + colOa, px + k * 8, lz + k * 128, desc_hi(dK), iO);
            }
            if (!wait(bS, i)) return false;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < DC / 16; ++k) {
                const uint32_t at = (k >> 2) * (kPanel >> 4) + (k & 3) * 2;
                if (k == 0) mma_ss_w<false>(lead, tb + colOb, lx, desc_hi(dK), ls, desc_hi(dK), iO);
                else mma_ss_w<true>(lead, tb + colOb, lx + at, desc_hi(dK), ls + k * 128, desc_hi(dK), iO);
            }
            mma_commit_w(lead, &bars[bO]);
            mma_commit_w(lead, &bars[bEmpty + i % NS]);
            return true;
        };
#pragma unroll 1
        for (int i = 0; i < count && ok; ++i) {
            ok = wait(bFull + i % NS, i / NS);
            if (!ok) break;
            tc_fence_after();
            if (!STATES) scores(i);
            ok = wait(bFeed, i) && (i == 0 || wait(bDSread, i - 1));
            if (!ok) break;
            tc_fence_after();
            delta(i);
            if (STATES) mma_commit_w(lead, &bars[bEmpty + i % NS]);
            else if (i > 0) ok = results(i - 1);
        }
        if (!STATES && ok && count > 0) ok = results(count - 1);
    } else if (warp < 4) {
        // ---- scores: thread = row of the block, TMEM lane
        if constexpr (!STATES) {
            const int r = tid, w = warp;
            for (int i = 0; i < count; ++i) {
                const int n = block_of(i);
                const uint32_t end = end_of(n);
                ok = wait(bX + (i & 1), i >> 1);
                if (!ok) break;
                tc_fence_after();
                const uint32_t tx = tmem_addr(tb, (uint32_t)w * 32u, colX + (i & 1) * 128);
                const uint32_t* pl = reinterpret_cast<const uint32_t*>(smem + C::offPlaces + (i % NS) * kT * 4);
                const bool simple = plain(end, n);
                const uint32_t own = DOCS && !simple ? pl[r] : 0u;
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {                        // 32 columns a time
                    uint32_t pk[16];
                    if (back ? c < w : c > w) {
#pragma unroll
                        for (int k = 0; k < 16; ++k) pk[k] = 0u;
                    } else {
                        uint32_t x[32];
                        tmem_ld32(tx + 32 * c, x);
                        tmem_wait_ld();
                        if (simple) {
                            if (c == w) {
#pragma unroll
                                for (int k = 0; k < 32; ++k) {
                                    const int steps = back ? k - lane : lane - k;
                                    x[k] = steps >= 0 ? __float_as_uint(__uint_as_float(x[k]) * pw[steps]) : 0u;
                                }
                            } else {                                 // steps from the row to the nearer end of the columns, and on from there
                                const float f = pw[back ? 32 * c - r : r - 32 * c - 31];
#pragma unroll
                                for (int k = 0; k < 32; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) * f * pw[back ? k : 31 - k]);
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
                    tmem_st16(tx + 16 * c, pk);                      // (over columns that this row has read, or does not need)
                }
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(&bars[bP + (i & 1)]);
            }
        }
    } else if (warp < 8) {
        // ---- state: thread = row of the state, TMEM lane
        const int w = warp & 3, c = 32 * w + lane;
        const bool rows = w * 32 < DC;                               // (the whole warp's)
        float s[64];
#pragma unroll
        for (int e = 0; e < 64; ++e) s[e] = 0.f;
        if (!STATES && rows) {
            if (p.state_in && c < p.dc) {
                const float* in = p.state_in + it.head * p.dc * p.de;
#pragma unroll
                for (int e = 0; e < 64; ++e)
                    if (e0 + e < p.de) s[e] = p.in_factor * in[p.turned ? (long long)(e0 + e) * p.dc + c : (long long)c * p.de + e0 + e];
            }
            for (int k = 0; k < it.segment; ++k) {
                const long long slot = decay_slot(it.pass, a.c.passes, it.head, a.tiles, it.tile, a.segments, k);
                const float f = a.factors[slot];
                const float4* from = reinterpret_cast<const float4*>(a.states + (slot * kDecayMaxWidth + c) * kDecayTile);
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
                uint8_t* row = smem + C::offS + c * 128;
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
        float whole = 1.f;
        for (int i = 0; i < count; ++i) {
            const uint32_t end = end_of(block_of(i));
            const float f = place_run(end) == 0 ? pw[place_count(end)] : 0.f;
            ok = wait(bDS, i);
            if (!ok) break;
            tc_fence_after();
            if (rows) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t x[16], y[16];
                    tmem_ld16(tmem_addr(tb, (uint32_t)w * 32u, colDS + 16 * q), x);
                    tmem_ld16(tmem_addr(tb, (uint32_t)w * 32u, colDS + 64 + 16 * q), y);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[16 * q + e] = fmaf(f, s[16 * q + e], __uint_as_float(x[e]) + __uint_as_float(y[e]));
                }
            }
            whole *= f;
            tc_fence_before();
            mbar_arrive(&bars[bDSread]);
            if (!STATES && i + 1 < count) {
                ok = wait(bO, i);                                    // (the products with the state before have read it)
                if (!ok) break;
                to_shared();
            }
        }
        if (ok && rows) {
            if (STATES) {
                const long long slot = decay_slot(it.pass, a.c.passes, it.head, a.tiles, it.tile, a.segments, it.segment);
                float4* to = reinterpret_cast<float4*>(a.states + (slot * kDecayMaxWidth + c) * kDecayTile);
#pragma unroll
                for (int e = 0; e < 64; e += 4) to[e / 4] = make_float4(s[e], s[e + 1], s[e + 2], s[e + 3]);
                if (c == 0) a.factors[slot] = whole;
            } else if (p.state_out && it.segment == a.segments - 1 && c < p.dc) {
                float* to = p.state_out + it.head * p.dc * p.de;
#pragma unroll
                for (int e = 0; e < 64; ++e)
                    if (e0 + e < p.de) to[p.turned ? (long long)(e0 + e) * p.dc + c : (long long)c * p.de + e0 + e] = p.out_factor * s[e];
            }
        }
    } else if (warp < 12) {
        // ---- feed: give z as two bf16 parts, 16 bytes of 8 rows per thread; rows of padding out of y and z
        const int u = tid & 127;
        for (int i = 0; i < count; ++i) {
            const int n = block_of(i);
            const uint32_t end = end_of(n);
            const bool simple = plain(end, n);
            const int c1 = place_count(end);
            ok = wait(bFull + i % NS, i / NS);
            if (ok && i > 0) ok = wait(bDS, i - 1);
            if (!ok) break;
            uint8_t* st = smem + (i % NS) * C::kStage;
            const uint32_t* pl = reinterpret_cast<const uint32_t*>(smem + C::offPlaces + (i % NS) * kT * 4);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int row = (u >> 3) + 16 * j;
                const uint32_t at = (uint32_t)(j * 128 + u) * 16;
                float w;
                if (simple) {
                    w = row < c1 ? pw[back ? row + 1 : c1 - 1 - row] : 0.f;
                } else {
                    const uint32_t q = pl[row];
                    if (q & kPadding) {
                        w = 0.f;
                        const uint4 zero = make_uint4(0, 0, 0, 0);
                        *reinterpret_cast<uint4*>(st + C::offZ + at) = zero;
#pragma unroll
                        for (int k = 0; k < C::kPanels; ++k) *reinterpret_cast<uint4*>(st + C::offY + k * kPanel + at) = zero;
                    } else {
                        w = back ? (place_run(q) == 0 ? pw[place_count(q)] : 0.f)
                                 : (place_run(q) == place_run(end) ? pw[c1 - place_count(q)] : 0.f);
                    }
                }
                const uint4 z = *reinterpret_cast<const uint4*>(st + C::offZ + at);
                const uint32_t in[4] = {z.x, z.y, z.z, z.w};
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float x0 = lo_f32(in[k]) * w, x1 = hi_f32(in[k]) * w;
                    hi[k] = pack2(x0, x1);
                    lo[k] = pack2(x0 - lo_f32(hi[k]), x1 - hi_f32(hi[k]));
                }
                *reinterpret_cast<uint4*>(smem + C::offFeed + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                *reinterpret_cast<uint4*>(smem + C::offFeed + kPanel + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
            fence_proxy_async_smem();
            mbar_arrive(&bars[bFeed]);
        }
    } else {
        // ---- results: thread = row of the block, TMEM lane
        if constexpr (!STATES) {
            const int w = warp & 3, r = tid & 127;
            uint8_t* row = smem + C::offOut + r * 128;
            const uint32_t sw = r & 7;
            const float factor = a.c.factor;
            for (int i = 0; i < count; ++i) {
                const int n = block_of(i);
                const uint32_t end = end_of(n);
                float take;
                if (plain(end, n)) {
                    take = back ? pw[max(place_count(end) - 1 - r, 0)] : pw[r + 1];
                } else {
                    const uint32_t q = places_of(n)[r];
                    take = q & kPadding ? 0.f
                           : back       ? (place_run(q) == place_run(end) ? pw[place_count(end) - place_count(q)] : 0.f)
                                        : (place_run(q) == 0 ? pw[place_count(q)] : 0.f);
                }
                ok = group_all(1, mbar_wait(&bars[bO], i & 1, abort_flag));
                if (!ok) break;
                tc_fence_after();
                uint32_t v[32];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t x[16], y[16];
                    tmem_ld16(tmem_addr(tb, (uint32_t)w * 32u, colOa + 16 * q), x);
                    tmem_ld16(tmem_addr(tb, (uint32_t)w * 32u, colOb + 16 * q), y);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        // (no product with a weight of 0: there the state's share need not be finite)
                        const float o0 = take == 0.f ? __uint_as_float(x[2 * e]) : fmaf(take, __uint_as_float(y[2 * e]), __uint_as_float(x[2 * e]));
                        const float o1 = take == 0.f ? __uint_as_float(x[2 * e + 1]) : fmaf(take, __uint_as_float(y[2 * e + 1]), __uint_as_float(x[2 * e + 1]));
                        v[8 * q + e] = pack2(o0 * factor, o1 * factor);
                    }
                }
                tc_fence_before();
                mbar_arrive(&bars[bOread]);
                if (r == 0) tma_store_wait_read<0>();
                group_all(1, true);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    *reinterpret_cast<uint4*>(row + (((uint32_t)j ^ sw) << 4)) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                fence_proxy_async_smem();
                group_all(1, true);
                if (r == 0) {
                    tma_store_4d(&maps.m[it.pass][3], smem + C::offOut, e0, n * kT, h, b);
                    tma_store_commit();
                }
            }
            if (r == 0) tma_store_wait<0>();
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

template <int DC, bool STATES, bool DOCS> based_status launch(const Maps& maps, const Args& a, long long ctas, cudaStream_t stream) {
    using C = Cfg<DC, STATES>;
    auto kern = decay_tc_kernel<DC, STATES, DOCS>;
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
template <int DC, bool DOCS> based_status launch_both(const Maps& maps, const Args& a, const DecayPlan& plan, cudaStream_t stream) {
    if (plan.segments > 1) {
        const based_status st = launch<DC, true, DOCS>(maps, a, plan.ctas / plan.segments * (plan.segments - 1), stream);
        if (st != BASED_OK) return st;
    }
    return launch<DC, false, DOCS>(maps, a, plan.ctas, stream);
}

}  // namespace

int decay_tc_slots() { return kSMs; }

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
        return wide ? launch_both<128, true>(maps, a, plan, stream) : launch_both<64, true>(maps, a, plan, stream);
    }
    return wide ? launch_both<128, false>(maps, a, plan, stream) : launch_both<64, false>(maps, a, plan, stream);
}

}  // namespace based
