// swa_backward, bf16 tensor-core path (tcgen05 + TMEM + TMA), one kernel, every input read once:
//
//   P_ij = exp(c (s_ij - m_i)) / l_i,  D_i = sum_j P_ij dP_ij,  dS_ij = c P_ij (dP_ij - D_i)        (s = Q K^T, dP = dO V^T)
//   dQ_i = sum_j dS_ij k_j,   dK_j = sum_i dS_ij q_i,   dV_j = sum_i P_ij dO_i
//
// Persistent CTAs (one per SM) walk contiguous runs of tiles of 128 queries.  The tile at i0 sees the keys from i0 - PAD on
// (PAD = 64 for windows up to 65, else 128): 128 + PAD columns.  Per tile
//   S, then dP   [128, 128 + PAD] into the same TMEM columns
//   softmax      two threads per query row, each with half of the 32 + PAD columns its warp's rows can touch; the statistics
//                m, l, sum P dP join through shared memory; P and dS go to shared memory as bf16
//   dQ           dS K, dS read with the queries as rows
//   dK, dV       dS^T Q, P^T dO, the same bytes read with the keys as rows
// Key blocks of 128 are shifted by PAD against the query tiles, so that block b = keys 128 b - PAD .. 128 b - PAD + 127 meets
// query tiles b - 1 and b alone: tile b - 1 starts its accumulators and tile b completes them.  They stay in TMEM (two sets)
// and no gradient is added into memory.  A run that starts inside a head first recomputes the tile before it, for the
// block that it completes next.
//
// P and dS are rounded to bf16 for the products, as the forward pass rounds P (by half a step, up to 2^-8 of each weight: tensor cores take
// both operands in one type, and K, Q, dO are bf16); scores, dP, statistics and sums are fp32.  The gradients are 0.0024 (2-norm,
// relative) off those of 64 bits, 0.0017 of it their own rounding; 64 bits with these roundings and no others are as far off.
//
// Shared memory (226 KB, which is why there is one CTA per SM): rings of 64-key halves of K (those under a tile and two of the
// next) and V (four), three places for Q, two for dO; P and dS.  A tile's results leave through its place of Q, once the products
// have read that: 32 rows a time and warp, by TMA.  Rows of warp u (32 of them) touch columns 32 u .. 32 u + 31 + PAD only; what
// lies outside is zeroed once and never written.  With PAD 64, P and dS have 32 KB each (column block 1 by all rows, the upper
// half of block 0, the lower half of block 2) and share one piece of 8 KB of zeros that stands for the blocks' other halves.
// With PAD 128 they take turns in one array of 64 KB, and dQ lies over dP in TMEM: the next tile's S starts with the three
// halves beside it, while dQ is read out.
//
// Order of the products of tile n: [PAD 64: S of n + 1,] dQ, [PAD 128: dV ahead of it, S of n + 1 after it,] dV, dK, then dP of
// n + 1, so that the softmax warps find S of the next tile when they are done with this one.
//
// Measured, bf16: 2 x 16 heads x 32768 queries, window 64: 178 us over 50 calls, 208 in a long run at the power limit (69 %
// of the copy rate; the chain S - softmax - dP - dS - products of a tile, some 5900 cycles where HBM's share is 4700).  3 x 16
// heads x 1777 queries, window 128: 36 us, some 8900 cycles per tile, 5.5 tiles per SM with the recomputed ones; of them 2300 for
// the exponentials, 1500 each for writing P and dS.  It was 51 us with S of the next tile behind all of this one's results and dS
// worked out behind dV's products; four softmax threads per row took 39.5 (80 registers, spills), and 248 with PAD 64.
#include <cuda_bf16.h>

#include "common.cuh"
#include "pairs.cuh"
#include "sm100.cuh"

namespace based {

using namespace sm100;

namespace {

constexpr int kQT = 128, kHD = 64;
constexpr int kWarpOut = 8, kWarpTma = 12, kWarpMma = 13, kThreads = 448;
constexpr uint32_t kTileBytes = kQT * kHD * 2, kHalfBytes = 64 * kHD * 2;       // 16 KB of Q or dO, 8 KB of 64 keys or values
template <int PAD> struct Cfg {
    static constexpr int kHalves = 2 + PAD / 64;                     // 64-key halves under a tile: 3 or 4
    // Rings of halves: of K all that are under a tile and two for the next; of V, whose halves are done with early, four in all
    static constexpr int kSlotsK = kHalves + 2, kSlotsV = 4;
    static constexpr int kSlotsQ = 3, kSlotsO = 2;                   // tiles of Q, dO
    static constexpr int kCols = (32 + PAD) / 2;                     // columns per softmax thread: 48 or 80
    static constexpr bool kShared = PAD == 128;                      // P and dS in one array
    static constexpr uint32_t offV = kSlotsK * kHalfBytes;
    static constexpr uint32_t offQ = offV + kSlotsV * kHalfBytes;
    static constexpr uint32_t offO = offQ + kSlotsQ * kTileBytes;
    static constexpr uint32_t offP = offO + kSlotsO * kTileBytes;    // P and dS
    static constexpr uint32_t offBars = offP + (PAD == 64 ? 73728u : 65536u);
    static constexpr uint32_t kSmemBytes = offBars + 512 + 1024;
    static_assert(kSmemBytes <= 232448, "shared memory budget");
    // Byte offset from offP of row 0 of the block of 64 columns cb in P or dS.  PAD 64: block 0 has rows 0 .. 63 only and block 2 rows
    // 64 .. 127 only; one piece of 8 KB of zeros at kZero stands for what is missing.  It lies behind dS's block 0 and before its block
    // 2, so that dQ's products read those with their missing rows; dK's and dV's reach it by their strides.
    static constexpr uint32_t kZero = 49152;
    static __host__ __device__ constexpr uint32_t block(bool ds, int cb) {
        return PAD == 64 ? (ds ? (cb == 1 ? 24576u : cb == 0 ? 40960u : 49152u) : (cb == 1 ? 0u : cb == 0 ? 16384u : 57344u))
                         : (cb == 1 ? 0u : cb == 0 ? 16384u : cb == 3 ? 32768u : 49152u);
    }
};
// TMEM columns: scores (and dP after them), dQ, two sets of (dK, dV)
constexpr uint32_t colX = 0, colAcc = 256;
template <int PAD> constexpr uint32_t colDQ = PAD == 64 ? 192 : 0;   // PAD 128: over dP once that is read

// One phase per tile each, of the pairs one in two tiles (so that nobody can be a whole turn behind):
//   bFullA  Q and the new halves of K are there      bFullB  dO and the new halves of V are there
//   bS, bDP  scores, dP are there                    bSread, bP, bPS  scores read; P (PAD 128), P and dS written
//   bPdone  dV's products are done (PAD 128)         bKdone  so are dQ's, and with them the use of K
//   bDone   all products are done                    bOut    the results have been read out of tensor memory
// and for each of the three places of Q, bEmptyQ: the results that went out through it have left.
enum Bar { bFullA = 0, bFullB = 2, bKdone = 4, bDone = 6, bEmptyQ = 8, bS = 11, bSread, bDP, bP, bPdone, bPS, bOutQ, bOut, bCount };
static_assert(bCount * 8 + 8 <= 512, "barrier area");

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
// barrier of 64 threads that also tells whether all of them say yes
__device__ __forceinline__ bool pair_all(int id, bool pred) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %1, 0;\n\t"
        "bar.red.and.pred q, %2, 64, p;\n\t"
        "selp.b32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)pred), "r"(id)
        : "memory");
    return r != 0;
}

struct Params {
    unsigned int* err;
    int L, window, tiles_per_head, total_tiles;
    float scale, scale_log2e;
};
// one of a CTA's tiles
struct Tile {
    int head, i;
    bool halo, first, last, end;       // recomputed only; a head's first, last; the run's last
};
struct Run {
    int g0, halo, count, nt;
    __device__ __forceinline__ Run(const Params& p) {
        g0 = (int)((long long)p.total_tiles * blockIdx.x / gridDim.x);
        const int g1 = (int)((long long)p.total_tiles * (blockIdx.x + 1) / gridDim.x);
        nt = p.tiles_per_head;
        halo = g1 > g0 && g0 % nt != 0;
        count = g1 - g0 + halo;
    }
    __device__ __forceinline__ Tile tile(int n) const {
        const int g = g0 - halo + n;
        Tile t;
        t.head = g / nt;
        t.i = g - t.head * nt;
        t.halo = n < halo;
        t.first = t.i == 0;
        t.last = t.i == nt - 1;
        t.end = n == count - 1;
        return t;
    }
};

// A row of 64 fp32 values in TMEM per lane, rounded to bf16: 8 chunks of 16 bytes
__device__ __forceinline__ void read_rows(uint32_t taddr, uint32_t (&c)[8][4]) {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        uint32_t t[16];
        tmem_ld16(taddr + 16 * h, t);
        tmem_wait_ld();
#pragma unroll
        for (int k = 0; k < 8; ++k) c[2 * h + (k >> 2)][k & 3] = pack2(__uint_as_float(t[2 * k]), __uint_as_float(t[2 * k + 1]));
    }
}
// to a piece of shared memory, swizzled as the TMA store of 32 rows reads it
__device__ __forceinline__ void stage_rows(const uint32_t (&c)[8][4], uint8_t* tile, int lane) {
    uint8_t* row = tile + (lane >> 3) * 1024 + (lane & 7) * 128;
    const uint32_t sw = lane & 7;
#pragma unroll
    for (int j = 0; j < 8; ++j) *reinterpret_cast<uint4*>(row + (((uint32_t)j ^ sw) << 4)) = make_uint4(c[j][0], c[j][1], c[j][2], c[j][3]);
}

}  // namespace

template <int PAD>
__global__ void __launch_bounds__(kThreads, 1)
    swa_backward_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                           const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_o,
                           const __grid_constant__ CUtensorMap tm_dq, const __grid_constant__ CUtensorMap tm_dk,
                           const __grid_constant__ CUtensorMap tm_dv, const Params p) {
    using C = Cfg<PAD>;
    constexpr int NH = C::kHalves, NK = C::kSlotsK, NV = C::kSlotsV, NC = C::kCols;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::offBars);
    uint32_t* tmem_base_s = reinterpret_cast<uint32_t*>(bars + bCount);
    volatile uint32_t* abort_flag = tmem_base_s + 1;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Run run(p);
    const int N = run.count;

    if (tid == 0) {
        for (int s = 0; s < bCount; ++s) mbar_init(&bars[s], s == bSread || s == bP || s == bPS ? 256 : s == bOut || s == bOutQ ? 128 : s >= bEmptyQ && s < bS ? 4 : 1);
        *abort_flag = 0;
        fence_mbar_init();
        prefetch_tensormap(&tm_q); prefetch_tensormap(&tm_k); prefetch_tensormap(&tm_v); prefetch_tensormap(&tm_o);
    }
    for (uint32_t i = tid * 16; i < C::offBars - C::offP; i += kThreads * 16) *reinterpret_cast<uint4*>(smem + C::offP + i) = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    if (warp == kWarpMma) { tmem_alloc(tmem_base_s, 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    enter_dependent();
    const uint32_t tb = *tmem_base_s;
    bool ok = true;

    if (warp == kWarpTma) {
        if (lane == 0) {
            int hk = 0, hv = 0;                                      // halves of K, of V loaded so far
            for (int n = 0; n < N; ++n) {
                const Tile t = run.tile(n);
                const int from = n == 0 || t.first ? 0 : NH - 2;     // (all halves are new, or the last two; rows outside the head read as zeros)
                const int o = n & 1, key = t.i * kQT - PAD;
                // Q and K: where tile n - 3 had its Q, tile n - 2 the halves that tile n - 1 did not use (a new head: that tile n - 1 had)
                const int sq = n % C::kSlotsQ;
                if (n >= C::kSlotsQ) ok = mbar_wait(&bars[bEmptyQ + sq], (n / C::kSlotsQ - 1) & 1, abort_flag);
                if (!ok) break;
                if (n >= 2) ok = mbar_wait(&bars[bKdone + o], ((n - 2) >> 1) & 1, abort_flag);
                if (ok && n > 0 && t.first) ok = mbar_wait(&bars[bKdone + (o ^ 1)], ((n - 1) >> 1) & 1, abort_flag);
                if (!ok) break;
                mbar_arrive_expect_tx(&bars[bFullA + o], kTileBytes + (NH - from) * kHalfBytes);
                tma_load_3d(smem + C::offQ + sq * kTileBytes, &tm_q, &bars[bFullA + o], 0, t.i * kQT, t.head);
                for (int j = from; j < NH; ++j, ++hk)
                    tma_load_3d(smem + (hk % NK) * kHalfBytes, &tm_k, &bars[bFullA + o], 0, key + 64 * j, t.head);
                // dO and V: where tile n - 2 had its dO, and once tile n - 1 is done with V
                if (n >= 2) ok = mbar_wait(&bars[bDone + o], ((n - 2) >> 1) & 1, abort_flag);
                if (ok && n > 0) ok = mbar_wait(&bars[bDP], (n - 1) & 1, abort_flag);
                if (!ok) break;
                mbar_arrive_expect_tx(&bars[bFullB + o], kTileBytes + (NH - from) * kHalfBytes);
                tma_load_3d(smem + C::offO + o * kTileBytes, &tm_o, &bars[bFullB + o], 0, t.i * kQT, t.head);
                for (int j = from; j < NH; ++j, ++hv)
                    tma_load_3d(smem + C::offV + (hv % NV) * kHalfBytes, &tm_v, &bars[bFullB + o], 0, key + 64 * j, t.head);
            }
        }
    } else if (warp == kWarpMma) {
        // the whole warp runs this block and one elected lane issues (see mma_ss_w)
        const uint32_t lead = elect_one();
        constexpr uint64_t d1 = make_smem_desc_base(16, 1024, kSwizzle128B);              // K-major rows, or one MN-major block of 64
        constexpr uint64_t dA = make_smem_desc_base(16384, 1024, kSwizzle128B);           // MN-major, blocks 1 and 0 (3 and 2)
        constexpr uint32_t iS0 = make_idesc_bf16(128, 0, 0, 0), iQ = make_idesc_bf16(128, 64, 0, 1), iK = make_idesc_bf16(128, 64, 1, 1);
        const uint32_t sm = smem_u32(smem);
        // (the same answer for the whole warp, and known to be: what depends on it stays in uniform registers)
        auto wait = [&](int bar, int phase) -> bool { return __all_sync(0xffffffffu, mbar_wait(&bars[bar], phase & 1, abort_flag)); };
        auto lo = [](uint64_t base, uint32_t addr) { return desc_lo(base) + (addr >> 4); };
        int hb = 0;                                                  // the tile's first half, counted as they are loaded
        int acc = 0;                                                 // the set its key block is in
        auto tile_q = [&](int n) { return sm + C::offQ + (n % C::kSlotsQ) * kTileBytes; };
        auto tile_o = [&](int n) { return sm + C::offO + (n & 1) * kTileBytes; };
        // scores or dP: rows of `a` (Q or dO) by halves j0 .. j1 - 1 in a ring of NR slots, as many at a time as lie side by side: a product
        // reads `a` once however many they are, and shared memory's bandwidth is what bounds the products
        auto scores = [&](uint32_t a, uint32_t ring, int NR, int j0, int j1) {
            const uint32_t la = lo(d1, a);
#pragma unroll 1
            for (int j = j0, count; j < j1; j += count) {
                const int slot = (hb + j) % NR;
                count = min(j1 - j, NR - slot);
                const uint32_t lb = lo(d1, ring + slot * kHalfBytes), d = tb + colX + 64 * j;
                const uint32_t i = iS0 | (uint32_t)(8 * count) << 17;
                mma_ss_w<false>(lead, d, la, desc_hi(d1), lb, desc_hi(d1), i);
#pragma unroll
                for (int k = 1; k < 4; ++k) mma_ss_w<true>(lead, d, la + k * 2, desc_hi(d1), lb + k * 2, desc_hi(d1), i);
            }
        };
        auto issue_s = [&](int n) -> bool {
            if (!wait(bFullA + (n & 1), n >> 1)) return false;
            tc_fence_after();
            if (PAD == 128 && n > 0) {                               // dQ of the tile before lies over the first half's scores
                scores(tile_q(n), sm, NK, 1, NH);
                if (!wait(bOutQ, n - 1)) return false;
                tc_fence_after();
                scores(tile_q(n), sm, NK, 0, 1);
            } else {
                scores(tile_q(n), sm, NK, 0, NH);
            }
            mma_commit_w(lead, &bars[bS]);
            return true;
        };
        auto issue_dp = [&](int n) -> bool {
            if (!wait(bSread, n) || !wait(bFullB + (n & 1), n >> 1)) return false;
            tc_fence_after();
            scores(tile_o(n), sm + C::offV, NV, 0, NH);
            mma_commit_w(lead, &bars[bDP]);
            return true;
        };
        // X^T Y of the tile's key block A (completing its accumulators) and of block B (starting the next one's); x: offset of P or dS
        auto part = [&](uint32_t x, uint32_t stride, uint32_t y, uint32_t d, int steps, bool begin) {
            const uint64_t base = make_smem_desc_base(stride, 1024, kSwizzle128B);
            const uint32_t lx = lo(base, x), ly = lo(d1, y);
            if (begin) mma_ss_w<false>(lead, d, lx, desc_hi(dA), ly, desc_hi(d1), iK);
            else mma_ss_w<true>(lead, d, lx, desc_hi(dA), ly, desc_hi(d1), iK);
#pragma unroll
            for (int k = 1; k < 4; ++k) mma_ss_w<true>(lead, d, lx + k * 128, desc_hi(dA), ly + k * 128, desc_hi(d1), iK);
            if (steps == 8) {
#pragma unroll
                for (int k = 4; k < 8; ++k) mma_ss_w<true>(lead, d, lx + k * 128, desc_hi(dA), ly + k * 128, desc_hi(d1), iK);
            }
        };
        auto block_a = [&](bool ds, uint32_t y, uint32_t d, bool begin) {
            const uint32_t x = sm + C::offP + C::block(ds, 1);
            if constexpr (PAD == 64) {                               // rows 64 .. 127 have no block 0: zeros
                part(x, 16384, y, d, 4, begin);
                part(x + 8192, C::kZero - C::block(ds, 1) - 8192, y + 8192, d, 4, false);
            } else {
                part(x, 16384, y, d, 8, begin);
            }
        };
        auto block_b = [&](bool ds, uint32_t y, uint32_t d) {
            if constexpr (PAD == 64)                                 // only rows 64 .. 127 see block 2; no block 3: zeros
                part(sm + C::offP + C::kZero, C::block(ds, 2) + 8192 - C::kZero, y + 8192, d, 4, true);
            else
                part(sm + C::offP + C::block(ds, 3), 16384, y, d, 8, true);
        };
        auto acc_col = [&](int a, int which) { return tb + colAcc + 128 * a + 64 * which; };     // 0: dK, 1: dV
        ok = issue_s(0) && issue_dp(0);
#pragma unroll 1
        for (int n = 0; n < N && ok; ++n) {
            const Tile t = run.tile(n);
            const bool with_b = !t.end || t.last;                    // the next block is this run's too
            const bool early = !t.end && !t.last;                    // (a new head's halves wait for this tile's slots)
            const int drop = t.last ? NH : 2;                        // halves that the next tile does not use
            // dV, or dV and dK.  What they begin was last used by the tile before and has been read out
            auto products = [&](int from, int to) {
#pragma unroll 1
                for (int which = from; which >= to; --which) {
                    const uint32_t y = which ? tile_o(n) : tile_q(n);
                    if (!t.halo) block_a(!which, y, acc_col(acc, which), t.first);
                    if (with_b) block_b(!which, y, acc_col(acc ^ 1, which));
                }
            };
            if constexpr (C::kShared) {
                ok = wait(bP, n) && (n == 0 || wait(bOut, n - 1));
                if (!ok) break;
                tc_fence_after();
                products(1, 1);
                mma_commit_w(lead, &bars[bPdone]);
            }
            ok = wait(bPS, n);
            if (!ok) break;
            tc_fence_after();
            if (PAD == 64 && early) {
                hb += drop;
                ok = issue_s(n + 1);
                hb -= drop;
            }
            if (PAD == 64 && ok && n > 0) ok = wait(bOut, n - 1);
            if (!ok) break;
            tc_fence_after();
            if (!t.halo) {
                const uint32_t d = tb + colDQ<PAD>;
#pragma unroll
                for (int j = 0; j < NH; ++j) {
                    const uint32_t la = lo(d1, sm + C::offP + C::block(true, j)), lb = lo(d1, sm + ((hb + j) % NK) * kHalfBytes);
                    if (j == 0) mma_ss_w<false>(lead, d, la, desc_hi(d1), lb, desc_hi(d1), iQ);
                    else mma_ss_w<true>(lead, d, la, desc_hi(d1), lb, desc_hi(d1), iQ);
#pragma unroll
                    for (int k = 1; k < 4; ++k) mma_ss_w<true>(lead, d, la + k * 2, desc_hi(d1), lb + k * 128, desc_hi(d1), iQ);
                }
            }
            mma_commit_w(lead, &bars[bKdone + (n & 1)]);
            hb += drop;
            if (PAD == 128 && early) ok = issue_s(n + 1);
            if (!ok) break;
            products(C::kShared ? 0 : 1, 0);
            mma_commit_w(lead, &bars[bDone + (n & 1)]);
            if (!t.last) acc ^= 1;
            if (!t.end) ok = (early || issue_s(n + 1)) && issue_dp(n + 1);
        }
    } else if (warp >= kWarpOut) {
        // ---- results: four warps, a TMEM lane per thread.  dQ; dK, dV of the key block that a tile completes (lanes 0 .. 63 hold its
        // keys 64 .. 127 and the other way round); of the one behind a head's last tile
        const int u = warp & 3;
        const uint32_t lanes = (uint32_t)u * 32u;
        int acc = 0;
        for (int n = 0; n < N && ok; ++n) {
            const Tile t = run.tile(n);
            uint32_t c[PAD == 64 ? 3 : 2][8][4];
            auto wait = [&](int bar) -> bool { return __all_sync(0xffffffffu, mbar_wait(&bars[bar + (n & 1)], (n >> 1) & 1, abort_flag)); };
            if constexpr (PAD == 128) {                              // (S of the next tile waits for it)
                ok = wait(bKdone);
                if (!ok) break;
                tc_fence_after();
                if (!t.halo) read_rows(tmem_addr(tb, lanes, colDQ<PAD>), c[0]);
                tc_fence_before();
                mbar_arrive(&bars[bOutQ]);
            }
            ok = wait(bDone);
            if (!ok) break;
            tc_fence_after();
            const int key = t.i * kQT - PAD + (int)(lanes ^ 64u);
            // out through the place of the tile's Q, which three tiles share: 32 rows a time per warp
            uint8_t* own = smem + C::offQ + (n % C::kSlotsQ) * kTileBytes + u * 4096;
            auto send = [&](const uint32_t (&c)[8][4], const CUtensorMap& map, int row) {
                if (lane == 0) tma_store_wait_read<0>();             // (the one before has been read)
                __syncwarp();
                stage_rows(c, own, lane);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (row >= 0 && row < p.L) tma_store_3d(&map, own, 0, row, t.head);
                    tma_store_commit();
                }
            };
            if (PAD == 128 && !t.halo) send(c[0], tm_dq, t.i * kQT + (int)lanes);
            if (t.last) {
                read_rows(tmem_addr(tb, lanes, colAcc + 128 * (acc ^ 1)), c[0]);
                send(c[0], tm_dk, key + kQT);
                read_rows(tmem_addr(tb, lanes, colAcc + 128 * (acc ^ 1) + 64), c[0]);
                send(c[0], tm_dv, key + kQT);
            }
            if (!t.halo) {
                read_rows(tmem_addr(tb, lanes, colAcc + 128 * acc), c[0]);
                read_rows(tmem_addr(tb, lanes, colAcc + 128 * acc + 64), c[1]);
                if constexpr (PAD == 64) read_rows(tmem_addr(tb, lanes, colDQ<PAD>), c[2]);
            }
            tc_fence_before();
            mbar_arrive(&bars[bOut]);
            if (!t.halo) {
                send(c[0], tm_dk, key);
                send(c[1], tm_dv, key);
                if constexpr (PAD == 64) send(c[2], tm_dq, t.i * kQT + (int)lanes);
            }
            if (lane == 0) {
                tma_store_wait_read<0>();
                mbar_arrive(&bars[bEmptyQ + n % C::kSlotsQ]);
            }
            if (!t.last) acc ^= 1;
        }
        if (lane == 0) tma_store_wait<0>();
    } else {
        // ---- softmax: warps u and u + 4 share the rows of TMEM lanes 32 u .. 32 u + 31, half of their columns each
        const int u = warp & 3, half = warp >> 2;
        const int r = 32 * u + lane;
        const int c0 = 32 * u + half * NC, c1 = 32 * u + (half ^ 1) * NC;      // first column, of this thread and of its partner
        const uint32_t tx = tmem_addr(tb, (uint32_t)u * 32u, colX + c0);
        const uint32_t sw = r & 7;
        // the 16 bytes of columns c .. c + 7 of this row in P or dS
        auto chunk = [&](bool ds, int c) {
            return smem + C::offP + C::block(ds, c >> 6) + (r >> 3) * 1024 + (r & 7) * 128 + ((((uint32_t)c >> 3 & 7u) ^ sw) << 4);
        };
        constexpr int NP = NC / 2;                                   // pairs of columns
        for (int n = 0; n < N; ++n) {
            const Tile t = run.tile(n);
            // visible columns: keys i - window + 1 .. i, and none before the head; a bit each
            const int hi = r + PAD - c0, first = max(r + PAD + 1 - p.window, PAD - t.i * kQT) - c0;
            uint32_t seen[(NC + 31) / 32];
#pragma unroll
            for (int b = 0; b < (NC + 31) / 32; ++b) {
                const int x = max(first - 32 * b, 0), y = min(hi - 32 * b, 31);
                seen[b] = x > y ? 0u : (0xffffffffu >> (31 - (y - x))) << x;
            }
            const bool all = __all_sync(0xffffffffu, first <= 0 && hi >= NC - 1);      // (of the whole warp's)
            float e[NC];
            ok = mbar_wait(&bars[bS], n & 1, abort_flag);
            __syncwarp();
            tc_fence_after();
#pragma unroll
            for (int b = 0; b < NC; b += 8) {
                uint32_t x[8];
                tmem_ld8(tx + b, x);
#pragma unroll
                for (int k = 0; k < 8; ++k) e[b + k] = __uint_as_float(x[k]);
            }
            tmem_wait_ld();
            tc_fence_before();
            mbar_arrive(&bars[bSread]);
            // (a branch: without it the compiler moves the loads' use about, and the case of 3 x 16 x 1777 takes 43 us, not 36)
            if (!all) {
#pragma unroll
                for (int k = 0; k < NC; ++k) e[k] = (seen[k >> 5] >> (k & 31)) & 1u ? e[k] : -INFINITY;
            }
            float mx = e[0];
#pragma unroll
            for (int k = 1; k < NC; ++k) mx = fmaxf(mx, e[k]);
            const float m0 = mx == -INFINITY ? 0.f : mx;             // (no key in this half)
            pairs::pair l2 = 0, ep[NP];
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                const float2 x = pairs::split(pairs::mul2(pairs::add2(pairs::make(e[2 * k], e[2 * k + 1]), pairs::both(-m0)), pairs::both(p.scale_log2e)));
                ep[k] = pairs::make(ex2(x.x), ex2(x.y));
                l2 = pairs::add2(l2, ep[k]);
            }
            ok = mbar_wait(&bars[bDP], n & 1, abort_flag) && ok;
            if (n > 0) ok = mbar_wait(&bars[bDone + ((n - 1) & 1)], ((n - 1) >> 1) & 1, abort_flag) && ok;
            __syncwarp();
            tc_fence_after();
            // dP: kept where there are registers for it, else read twice
            constexpr bool kKeep = NC <= 48;
            pairs::pair dp[kKeep ? NP : 1], w2 = 0;
#pragma unroll
            for (int b = 0; b < NC; b += 8) {
                uint32_t x[8];
                tmem_ld8(tx + b, x);
                if constexpr (!kKeep) tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const pairs::pair y = pairs::make(__uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1]));
                    if constexpr (kKeep) dp[b / 2 + k] = y;
                    else w2 = pairs::fma2(ep[b / 2 + k], y, w2);
                }
            }
            if constexpr (kKeep) {
                tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < NP; ++k) w2 = pairs::fma2(ep[k], dp[k], w2);
            }
            const float2 ls = pairs::split(l2), ws = pairs::split(w2);
            const float l = ls.x + ls.y, w = ws.x + ws.y;
            // the partner's statistics lie in the first chunk that this thread itself overwrites, and the other way round
            *reinterpret_cast<float4*>(chunk(false, c1)) = make_float4(mx, l, w, 0.f);
            ok = pair_all(1 + u, ok);
            if (!ok) break;
            const float4 other = *reinterpret_cast<const float4*>(chunk(false, c0));
            const float m = fmaxf(mx, other.x);                      // (finite: a row sees its own key)
            const float f0 = ex2((mx - m) * p.scale_log2e), f1 = ex2((other.x - m) * p.scale_log2e);
            const float inv = 1.f / fmaf(l, f0, other.y * f1);
            const float D = fmaf(w, f0, other.z * f1) * inv;
            const pairs::pair pf = pairs::both(f0 * inv), df = pairs::both(p.scale), nD = pairs::both(-D);
            auto packed = [](pairs::pair x) {
                const float2 f = pairs::split(x);
                return pack2(f.x, f.y);
            };
            // (the weights all at once or chunk by chunk, whichever the compiler's schedule is better with: PAD 64, 2 x 16 x 32768: 214 us
            // at once, 208 by chunks; PAD 128, 3 x 16 x 1777: 36 and 48)
            if constexpr (C::kShared) {
#pragma unroll
                for (int k = 0; k < NP; ++k) ep[k] = pairs::mul2(ep[k], pf);
            }
#pragma unroll
            for (int k = 0; k < NP; k += 4) {
                if constexpr (!C::kShared) {
#pragma unroll
                    for (int j = k; j < k + 4; ++j) ep[j] = pairs::mul2(ep[j], pf);
                    asm volatile("" ::: "memory");
                }
                *reinterpret_cast<uint4*>(chunk(false, c0 + 2 * k)) = make_uint4(packed(ep[k]), packed(ep[k + 1]), packed(ep[k + 2]), packed(ep[k + 3]));
            }
            if constexpr (C::kShared) {
                fence_proxy_async_smem();
                mbar_arrive(&bars[bP]);
            }
            uint32_t ds[NP];
#pragma unroll
            for (int b = 0; b < NP; b += 4) {
                uint32_t x[8];
                if constexpr (!kKeep) {
                    tmem_ld8(tx + 2 * b, x);
                    tmem_wait_ld();
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    pairs::pair y;
                    if constexpr (kKeep) y = dp[b + k];
                    else y = pairs::make(__uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1]));
                    ds[b + k] = packed(pairs::mul2(pairs::mul2(ep[b + k], df), pairs::add2(y, nD)));
                }
            }
            if constexpr (C::kShared) {                              // dS takes P's place
                ok = pair_all(1 + u, mbar_wait(&bars[bPdone], n & 1, abort_flag));
                if (!ok) break;
            }
#pragma unroll
            for (int k = 0; k < NP; k += 4) *reinterpret_cast<uint4*>(chunk(true, c0 + 2 * k)) = make_uint4(ds[k], ds[k + 1], ds[k + 2], ds[k + 3]);
            tc_fence_before();
            fence_proxy_async_smem();
            mbar_arrive(&bars[bPS]);
        }
    }

    if (!ok && lane == 0) atomicOr(p.err, 1u);
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        for (int it = 0; it < 200; ++it) __nanosleep(1000);
    }
    __syncthreads();
    if (warp == kWarpMma) tmem_dealloc(tb, 512);
}

template <int PAD>
static based_status launch_pad(const void* q, const void* k, const void* v, const void* dout, void* dq, void* dk, void* dv, int BH, int L,
                               int window, float scale, cudaStream_t stream) {
    using C = Cfg<PAD>;
    CUtensorMap tq, tk, tv, to, tdq, tdk, tdv;
    const CUtensorMapSwizzle s128 = CU_TENSOR_MAP_SWIZZLE_128B;
    if (!make_rows_map_bf16(&tq, q, BH, L, kHD, kHD, kQT, s128) || !make_rows_map_bf16(&tk, k, BH, L, kHD, kHD, 64, s128) ||
        !make_rows_map_bf16(&tv, v, BH, L, kHD, kHD, 64, s128) || !make_rows_map_bf16(&to, dout, BH, L, kHD, kHD, kQT, s128) ||
        !make_rows_map_bf16(&tdq, dq, BH, L, kHD, kHD, 32, s128) || !make_rows_map_bf16(&tdk, dk, BH, L, kHD, kHD, 32, s128) ||
        !make_rows_map_bf16(&tdv, dv, BH, L, kHD, kHD, 32, s128))
        return BASED_ERR_CUDA;
    Params p;
    if (error_word_ptr(&p.err) != BASED_OK) return BASED_ERR_CUDA;
    p.L = L;
    p.window = window;
    p.tiles_per_head = (int)(((long long)L + kQT - 1) / kQT);
    const long long total = (long long)p.tiles_per_head * BH;
    if (total > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    p.total_tiles = (int)total;
    p.scale = scale;
    p.scale_log2e = scale * 1.4426950408889634f;
    static std::atomic<int> sm_count[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return BASED_ERR_CUDA;
    int sms = sm_count[dev].load(std::memory_order_acquire);
    if (sms == 0) {
        if (cudaFuncSetAttribute(swa_backward_tc_kernel<PAD>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kSmemBytes) != cudaSuccess)
            return BASED_ERR_CUDA;
        if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms <= 0) sms = kSMs;
        sm_count[dev].store(sms, std::memory_order_release);
    }
    const int grid = p.total_tiles < sms ? p.total_tiles : sms;
    const cudaError_t e = launch_ex(swa_backward_tc_kernel<PAD>, dim3(grid), dim3(kThreads), C::kSmemBytes, 1, true, stream, tq, tk, tv, to, tdq, tdk, tdv, p);
    note_launch();
    const based_status st = check_launch("swa_backward_tc_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}

based_status launch_swa_backward_tc(const void* q, const void* k, const void* v, const void* dout, void* dq, void* dk, void* dv, int BH,
                                    int L, int window, float scale, cudaStream_t stream) {
    // (a query's first key lies window - 1 before it)
    if (window <= 65) return launch_pad<64>(q, k, v, dout, dq, dk, dv, BH, L, window, scale, stream);
    return launch_pad<128>(q, k, v, dout, dq, dk, dv, BH, L, window, scale, stream);
}

}  // namespace based
