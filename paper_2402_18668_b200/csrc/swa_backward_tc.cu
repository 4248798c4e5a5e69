// swa_backward, bf16 tensor-core path (tcgen05 + TMEM + TMA), one kernel, every input read once:
//
//   P_ij = exp(c (s_ij - m_i)) / l_i,  D_i = sum_j P_ij dP_ij,  dS_ij = c P_ij (dP_ij - D_i)        (s = Q K^T, dP = dO V^T)
//   dQ_i = sum_j dS_ij k_j,   dK_j = sum_i dS_ij q_i,   dV_j = sum_i P_ij dO_i
//
// Persistent CTAs (one per SM) walk contiguous runs of tiles of 128 queries.  The tile at i0 sees the keys from i0 - PAD on
// (PAD = 64 for windows up to 65, else 128): 128 + PAD columns.  Per tile
//   S, then dP   [128, 128 + PAD] into the same TMEM columns, 64 keys at a time
//   softmax      two threads per query row, each with half of the 32 + PAD columns its warp's rows can touch; the statistics
//                m, l, sum P dP join through shared memory; P and dS go to shared memory as bf16
//   dQ           dS K, dS read with the queries as rows
//   dK, dV       dS^T Q, P^T dO, the same bytes read with the keys as rows
// Key blocks of 128 are shifted by PAD against the query tiles, so that block b = keys 128 b - PAD .. 128 b - PAD + 127 meets
// query tiles b - 1 and b alone: tile b - 1 starts its accumulators and tile b completes them.  They stay in TMEM (two sets)
// and no gradient is added into memory.  A run that starts inside a head first recomputes the tile before it, for the
// block that it completes next.
//
// Shared memory (227 KB, which is why there is one CTA per SM): a ring of 64-key halves of K and V, of which two are the next
// tile's; two slots of Q and dO; P and dS.  Rows of warp u (32 of them) touch columns 32 u .. 32 u + 31 + PAD only, what lies outside
// is zeroed once and never written.  With PAD 64, P and dS have 40 KB each: column blocks 1 and 0 of 64 by all 128 rows, then the
// lower half of block 2; the zeros that stand for its upper half (as rows, in dQ) and for the missing block 3 (as columns, in
// dK and dV) are block 0's lower half, which lies where either view looks for them.  With PAD 128, P and dS take turns in one array of
// 64 KB.
//
// Work per tile at PAD 64: five products of 128 x 192 x 64 (and the zeros: 2200 cycles of the tensor pipe) and 7 x 16 KB of HBM
// traffic (2.6 us of an SM's share): bound by HBM where the chain load - S - softmax - dP - products - store of a tile
// overlaps its neighbours'.  S of the next tile is issued ahead of this one's gradients, four warps of their own write results out.
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
    static constexpr int kSlots = PAD == 64 ? 5 : 6;                 // of the ring
    static constexpr int kCols = (32 + PAD) / 2;                     // columns per softmax thread: 48 or 80
    static constexpr bool kShared = PAD == 128;                      // P and dS in one array
    static constexpr uint32_t offQ = kSlots * 2 * kHalfBytes;        // two slots of Q and dO
    static constexpr uint32_t offP = offQ + 4 * kTileBytes;
    static constexpr uint32_t kPBytes = PAD == 64 ? 40960 : 65536;
    static constexpr uint32_t offD = kShared ? offP : offP + kPBytes;
    static constexpr uint32_t offBars = offD + kPBytes;
    static constexpr uint32_t kSmemBytes = offBars + 256 + 1024;
    static_assert(kSmemBytes <= 232448, "shared memory budget");
    // byte offset of row 0 of the block of 64 columns cb in P or dS (PAD 64, block 2: its rows 0 .. 63 are block 0's 64 .. 127)
    static __host__ __device__ constexpr uint32_t block(int cb) {
        return PAD == 64 ? (cb == 1 ? 0u : cb == 0 ? 16384u : 24576u) : (cb == 1 ? 0u : cb == 0 ? 16384u : cb == 3 ? 32768u : 49152u);
    }
};
// TMEM columns: scores (and dP after them), dQ, two sets of (dK, dV)
constexpr uint32_t colX = 0, colAcc = 256;
template <int PAD> constexpr uint32_t colDQ = PAD == 64 ? 192 : 0;   // PAD 128: over dP once that is read

enum Bar {
    bFullQ = 0, bFullO = 2, bEmptyO = 4, bFullKV = 6, bEmptyKV = 12, bS = 18, bSread, bDP, bP, bPdone, bPS, bDone, bDQfree, bAccFree,
    bCount = bAccFree + 2
};
static_assert(bCount * 8 + 8 <= 256, "barrier area");

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

__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(r)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return r != 0;
}
// 32 rows of 32 fp32 values in TMEM (a row per lane) to bf16 rows of 64 bytes in shared memory, swizzled as the TMA store reads them
__device__ __forceinline__ void stage_rows(uint32_t taddr, uint8_t* tile, int lane) {
    uint32_t t[32];
    tmem_ld32(taddr, t);
    tmem_wait_ld();
    uint8_t* row = tile + lane * 64;
    const uint32_t sw = (lane >> 1) & 3;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = pack2(__uint_as_float(t[8 * j + 2 * k]), __uint_as_float(t[8 * j + 2 * k + 1]));
        *reinterpret_cast<uint4*>(row + (((uint32_t)j ^ sw) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

}  // namespace

template <int PAD>
__global__ void __launch_bounds__(kThreads, 1)
    swa_backward_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                           const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_o,
                           const __grid_constant__ CUtensorMap tm_dq, const __grid_constant__ CUtensorMap tm_dk,
                           const __grid_constant__ CUtensorMap tm_dv, const Params p) {
    using C = Cfg<PAD>;
    constexpr int NH = C::kHalves, NS = C::kSlots, NC = C::kCols;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::offBars);
    uint32_t* tmem_base_s = reinterpret_cast<uint32_t*>(bars + bCount);
    volatile uint32_t* abort_flag = tmem_base_s + 1;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Run run(p);
    const int N = run.count;

    if (tid == 0) {
        for (int s = 0; s < 2; ++s) {
            mbar_init(&bars[bFullQ + s], 1); mbar_init(&bars[bFullO + s], 1); mbar_init(&bars[bEmptyO + s], 4);
            mbar_init(&bars[bAccFree + s], 128);
        }
        for (int s = 0; s < NS; ++s) { mbar_init(&bars[bFullKV + s], 1); mbar_init(&bars[bEmptyKV + s], 1); }
        mbar_init(&bars[bS], 1); mbar_init(&bars[bSread], 256); mbar_init(&bars[bDP], 1);
        mbar_init(&bars[bP], 256); mbar_init(&bars[bPdone], 1); mbar_init(&bars[bPS], 256);
        mbar_init(&bars[bDone], 1); mbar_init(&bars[bDQfree], 128);
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
            int hc = 0;                                              // halves loaded so far
            for (int n = 0; n < N && ok; ++n) {
                const Tile t = run.tile(n);
                const bool fresh = n == 0 || t.first;                // all halves are new, else the last two
                for (int j = fresh ? 0 : NH - 2; j < NH && ok; ++j, ++hc) {
                    const int s = hc % NS;
                    ok = mbar_wait(&bars[bEmptyKV + s], ((hc / NS) & 1) ^ 1, abort_flag);
                    if (!ok) break;
                    uint8_t* st = smem + s * 2 * kHalfBytes;
                    const int key = t.i * kQT - PAD + 64 * j;        // (rows outside the head read as zeros)
                    mbar_arrive_expect_tx(&bars[bFullKV + s], 2 * kHalfBytes);
                    tma_load_3d(st, &tm_k, &bars[bFullKV + s], 0, key, t.head);
                    tma_load_3d(st + kHalfBytes, &tm_v, &bars[bFullKV + s], 0, key, t.head);
                }
                if (!ok) break;
                // Q goes where the tile before last had it, once that tile's products are done; dO once its results are out, too
                const int s = n & 1;
                if (n >= 2) ok = mbar_wait(&bars[bDone], (n - 2) & 1, abort_flag);
                if (!ok) break;
                uint8_t* st = smem + C::offQ + s * 2 * kTileBytes;
                mbar_arrive_expect_tx(&bars[bFullQ + s], kTileBytes);
                tma_load_3d(st, &tm_q, &bars[bFullQ + s], 0, t.i * kQT, t.head);
                ok = mbar_wait(&bars[bEmptyO + s], ((n >> 1) & 1) ^ 1, abort_flag);
                if (!ok) break;
                mbar_arrive_expect_tx(&bars[bFullO + s], kTileBytes);
                tma_load_3d(st + kTileBytes, &tm_o, &bars[bFullO + s], 0, t.i * kQT, t.head);
            }
        }
    } else if (warp == kWarpMma) {
        // the whole warp runs this block and one elected lane issues (see mma_ss_w)
        const uint32_t lead = elect_one();
        constexpr uint64_t d1 = make_smem_desc_base(16, 1024, kSwizzle128B);              // K-major rows, or one MN-major block of 64
        constexpr uint64_t dA = make_smem_desc_base(16384, 1024, kSwizzle128B);           // MN-major, blocks 1 and 0 (3 and 2)
        constexpr uint64_t dB = make_smem_desc_base(PAD == 64 ? 8192 : 16384, 1024, kSwizzle128B);   // zeros and block 2 (blocks 3, 2)
        constexpr uint32_t iS = make_idesc_bf16(128, 64, 0, 0), iQ = make_idesc_bf16(128, 64, 0, 1), iK = make_idesc_bf16(128, 64, 1, 1);
        const uint32_t sm = smem_u32(smem);
        auto lo = [](uint64_t base, uint32_t addr) { return desc_lo(base) + (addr >> 4); };
        int hb = 0;                                                  // the tile's first half, counted as they are loaded
        int acc = 0, uses[2] = {0, 0};                               // the set its key block is in; times a set was begun
        auto kv = [&](int j) { return sm + ((hb + j) % NS) * 2 * kHalfBytes; };
        auto qo = [&](int n) { return sm + C::offQ + (n & 1) * 2 * kTileBytes; };
        // scores or dP: rows of `a` (Q or dO) by the halves of K or V, `off` bytes into a half's slot
        auto scores = [&](uint32_t a, uint32_t off) {
            const uint32_t la = lo(d1, a);
            for (int j = 0; j < NH; ++j) {
                const uint32_t lb = lo(d1, kv(j) + off), d = tb + colX + 64 * j;
                mma_ss_w<false>(lead, d, la, desc_hi(d1), lb, desc_hi(d1), iS);
#pragma unroll
                for (int k = 1; k < 4; ++k) mma_ss_w<true>(lead, d, la + k * 2, desc_hi(d1), lb + k * 2, desc_hi(d1), iS);
            }
        };
        auto issue_s = [&](int n) -> bool {
            if (!mbar_wait(&bars[bFullQ + (n & 1)], (n >> 1) & 1, abort_flag)) return false;
            for (int j = 0; j < NH; ++j)
                if (!mbar_wait(&bars[bFullKV + (hb + j) % NS], ((hb + j) / NS) & 1, abort_flag)) return false;
            if (PAD == 128 && n > 0)                                 // dQ of the tile before lies over the scores
                if (!mbar_wait(&bars[bDQfree], (n - 1) & 1, abort_flag)) return false;
            tc_fence_after();
            scores(qo(n), 0);
            mma_commit_w(lead, &bars[bS]);
            return true;
        };
        // X^T Y of the tile's key block A (completing its accumulators) and of block B (starting the next one's)
        auto block_a = [&](uint32_t x, uint32_t y, uint32_t d, bool begin) {
            const uint32_t lx = lo(dA, x), ly = lo(d1, y);
            if (begin) mma_ss_w<false>(lead, d, lx, desc_hi(dA), ly, desc_hi(d1), iK);
            else mma_ss_w<true>(lead, d, lx, desc_hi(dA), ly, desc_hi(d1), iK);
#pragma unroll
            for (int k = 1; k < 8; ++k) mma_ss_w<true>(lead, d, lx + k * 128, desc_hi(dA), ly + k * 128, desc_hi(d1), iK);
        };
        auto block_b = [&](uint32_t x, uint32_t y, uint32_t d) {
            // (PAD 64: only rows 64 .. 127 see block 2; block(2) is where their zeros lie)
            constexpr int k0 = PAD == 64 ? 4 : 0;
            const uint32_t lx = lo(dB, x + C::block(PAD == 64 ? 2 : 3)), ly = lo(d1, y) + k0 * 128;
            mma_ss_w<false>(lead, d, lx, desc_hi(dB), ly, desc_hi(d1), iK);
#pragma unroll
            for (int k = 1; k < 8 - k0; ++k) mma_ss_w<true>(lead, d, lx + k * 128, desc_hi(dB), ly + k * 128, desc_hi(d1), iK);
        };
        auto acc_col = [&](int a, int which) { return tb + colAcc + 128 * a + 64 * which; };     // 0: dK, 1: dV
        auto free_acc = [&](int a) { return uses[a] == 0 || mbar_wait(&bars[bAccFree + a], (uses[a] - 1) & 1, abort_flag); };
        auto issue_dp = [&](int n) -> bool {
            if (!mbar_wait(&bars[bSread], n & 1, abort_flag) || !mbar_wait(&bars[bFullO + (n & 1)], (n >> 1) & 1, abort_flag)) return false;
            tc_fence_after();
            scores(qo(n) + kTileBytes, kHalfBytes);
            mma_commit_w(lead, &bars[bDP]);
            return true;
        };
        bool dp_asked = false;
        ok = issue_s(0);
#pragma unroll 1
        for (int n = 0; n < N && ok; ++n) {
            const Tile t = run.tile(n);
            const bool with_b = !t.end || t.last;                    // the next block is this run's too
            const bool early = PAD == 64 && !t.end && !t.last;       // (a new head's halves wait for this tile's slots)
            const int drop = t.last ? NH : 2;                        // halves that the next tile does not use
            const uint32_t sQ = qo(n), sO = sQ + kTileBytes, sP = sm + C::offP, sD = sm + C::offD;
            auto begin_sets = [&]() -> bool {                        // the sets that this tile's products begin must have been read
                if (!t.halo && t.first && !free_acc(acc)) return false;
                return !with_b || free_acc(acc ^ 1);
            };
            // dV, or dV and dK
            auto products = [&](int from, int to) {
#pragma unroll 1
                for (int which = from; which >= to; --which) {
                    const uint32_t x = which ? sP : sD, y = which ? sO : sQ;
                    if (!t.halo) block_a(x, y, acc_col(acc, which), t.first);
                    if (with_b) block_b(x, y, acc_col(acc ^ 1, which));
                }
            };
            if (!dp_asked) ok = issue_dp(n);
            if (!ok) break;
            if constexpr (C::kShared) {
                ok = mbar_wait(&bars[bP], n & 1, abort_flag) && begin_sets();
                if (!ok) break;
                tc_fence_after();
                products(1, 1);
                mma_commit_w(lead, &bars[bPdone]);
            }
            ok = mbar_wait(&bars[bPS], n & 1, abort_flag);
            if (!ok) break;
            tc_fence_after();
            if (early) {
                hb += drop;
                ok = issue_s(n + 1);
                hb -= drop;
            }
            // (also what keeps a tile's end from being told before the end of the tile before it was seen)
            if (ok && n > 0) ok = mbar_wait(&bars[bDQfree], (n - 1) & 1, abort_flag);
            if (!ok) break;
            tc_fence_after();
            if (!t.halo) {
                const uint32_t d = tb + colDQ<PAD>;
#pragma unroll
                for (int j = 0; j < NH; ++j) {
                    const uint32_t la = lo(d1, sD + C::block(j)), lb = lo(d1, kv(j));
                    if (j == 0) mma_ss_w<false>(lead, d, la, desc_hi(d1), lb, desc_hi(d1), iQ);
                    else mma_ss_w<true>(lead, d, la, desc_hi(d1), lb, desc_hi(d1), iQ);
#pragma unroll
                    for (int k = 1; k < 4; ++k) mma_ss_w<true>(lead, d, la + k * 2, desc_hi(d1), lb + k * 128, desc_hi(d1), iQ);
                }
            }
            for (int j = 0; j < drop; ++j) mma_commit_w(lead, &bars[bEmptyKV + (hb + j) % NS]);
            hb += drop;
            // the next tile's dP goes ahead of this one's products where its dO is there: its softmax waits for it, nothing of this tile does
            dp_asked = early && __all_sync(0xffffffffu, mbar_test(&bars[bFullO + ((n + 1) & 1)], ((n + 1) >> 1) & 1));
            if (dp_asked) ok = issue_dp(n + 1);
            if constexpr (!C::kShared) ok = ok && begin_sets();
            if (!ok) break;
            tc_fence_after();
            products(C::kShared ? 0 : 1, 0);
            mma_commit_w(lead, &bars[bDone]);
            if (!t.halo && t.first) ++uses[acc];
            if (with_b) ++uses[acc ^ 1];
            if (!t.last) acc ^= 1;
            if (!early && !t.end) ok = issue_s(n + 1);
        }
    } else if (warp >= kWarpOut) {
        // ---- results: four warps, a TMEM lane per thread.  Once a tile's products are done, the place of its dO holds the results on
        // their way out (per warp two pieces of 32 rows by 32 columns in turn); then it goes back to the loads.  (Stores from registers
        // crowd out the softmax's accesses to shared memory, whose pipe they share.)
        const int u = warp & 3;
        const uint32_t lanes = (uint32_t)u * 32u;
        int acc = 0;
        for (int n = 0; n < N && ok; ++n) {
            const Tile t = run.tile(n);
            ok = __all_sync(0xffffffffu, mbar_wait(&bars[bDone], n & 1, abort_flag));
            if (!ok) break;
            tc_fence_after();
            if (t.halo) mbar_arrive(&bars[bDQfree]);
            uint8_t* own = smem + C::offQ + (n & 1) * 2 * kTileBytes + kTileBytes + u * 4096;
            // dQ; dK, dV of the key block that this tile completes (lanes 0 .. 63 hold its keys 64 .. 127 and the other way round); of
            // the one behind a head's last tile
            const int from = t.halo ? 10 : 0, to = t.halo || !t.last ? 6 : 10;
#pragma unroll 1
            for (int q = from; q < to; ++q) {
                const int k = q >> 1, col = (q & 1) * 32, a = k < 3 ? acc : acc ^ 1;
                const bool value = k == 2 || k == 4;
                uint8_t* tile = own + (q & 1) * 2048;
                if (q > 1) {                                         // (the store before last has read its rows)
                    if (lane == 0) tma_store_wait_read<1>();
                    __syncwarp();
                }
                stage_rows(tmem_addr(tb, lanes, (k == 0 ? colDQ<PAD> : colAcc + 128 * a + 64 * value) + col), tile, lane);
                tc_fence_before();
                if (q == 1) mbar_arrive(&bars[bDQfree]);
                else if (value && (q & 1)) mbar_arrive(&bars[bAccFree + a]);
                fence_proxy_async_smem();
                __syncwarp();
                const int row = k == 0 ? t.i * kQT + (int)lanes : (k < 3 ? t.i : t.i + 1) * kQT - PAD + (int)(lanes ^ 64u);
                if (lane == 0) {
                    if (row >= 0 && row < p.L) tma_store_3d(k == 0 ? &tm_dq : value ? &tm_dv : &tm_dk, tile, col, row, t.head);
                    tma_store_commit();
                }
            }
            if (lane == 0) {
                tma_store_wait_read<0>();
                mbar_arrive(&bars[bEmptyO + (n & 1)]);
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
        auto chunk = [&](uint32_t off, int c) {
            return smem + off + C::block(c >> 6) + (r >> 3) * 1024 + (r & 7) * 128 + ((((uint32_t)c >> 3 & 7u) ^ sw) << 4);
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
            float e[NC];
            ok = mbar_wait(&bars[bS], n & 1, abort_flag);
            __syncwarp();
            tc_fence_after();
#pragma unroll
            for (int b = 0; b < NC; b += 16) {
                uint32_t x[16];
                tmem_ld16(tx + b, x);
#pragma unroll
                for (int k = 0; k < 16; ++k) e[b + k] = __uint_as_float(x[k]);
            }
            tmem_wait_ld();
            tc_fence_before();
            mbar_arrive(&bars[bSread]);
            float mx = -INFINITY;
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                e[k] = (seen[k >> 5] >> (k & 31)) & 1u ? e[k] : -INFINITY;
                mx = fmaxf(mx, e[k]);
            }
            const float m0 = mx == -INFINITY ? 0.f : mx;             // (no key in this half)
            pairs::pair l2 = 0, ep[NP];
#pragma unroll
            for (int k = 0; k < NP; ++k) {
                const float2 x = pairs::split(pairs::mul2(pairs::add2(pairs::make(e[2 * k], e[2 * k + 1]), pairs::both(-m0)), pairs::both(p.scale_log2e)));
                ep[k] = pairs::make(ex2(x.x), ex2(x.y));
                l2 = pairs::add2(l2, ep[k]);
            }
            ok = mbar_wait(&bars[bDP], n & 1, abort_flag) && ok;
            if (n > 0) ok = mbar_wait(&bars[bDone], (n - 1) & 1, abort_flag) && ok;
            __syncwarp();
            tc_fence_after();
            // dP: kept where there are registers for it, else read twice
            constexpr bool kKeep = NC <= 48;
            pairs::pair dp[kKeep ? NP : 1], w2 = 0;
#pragma unroll
            for (int b = 0; b < NC; b += 16) {
                uint32_t x[16];
                tmem_ld16(tx + b, x);
                if constexpr (!kKeep) tmem_wait_ld();
#pragma unroll
                for (int k = 0; k < 8; ++k) {
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
            *reinterpret_cast<float4*>(chunk(C::offP, c1)) = make_float4(mx, l, w, 0.f);
            ok = pair_all(1 + u, ok);
            if (!ok) break;
            const float4 other = *reinterpret_cast<const float4*>(chunk(C::offP, c0));
            const float m = fmaxf(mx, other.x);                      // (finite: a row sees its own key)
            const float f0 = ex2((mx - m) * p.scale_log2e), f1 = ex2((other.x - m) * p.scale_log2e);
            const float inv = 1.f / fmaf(l, f0, other.y * f1);
            const float D = fmaf(w, f0, other.z * f1) * inv;
            const pairs::pair pf = pairs::both(f0 * inv), df = pairs::both(p.scale), nD = pairs::both(-D);
            auto packed = [](pairs::pair x) {
                const float2 f = pairs::split(x);
                return pack2(f.x, f.y);
            };
#pragma unroll
            for (int k = 0; k < NP; ++k) ep[k] = pairs::mul2(ep[k], pf);
            if constexpr (C::kShared) {
#pragma unroll
                for (int k = 0; k < NP; k += 4)
                    *reinterpret_cast<uint4*>(chunk(C::offP, c0 + 2 * k)) = make_uint4(packed(ep[k]), packed(ep[k + 1]), packed(ep[k + 2]), packed(ep[k + 3]));
                fence_proxy_async_smem();
                mbar_arrive(&bars[bP]);
                ok = pair_all(1 + u, mbar_wait(&bars[bPdone], n & 1, abort_flag));
                if (!ok) break;
            }
#pragma unroll
            for (int b = 0; b < NP; b += 8) {
                uint32_t x[16];
                if constexpr (!kKeep) {
                    tmem_ld16(tx + 2 * b, x);
                    tmem_wait_ld();
                }
#pragma unroll
                for (int g = 0; g < 8; g += 4) {
                    uint32_t ds[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        pairs::pair y;
                        if constexpr (kKeep) y = dp[b + g + k];
                        else y = pairs::make(__uint_as_float(x[2 * (g + k)]), __uint_as_float(x[2 * (g + k) + 1]));
                        ds[k] = packed(pairs::mul2(pairs::mul2(ep[b + g + k], df), pairs::add2(y, nD)));
                    }
                    const int c = c0 + 2 * (b + g);
                    if constexpr (!C::kShared)
                        *reinterpret_cast<uint4*>(chunk(C::offP, c)) =
                            make_uint4(packed(ep[b + g]), packed(ep[b + g + 1]), packed(ep[b + g + 2]), packed(ep[b + g + 3]));
                    *reinterpret_cast<uint4*>(chunk(C::offD, c)) = make_uint4(ds[0], ds[1], ds[2], ds[3]);
                }
            }
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
    const CUtensorMapSwizzle s128 = CU_TENSOR_MAP_SWIZZLE_128B, s64 = CU_TENSOR_MAP_SWIZZLE_64B;
    if (!make_rows_map_bf16(&tq, q, BH, L, kHD, kHD, kQT, s128) || !make_rows_map_bf16(&tk, k, BH, L, kHD, kHD, 64, s128) ||
        !make_rows_map_bf16(&tv, v, BH, L, kHD, kHD, 64, s128) || !make_rows_map_bf16(&to, dout, BH, L, kHD, kHD, kQT, s128) ||
        !make_rows_map_bf16(&tdq, dq, BH, L, kHD, 32, 32, s64) || !make_rows_map_bf16(&tdk, dk, BH, L, kHD, 32, 32, s64) ||
        !make_rows_map_bf16(&tdv, dv, BH, L, kHD, 32, 32, s64))
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
