// Decay attention with documents: each token's place in its block of tokens, once for all heads and passes.
//
// One CTA per block and sequence, a thread per token.  A block's first token that counts begins a document if the last token before
// it that counts is of another one: that is looked up backwards, 2048 tokens a turn, and only in blocks that hold tokens
// that count (behind a padded sequence's end nobody looks).
#include "decay.cuh"

namespace based {

namespace {

__global__ void __launch_bounds__(128) decay_places_kernel(const int* __restrict__ documents, uint32_t* __restrict__ places, int L, int T,
                                                           int blocks) {
    enter_dependent();
    const int b = blockIdx.x / blocks, n = blockIdx.x % blocks, t = n * T + threadIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int* ids = documents + (long long)b * L;
    __shared__ int s_last[4], s_any[4];
    const bool in = (int)threadIdx.x < T;
    const int id = in && t < L ? ids[t] : -1;
    const bool counts = id >= 0;
    // the token before this one that counts, in this block
    const uint32_t m = __ballot_sync(0xffffffffu, counts), below = m & ((1u << lane) - 1u);
    const int prev_lane = below ? 31 - __clz(below) : -1;
    int prev = __shfl_sync(0xffffffffu, id, prev_lane < 0 ? 0 : prev_lane);
    const int last = __shfl_sync(0xffffffffu, id, m ? 31 - __clz(m) : 0);
    if (lane == 0) {
        s_any[warp] = m != 0;
        s_last[warp] = last;
    }
    __syncthreads();
    bool known = prev_lane >= 0;
    for (int w = warp - 1; w >= 0 && !known; --w)
        if (s_any[w]) {
            known = true;
            prev = s_last[w];
        }
    const bool any = s_any[0] || s_any[1] || s_any[2] || s_any[3];
    __syncthreads();
    // before this block
    int before = -1;
    if (any) {
        for (int end = n * T; end > 0; end -= 2048) {
            int mine = -1, at = -1;
            for (int k = 0; k < 16; ++k) {
                const int p = end - 2048 + k * 128 + (int)threadIdx.x;
                if (p >= 0) {
                    const int x = ids[p];
                    if (x >= 0) { mine = x; at = p; }
                }
            }
            const int far = __reduce_max_sync(0xffffffffu, at);
            const uint32_t who = __ballot_sync(0xffffffffu, at == far && at >= 0);
            const int x = __shfl_sync(0xffffffffu, mine, who ? __ffs(who) - 1 : 0);
            if (lane == 0) {
                s_any[warp] = far;
                s_last[warp] = x;
            }
            __syncthreads();
            int best = -1;
            for (int w = 0; w < 4; ++w)
                if (s_any[w] > best) {
                    best = s_any[w];
                    before = s_last[w];
                }
            __syncthreads();
            if (best >= 0) break;
            before = -1;
        }
    }
    if (!known) prev = before;                         // (-1: nothing before it counts, and the state given goes on)
    const bool begins = counts && prev >= 0 && prev != id;
    const uint32_t mb = __ballot_sync(0xffffffffu, begins), upto = 0xffffffffu >> (31 - lane);
    __shared__ uint32_t s_counts[4], s_begins[4];
    if (lane == 0) {
        s_counts[warp] = m;
        s_begins[warp] = mb;
    }
    __syncthreads();
    int count = __popc(m & upto), run = __popc(mb & upto), first = 128, last_one = -1, all = 0;
    for (int w = 0; w < 4; ++w) {
        if (w < warp) {
            count += __popc(s_counts[w]);
            run += __popc(s_begins[w]);
        }
        all += __popc(s_counts[w]);
        if (s_counts[w]) {
            first = min(first, 32 * w + __ffs(s_counts[w]) - 1);
            last_one = 32 * w + 31 - __clz(s_counts[w]);
        }
    }
    // this token's document: from the last beginning up to it (or the block's first token that counts) to the token that counts ahead of the
    // next beginning (or the last one)
    int from = first, to = last_one;
    const uint32_t mine = mb & upto, after = mb & ~upto;
    if (mine) {
        from = 32 * warp + 31 - __clz(mine);
    } else {
        for (int w = warp - 1; w >= 0; --w)
            if (s_begins[w]) {
                from = 32 * w + 31 - __clz(s_begins[w]);
                break;
            }
    }
    int next = after ? 32 * warp + __ffs(after) - 1 : 128;
    for (int w = warp + 1; w < 4 && next == 128; ++w)
        if (s_begins[w]) next = 32 * w + __ffs(s_begins[w]) - 1;
    if (next < 128) {                                  // (with padding ahead of it, a token that does not count: no matter)
        to = next - 1;
    }
    const bool compact = all == last_one - first + 1;
    if (in)
        places[((long long)b * blocks + n) * T + threadIdx.x] = (uint32_t)count | (uint32_t)run << 8 | (uint32_t)(from & 127) << 16 |
                                                                 (uint32_t)(to & 127) << 23 | (compact ? kCompact : 0u) | (counts ? 0u : kPadding);
}

}  // namespace

based_status launch_decay_places(const int* documents, uint32_t* places, int B, int L, int T, cudaStream_t stream) {
    const int blocks = (L + T - 1) / T;
    const cudaError_t e = launch_ex(decay_places_kernel, dim3((unsigned)((long long)B * blocks)), dim3(128), 0, 1, true, stream, documents, places, L,
                                    T, blocks);
    note_launch();
    const based_status st = check_launch("decay_places_kernel");
    return e == cudaSuccess ? st : BASED_ERR_CUDA;
}

DecayPlan decay_plan(int passes, int max_de, int B, int H, int L, bool documents, int T, int width, int slots, DecayCosts costs) {
    DecayPlan p{};
    p.T = T;
    p.width = width;
    p.blocks = (int)(((long long)L + T - 1) / T);
    p.tiles = (max_de + width - 1) / width;
    const long long items = (long long)passes * p.tiles * B * H;
    // Time in blocks of a CTA: all segments of all items in turns; ahead of them the states of all but the last segments, a launch and the
    // segments' states that each has to add up
    p.segments = 1;
    for (int n = 1; n <= p.blocks && n <= 64 && (n == 1 || items * n <= 4ll * slots); ++n) {
        auto turns = [&](long long ctas) { return (double)((ctas + slots - 1) / slots); };
        const double each = (double)((p.blocks + n - 1) / n) * costs.block;
        const double time = turns(items * n) * each + (n == 1 ? 0 : costs.states * turns(items * (n - 1)) * each + costs.launch + costs.sum * n);
        if (n == 1 || time < p.time) {
            p.time = time;
            p.segments = n;
        }
    }
    p.ctas = items * p.segments;
    p.places_bytes = documents ? (size_t)B * p.blocks * T * sizeof(uint32_t) : 0;
    const size_t kept = (size_t)(items * (p.segments - 1));
    p.states_bytes = kept * kDecayMaxWidth * width * sizeof(float);
    p.factors_bytes = (kept * sizeof(float) + 255) / 256 * 256;
    return p;
}

}  // namespace based
