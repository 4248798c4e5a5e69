// Linear attention with a decay per head: what the passes share.  One form serves the forward pass and the three gradients.
// With a = exp(-rate) and c_t the tokens up to t that count (documents >= 0), over the tokens of one document,
//
//   o_t = factor sum_{j <= t} a^(c_t - c_j) (x_t . y_j) z_j            (back: over j >= t, a^(c_j - c_t))
//
//   forward  x = q,  y = k,  z = v          dq  x = dout, y = v,    z = k
//   dk       x = v,  y = dout, z = q, back  dv  x = k,    y = q,    z = dout, back
//
// computed block by block of tokens: the pairs inside a block as products masked and faded one by one, everything before (behind)
// it through the state S = sum a^.. y z^T, [dc, de] fp32:
//   out      sum over the block + a^(steps from the block's border to t) x_t S
//   state    S <- a^(the block's tokens) S + sum_j a^(steps from j to the block's other border) y_j z_j^T
// With documents the border's terms hold for the tokens of the document that reaches over it, and the state passes a block
// only if one document does.
#pragma once
#include "common.cuh"

namespace based {

constexpr int kDecayMaxWidth = 128;        // d_k, d_v at most

// one pass: x, y [B,H,L,dc], z, out [B,H,L,de]
struct DecayPass {
    based_heads x, y, z, out;
    int dc, de;
    // the states before the first token (back: behind the last) and behind the last (before the first), [B,H,dc,de], or [B,H,de,dc]
    // (turned); null: zeros, not wanted.  What is read is multiplied by in_factor, what is written by out_factor.
    const float* state_in;
    float* state_out;
    int turned, back;
    float in_factor, out_factor;
};
struct DecayCall {
    DecayPass pass[3];
    int passes;
    const float* rate;                     // [H]
    const int* documents;                  // [B,L] or null
    int B, H, L;
    float factor;                          // of the outputs
};

// A token's place in its block of kT tokens: bits 0-7 how many tokens up to it count, bits 8-15 how many documents have begun up to it
// (0: the one that reaches over the block's border), bits 16-22 and 23-29 the first and the last token of its document in the
// block, bit 30: no padding lies between the block's tokens that count, bit 31: it is padding.  Past the sequence: padding.
constexpr uint32_t kPadding = 0x80000000u, kCompact = 0x40000000u;
__device__ __forceinline__ int place_count(uint32_t w) { return (int)(w & 255u); }
__device__ __forceinline__ int place_run(uint32_t w) { return (int)(w >> 8 & 255u); }
__device__ __forceinline__ int place_from(uint32_t w) { return (int)(w >> 16 & 127u); }
__device__ __forceinline__ int place_to(uint32_t w) { return (int)(w >> 23 & 127u); }

// exp(-rate n) for a rate held as rate log2(e); n = 0 gives 1 whatever the rate
__device__ __forceinline__ float faded(float rate2, int n) { return n == 0 ? 1.f : exp2f(-rate2 * (float)n); }
// (finite: an infinite rate, or one that is after the product, fades all within a token either way.  NaN stays NaN, and shows in all that it fades)
__device__ __forceinline__ float rate_of(float rate) {
    const float rate2 = rate * 1.4426950408889634f;
    return rate2 > 1e30f ? 1e30f : rate2;
}

// How a call is cut: every pass and head into tiles of `width` output columns, every one of those into segments of whole blocks of tokens.
// More than one segment: a launch ahead writes every segment's own state.
struct DecayPlan {
    int T, width;                          // tokens in a block, columns of z and of the output that a CTA works on
    int blocks, segments;                  // blocks of a sequence, segments they are cut into
    int tiles;                             // tiles of the widest pass
    long long ctas;                        // passes x tiles x segments x heads
    double time;                           // what the choice went by
    size_t places_bytes, states_bytes, factors_bytes;
    size_t bytes() const { return places_bytes + states_bytes + factors_bytes; }
};
// Times in blocks of width 64: a block's at this width, the share of it that its state alone takes, a launch, adding up one segment
struct DecayCosts { double block, states, launch, sum; };
// slots: CTAs that the device holds at a time
DecayPlan decay_plan(int passes, int max_de, int B, int H, int L, bool documents, int T, int width, int slots, DecayCosts costs);
// the first block of a segment
__host__ __device__ inline int decay_first(int blocks, int segments, int s) { return (int)((long long)blocks * s / segments); }

// what a CTA works on
struct DecayItem {
    int pass, tile, segment;               // the segment as the pass goes through them: back passes begin with the last one
    long long head;                        // b H + h
    __device__ __forceinline__ DecayItem(unsigned i, int passes, int tiles, int segments) {
        pass = (int)(i % (unsigned)passes); i /= (unsigned)passes;
        tile = (int)(i % (unsigned)tiles); i /= (unsigned)tiles;
        segment = (int)(i % (unsigned)segments);
        head = i / (unsigned)segments;
    }
};
// the segments' states and factors in the workspace, of all but the last: states [128][width] each
__host__ __device__ inline long long decay_slot(int pass, int passes, long long head, int tiles, int tile, int segments, int segment) {
    return ((head * passes + pass) * tiles + tile) * (segments - 1) + segment;
}

// places [B][blocks * T] of the tokens (decay_places.cu)
based_status launch_decay_places(const int* documents, uint32_t* places, int B, int L, int T, cudaStream_t stream);
// fp32 io on multiply-adds (decay_f32.cu), bf16 io on tensor cores (decay_tc.cu)
DecayPlan decay_plan_f32(const DecayCall& c);
based_status launch_decay_f32(const DecayCall& c, const DecayPlan& plan, void* workspace, cudaStream_t stream);
DecayPlan decay_plan_tc(const DecayCall& c);
based_status launch_decay_tc(const DecayCall& c, const DecayPlan& plan, void* workspace, cudaStream_t stream);
// one token (decay_step.cu): state [B,H,dk,dv] read, updated, written
based_status launch_decay_step(const void* q, const void* k, const void* v, const float* rate, const float* state_in, void* out,
                               float* state_out, long long BH, int H, int dk, int dv, float scale, based_dtype io, cudaStream_t stream);

constexpr int kDecayBlockF32 = 64, kDecayBlockTc = 128;

}  // namespace based
