// C ABI of libbased: argument validation and dispatch.  See include/based.h for the
// contract of every entry point.
#include <atomic>
#include <mutex>
#include <cmath>
#include <cstdio>
#include <initializer_list>
#include <new>
#include <vector>

#include "common.cuh"
#include "decay.cuh"
#include "paged.cuh"

namespace based {

__device__ unsigned int g_error_word = 0;

based_status error_word_ptr(unsigned int** ptr) {
    // the symbol has one instance per device: resolve it once per device, with that device current
    static std::atomic<unsigned int*> cache[64];
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return BASED_ERR_CUDA;
    unsigned int* p = cache[dev].load(std::memory_order_acquire);
    if (p == nullptr) {
        void* q = nullptr;
        if (cudaGetSymbolAddress(&q, g_error_word) != cudaSuccess) return BASED_ERR_CUDA;
        p = static_cast<unsigned int*>(q);
        cache[dev].store(p, std::memory_order_release);
    }
    *ptr = p;
    return BASED_OK;
}

std::mutex& setup_mutex() {
    static std::mutex mu;
    return mu;
}

static std::atomic<unsigned long long> g_launches{0};

void note_launch() { g_launches.fetch_add(1, std::memory_order_relaxed); }

based_status check_launch(const char* what) {
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) {
        std::fprintf(stderr, "libbased: launch of %s failed: %s\n", what, cudaGetErrorString(e));
        return BASED_ERR_CUDA;
    }
    return BASED_OK;
}

static inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// value head dimensions: 64 (360M-scale heads), 128, and 112 (the 1.3B configuration's 1792 / 16)
static inline bool dv_ok(int d_v) { return d_v == 64 || d_v == 112 || d_v == 128; }
// feature dimensions of the paper's ablation other than 16: served by the fp32 definition-form kernels
static inline bool df_generic(int d_feat) { return d_feat == 8 || d_feat == 24 || d_feat == 32; }

}  // namespace based

using namespace based;

// Several kernels index heads by the y dimension of the grid (at most 65535).  Larger batches are cut into
// slabs of heads here: every tensor is [B*H, ...] with the heads outermost, so a slab is a contiguous piece,
// and the slabs run one after another on the caller's stream (sharing the caller's workspace, which is sized
// for the largest slab).
constexpr long long kHeadSlab = 65532;      // a multiple of 4: a slab's K-state (an odd number of floats per head) stays 16-byte aligned
static inline const void* off(const void* p, size_t bytes) { return p ? static_cast<const char*>(p) + bytes : nullptr; }
static inline void* off(void* p, size_t bytes) { return p ? static_cast<char*>(p) + bytes : nullptr; }
static inline float* off(float* p, size_t floats) { return p ? p + floats : nullptr; }
static inline size_t esize(based_dtype io) { return io == BASED_BF16 ? 2 : 4; }

extern "C" {

int based_version(void) { return 1; }

unsigned long long based_launch_count(void) { return g_launches.load(std::memory_order_relaxed); }

const char* based_status_string(based_status s) {
    switch (s) {
        case BASED_OK: return "ok";
        case BASED_ERR_INVALID_ARG: return "invalid argument";
        case BASED_ERR_UNSUPPORTED: return "unsupported shape or dtype";
        case BASED_ERR_ALIGNMENT: return "pointer not 16-byte aligned";
        case BASED_ERR_CUDA: return "CUDA error";
        case BASED_ERR_DEVICE_TIMEOUT: return "bounded device-side wait timed out";
        case BASED_ERR_WORKSPACE: return "workspace missing or too small";
    }
    return "unknown status";
}

size_t based_prefill_workspace_bytes(int B, int H, int L, int d_feat, int d_v, based_dtype io) {
    if (B <= 0 || H <= 0 || L <= 0 || d_feat != kDFeat || !dv_ok(d_v)) return 0;
    if (io != BASED_BF16) return 0;            // the fp32 path keeps its states on chip
    const long long BH = (long long)B * H;
    if (BH > kHeadSlab) {
        const size_t a = prefill_tc_workspace_bytes((int)kHeadSlab, L, d_v);
        const size_t b = BH % kHeadSlab ? prefill_tc_workspace_bytes((int)(BH % kHeadSlab), L, d_v) : 0;
        return a > b ? a : b;
    }
    return prefill_tc_workspace_bytes(B * H, L, d_v);
}

size_t based_f32_parts_bytes(int B, int H, int L, int d_feat, int d_v, int backward) {
    if (B <= 0 || H <= 0 || L <= 0 || d_feat != kDFeat || !dv_ok(d_v)) return 0;
    const int heads = (long long)B * H > kHeadSlab ? (int)kHeadSlab : B * H;       // the largest slab of heads
    return quadratic_f32_workspace_bytes(heads, L, d_v, backward != 0);
}

static based_status prefill_impl(const void* q, const void* k, const void* v, void* out, float* kv_state, float* z_state,
                                 int B, int H, int L, int d_feat, int d_v, based_dtype io, int flags, void* workspace,
                                 size_t workspace_bytes, void* cuda_stream, bool fit) {
    if (!q || !k || !v || !out || B <= 0 || H <= 0 || L <= 0) return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if (flags & ~(BASED_STATE_CONTINUE | BASED_STATE_SYM | BASED_NUMERATOR_ONLY)) return BASED_ERR_INVALID_ARG;
    if ((kv_state == nullptr) != (z_state == nullptr)) return BASED_ERR_INVALID_ARG;
    if ((flags & BASED_STATE_CONTINUE) && !kv_state) return BASED_ERR_INVALID_ARG;
    if (out == q || out == k || out == v) return BASED_ERR_INVALID_ARG;
    if ((d_feat != kDFeat && !df_generic(d_feat)) || !dv_ok(d_v)) return BASED_ERR_UNSUPPORTED;
    if ((long long)B * H > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(kv_state) ||
        !aligned16(z_state) || !aligned16(workspace))
        return BASED_ERR_ALIGNMENT;
    if ((long long)B * H > kHeadSlab) {
        const size_t es = esize(io), rows = (flags & BASED_STATE_SYM) ? kDSym : 1 + d_feat + d_feat * d_feat;
        for (long long h0 = 0; h0 < (long long)B * H; h0 += kHeadSlab) {
            const int n = (int)((long long)B * H - h0 < kHeadSlab ? (long long)B * H - h0 : kHeadSlab);
            const based_status st = prefill_impl(
                off(q, (size_t)h0 * L * d_feat * es), off(k, (size_t)h0 * L * d_feat * es), off(v, (size_t)h0 * L * d_v * es),
                off(out, (size_t)h0 * L * d_v * es), off(kv_state, (size_t)h0 * rows * d_v), off(z_state, (size_t)h0 * rows),
                1, n, L, d_feat, d_v, io, flags, workspace, workspace_bytes, cuda_stream, fit);
            if (st != BASED_OK) return st;
        }
        return BASED_OK;
    }
    if (d_feat != kDFeat) {
        if (flags & BASED_STATE_SYM) return BASED_ERR_UNSUPPORTED;
        // bf16 io from the empty state: outputs (definition form) and state on the tensor cores, side by side
        if (io == BASED_BF16 && !(flags & BASED_STATE_CONTINUE)) {
            cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
            if (kv_state) {
                const based_status st = launch_state_generic_tc(k, v, kv_state, z_state, B * H, L, d_feat, d_v, 0, stream);
                if (st != BASED_OK) return st;
            }
            return launch_quadratic_forward_tc(q, k, v, out, B * H, L, d_feat, d_v, (flags & BASED_NUMERATOR_ONLY) ? 1 : 0,
                                               kv_state != nullptr, stream);
        }
        return launch_prefill_generic(q, k, v, out, kv_state, z_state, B * H, L, d_feat, d_v, io, flags,
                                      static_cast<cudaStream_t>(cuda_stream));
    }
    const size_t need = based_prefill_workspace_bytes(B, H, L, d_feat, d_v, io);
    if (!fit && need > 0 && (!workspace || workspace_bytes < need)) {
        // a few words for continued calls alone: others need none, and a continued call without them takes a plan without them
        if (need > BASED_WORDS_BYTES) return BASED_ERR_WORKSPACE;
        fit = true;
        if (!workspace) workspace_bytes = 0;
    }
    // One chunk and no state to write: the chunk's pairs are all there is, and the definition form's kernels, the same sums of the same
    // bf16 weights in the same order (the outputs are the bits that a call with a state gives), have less to set up (us, chunked / this: d_v 64, 16 heads L64 4.8 / 3.4, L128 5.7 / 3.8, 200 heads L64 10.6 / 4.0;
    // d_v 128, 16 heads L64 5.9 / 3.8, 400 heads L128 23 / 9).  Longer calls would be faster so up to L 1500 with 16 heads (L1024 10.2 /
    // 7.2), but the chunked form holds what is before the chunk more precisely (2.25e-3 against 2.29e-3 of 64-bit results).
    if (io == BASED_BF16 && !kv_state && L <= 128)
        return launch_quadratic_forward_tc(q, k, v, out, B * H, L, d_feat, d_v, (flags & BASED_NUMERATOR_ONLY) ? 1 : 0, false,
                                           static_cast<cudaStream_t>(cuda_stream));
    if (io == BASED_BF16)
        return launch_prefill_tc(q, k, v, out, kv_state, z_state, B * H, L, d_v, flags, workspace,
                                 static_cast<cudaStream_t>(cuda_stream), fit ? workspace_bytes : ~(size_t)0);
    return launch_prefill_f32(q, k, v, out, kv_state, z_state, B * H, L, d_v, flags,
                              static_cast<cudaStream_t>(cuda_stream));
}

based_status based_prefill(const void* q, const void* k, const void* v, void* out, float* kv_state, float* z_state,
                           int B, int H, int L, int d_feat, int d_v, based_dtype io, int flags, void* workspace,
                           size_t workspace_bytes, void* cuda_stream) {
    return prefill_impl(q, k, v, out, kv_state, z_state, B, H, L, d_feat, d_v, io, flags, workspace, workspace_bytes,
                        cuda_stream, false);
}

based_status based_prefill_f32_parts(const float* q, const float* k, const float* v, float* out, int B, int H, int L, int d_feat,
                                     int d_v, int flags, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!q || !k || !v || !out || B <= 0 || H <= 0 || L <= 0) return BASED_ERR_INVALID_ARG;
    if (flags & ~BASED_NUMERATOR_ONLY) return BASED_ERR_INVALID_ARG;
    if (out == q || out == k || out == v) return BASED_ERR_INVALID_ARG;
    const size_t need = based_f32_parts_bytes(B, H, L, d_feat, d_v, 0);
    if (need == 0 || (long long)B * H > kHeadSlab) return BASED_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(workspace)) return BASED_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < need) return BASED_ERR_WORKSPACE;
    return launch_quadratic_forward_f32(q, k, v, out, workspace, B * H, L, d_v, (flags & BASED_NUMERATOR_ONLY) ? 1 : 0,
                                        static_cast<cudaStream_t>(cuda_stream));
}

size_t based_prefill_state_workspace_bytes(int B, int H, int L, int d_feat, int d_v, based_dtype io) {
    if (B <= 0 || H <= 0 || L <= 0 || d_feat != kDFeat || !dv_ok(d_v) || io != BASED_BF16) return 0;
    if ((long long)B * H > kHeadSlab) return prefill_tc_state_workspace_bytes((int)kHeadSlab, L, d_v);   // heads x one partial state: the largest slab's
    return prefill_tc_state_workspace_bytes(B * H, L, d_v);
}

based_status based_prefill_state(const void* k, const void* v, float* kv_state, float* z_state, int B, int H, int L,
                                 int d_feat, int d_v, based_dtype io, int flags, void* workspace,
                                 size_t workspace_bytes, void* cuda_stream) {
    if (!k || !v || !kv_state || !z_state || B <= 0 || H <= 0 || L <= 0) return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if (flags & ~(BASED_STATE_CONTINUE | BASED_STATE_SYM)) return BASED_ERR_INVALID_ARG;
    if ((d_feat != kDFeat && !df_generic(d_feat)) || !dv_ok(d_v)) return BASED_ERR_UNSUPPORTED;
    if ((long long)B * H > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    const bool tc16 = d_feat == kDFeat && io == BASED_BF16;
    if ((flags & BASED_STATE_SYM) && !tc16) return BASED_ERR_UNSUPPORTED;      // symmetric rows: d' = 16, bf16 io
    if (!aligned16(k) || !aligned16(v) || !aligned16(kv_state) || !aligned16(z_state) || !aligned16(workspace))
        return BASED_ERR_ALIGNMENT;
    if ((long long)B * H > kHeadSlab) {
        const size_t es = esize(io), rows = (flags & BASED_STATE_SYM) ? kDSym : 1 + d_feat + d_feat * d_feat;
        for (long long h0 = 0; h0 < (long long)B * H; h0 += kHeadSlab) {
            const int n = (int)((long long)B * H - h0 < kHeadSlab ? (long long)B * H - h0 : kHeadSlab);
            const based_status st = based_prefill_state(
                off(k, (size_t)h0 * L * d_feat * es), off(v, (size_t)h0 * L * d_v * es), off(kv_state, (size_t)h0 * rows * d_v),
                off(z_state, (size_t)h0 * rows), 1, n, L, d_feat, d_v, io, flags, workspace, workspace_bytes, cuda_stream);
            if (st != BASED_OK) return st;
        }
        return BASED_OK;
    }
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (tc16) {
        if (!workspace || workspace_bytes < based_prefill_state_workspace_bytes(B, H, L, d_feat, d_v, io))
            return BASED_ERR_WORKSPACE;
        return launch_prefill_tc_state(k, v, kv_state, z_state, B * H, L, d_v, flags, workspace, stream);
    }
    return launch_state_generic(k, v, kv_state, z_state, B * H, L, d_feat, d_v, io,
                                (flags & BASED_STATE_CONTINUE) ? 1 : 0, stream);
}

based_status based_decode_step(const void* q, const void* k, const void* v, float* kv_state, float* z_state,
                               void* out, int B, int H, int d_feat, int d_v, based_dtype io, void* cuda_stream) {
    if (!q || !k || !v || !out || !kv_state || !z_state || B <= 0 || H <= 0) return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if ((d_feat != kDFeat && !df_generic(d_feat)) || !dv_ok(d_v)) return BASED_ERR_UNSUPPORTED;
    if ((long long)B * H > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(kv_state) ||
        !aligned16(z_state))
        return BASED_ERR_ALIGNMENT;
    if (d_feat != kDFeat)
        return launch_decode_generic(q, k, v, kv_state, z_state, out, B * H, d_feat, d_v, io, false,
                                     static_cast<cudaStream_t>(cuda_stream));
    return launch_decode(q, k, v, kv_state, z_state, out, B * H, d_v, io, false, false,
                         static_cast<cudaStream_t>(cuda_stream));
}

based_status based_decode_step_flags(const void* q, const void* k, const void* v, float* kv_state, float* z_state,
                                     void* out, int B, int H, int d_feat, int d_v, based_dtype io, int flags,
                                     void* cuda_stream) {
    if (!q || !k || !v || !out || !kv_state || !z_state || B <= 0 || H <= 0) return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if (flags & ~(BASED_STATE_SYM | BASED_NUMERATOR_ONLY)) return BASED_ERR_INVALID_ARG;
    if ((d_feat != kDFeat && !df_generic(d_feat)) || !dv_ok(d_v)) return BASED_ERR_UNSUPPORTED;
    if ((long long)B * H > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(kv_state) ||
        !aligned16(z_state))
        return BASED_ERR_ALIGNMENT;
    if (d_feat != kDFeat) {
        if (flags & BASED_STATE_SYM) return BASED_ERR_UNSUPPORTED;
        return launch_decode_generic(q, k, v, kv_state, z_state, out, B * H, d_feat, d_v, io,
                                     (flags & BASED_NUMERATOR_ONLY) != 0, static_cast<cudaStream_t>(cuda_stream));
    }
    return launch_decode(q, k, v, kv_state, z_state, out, B * H, d_v, io, (flags & BASED_STATE_SYM) != 0,
                         (flags & BASED_NUMERATOR_ONLY) != 0, static_cast<cudaStream_t>(cuda_stream));
}

based_status based_decode_step_sym(const void* q, const void* k, const void* v, float* kv_sym, float* z_sym,
                                   void* out, int B, int H, int d_feat, int d_v, based_dtype io,
                                   void* cuda_stream) {
    if (!q || !k || !v || !out || !kv_sym || !z_sym || B <= 0 || H <= 0) return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if (d_feat != kDFeat || !dv_ok(d_v)) return BASED_ERR_UNSUPPORTED;
    if ((long long)B * H > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(kv_sym) ||
        !aligned16(z_sym))
        return BASED_ERR_ALIGNMENT;
    return launch_decode(q, k, v, kv_sym, z_sym, out, B * H, d_v, io, true, false,
                         static_cast<cudaStream_t>(cuda_stream));
}

static based_status state_convert(const float* kv_in, const float* z_in, float* kv_out, float* z_out, int B, int H,
                                  int d_feat, int d_v, bool to_sym, void* cuda_stream) {
    if (!kv_in || !z_in || !kv_out || !z_out || B <= 0 || H <= 0) return BASED_ERR_INVALID_ARG;
    if (kv_in == kv_out || z_in == z_out) return BASED_ERR_INVALID_ARG;
    if (d_feat != kDFeat || !dv_ok(d_v)) return BASED_ERR_UNSUPPORTED;
    if ((long long)B * H > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    if (!aligned16(kv_in) || !aligned16(z_in) || !aligned16(kv_out) || !aligned16(z_out)) return BASED_ERR_ALIGNMENT;
    return launch_state_convert(kv_in, z_in, kv_out, z_out, B * H, d_v, to_sym,
                                static_cast<cudaStream_t>(cuda_stream));
}

based_status based_state_to_sym(const float* kv_state, const float* z_state, float* kv_sym, float* z_sym, int B,
                                int H, int d_feat, int d_v, void* cuda_stream) {
    return state_convert(kv_state, z_state, kv_sym, z_sym, B, H, d_feat, d_v, true, cuda_stream);
}

based_status based_state_from_sym(const float* kv_sym, const float* z_sym, float* kv_state, float* z_state, int B,
                                  int H, int d_feat, int d_v, void* cuda_stream) {
    return state_convert(kv_sym, z_sym, kv_state, z_state, B, H, d_feat, d_v, false, cuda_stream);
}

based_status swa_forward(const void* q, const void* k, const void* v, void* out, int B, int H, int L, int d,
                         int window, float softmax_scale, based_dtype io, void* cuda_stream) {
    if (!q || !k || !v || !out || B <= 0 || H <= 0 || L <= 0 || window <= 0) return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if (out == q || out == k || out == v) return BASED_ERR_INVALID_ARG;
    if (d != 64 || window > 128) return BASED_ERR_UNSUPPORTED;
    if ((long long)B * H > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out)) return BASED_ERR_ALIGNMENT;
    if ((long long)B * H > kHeadSlab) {
        const size_t hb = (size_t)L * d * esize(io);
        for (long long h0 = 0; h0 < (long long)B * H; h0 += kHeadSlab) {
            const int n = (int)((long long)B * H - h0 < kHeadSlab ? (long long)B * H - h0 : kHeadSlab);
            const based_status st = swa_forward(off(q, h0 * hb), off(k, h0 * hb), off(v, h0 * hb), off(out, h0 * hb), 1, n, L,
                                                d, window, softmax_scale, io, cuda_stream);
            if (st != BASED_OK) return st;
        }
        return BASED_OK;
    }
    const float scale = softmax_scale > 0.f ? softmax_scale : 0.125f;   // 1/sqrt(64)
    if (io == BASED_BF16 && swa_tc_supported(window))
        return launch_swa_tc(q, k, v, out, B * H, L, window, scale, static_cast<cudaStream_t>(cuda_stream));
    return launch_swa_simt(q, k, v, out, B * H, L, window, scale, io, static_cast<cudaStream_t>(cuda_stream));
}

based_status swa_decode_step(const void* q, const void* k, const void* v, void* k_cache, void* v_cache, void* out,
                             int B, int H, int d, int window, int pos, float softmax_scale, based_dtype io,
                             void* cuda_stream) {
    if (!q || !k || !v || !k_cache || !v_cache || !out || B <= 0 || H <= 0 || window <= 0 || pos < 0)
        return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if (d != 64 || window > 128) return BASED_ERR_UNSUPPORTED;
    if ((long long)B * H > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(k_cache) || !aligned16(v_cache) ||
        !aligned16(out))
        return BASED_ERR_ALIGNMENT;
    const float scale = softmax_scale > 0.f ? softmax_scale : 0.125f;   // 1/sqrt(64)
    return launch_swa_decode(q, k, v, k_cache, v_cache, out, B * H, window, pos, nullptr, nullptr, scale, io,
                             static_cast<cudaStream_t>(cuda_stream));
}

based_status swa_decode_step_at(const void* q, const void* k, const void* v, void* k_cache, void* v_cache,
                                void* out, int B, int H, int d, int window, const int* pos_device,
                                float softmax_scale, based_dtype io, void* cuda_stream) {
    if (!q || !k || !v || !k_cache || !v_cache || !out || !pos_device || B <= 0 || H <= 0 || window <= 0)
        return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if (d != 64 || window > 128) return BASED_ERR_UNSUPPORTED;
    if ((long long)B * H > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(k_cache) || !aligned16(v_cache) ||
        !aligned16(out) || (reinterpret_cast<uintptr_t>(pos_device) & 3u))
        return BASED_ERR_ALIGNMENT;
    const float scale = softmax_scale > 0.f ? softmax_scale : 0.125f;   // 1/sqrt(64)
    return launch_swa_decode(q, k, v, k_cache, v_cache, out, B * H, window, 0, pos_device, nullptr, scale, io,
                             static_cast<cudaStream_t>(cuda_stream));
}

based_status swa_decode_step_ragged(const void* q, const void* k, const void* v, void* k_cache, void* v_cache,
                                    void* out, int B, int H, int d, int window, const int* pos_per_sequence,
                                    float softmax_scale, based_dtype io, void* cuda_stream) {
    if (!q || !k || !v || !k_cache || !v_cache || !out || !pos_per_sequence || B <= 0 || H <= 0 || window <= 0)
        return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if (d != 64 || window > 128) return BASED_ERR_UNSUPPORTED;
    if ((long long)B * H > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(k_cache) || !aligned16(v_cache) ||
        !aligned16(out) || (reinterpret_cast<uintptr_t>(pos_per_sequence) & 3u))
        return BASED_ERR_ALIGNMENT;
    const float scale = softmax_scale > 0.f ? softmax_scale : 0.125f;   // 1/sqrt(64)
    return launch_swa_decode(q, k, v, k_cache, v_cache, out, B * H, window, 0, pos_per_sequence, nullptr, scale, io,
                             static_cast<cudaStream_t>(cuda_stream), H);
}

based_status swa_decode_step_advance(const void* q, const void* k, const void* v, void* k_cache, void* v_cache,
                                     void* out, int B, int H, int d, int window, int* pos_state,
                                     float softmax_scale, based_dtype io, void* cuda_stream) {
    if (!q || !k || !v || !k_cache || !v_cache || !out || !pos_state || B <= 0 || H <= 0 || window <= 0)
        return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if (d != 64 || window > 128) return BASED_ERR_UNSUPPORTED;
    if ((long long)B * H > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(k_cache) || !aligned16(v_cache) ||
        !aligned16(out) || (reinterpret_cast<uintptr_t>(pos_state) & 7u))
        return BASED_ERR_ALIGNMENT;
    const float scale = softmax_scale > 0.f ? softmax_scale : 0.125f;   // 1/sqrt(64)
    return launch_swa_decode(q, k, v, k_cache, v_cache, out, B * H, window, 0, pos_state, pos_state, scale, io,
                             static_cast<cudaStream_t>(cuda_stream));
}

static based_status generation_step_check(const void* q, const void* k, const void* v, const float* kv_state, const float* z_state,
                                          const void* out, const void* qw, const void* kw, const void* vw, const void* k_cache,
                                          const void* v_cache, const void* out_w, int B, int H, int d_feat, int d_v, int H_w, int d_w,
                                          int window, const int* pos_state, based_dtype io, int flags) {
    if (!q || !k || !v || !kv_state || !z_state || !out || !qw || !kw || !vw || !k_cache || !v_cache || !out_w ||
        !pos_state || B <= 0 || H <= 0 || H_w <= 0 || window <= 0)
        return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if (flags & ~(BASED_STATE_SYM | BASED_NUMERATOR_ONLY)) return BASED_ERR_INVALID_ARG;
    if (d_feat != kDFeat || !dv_ok(d_v) || d_w != 64 || window > 128) return BASED_ERR_UNSUPPORTED;
    if ((long long)B * H + ((long long)B * H_w + 1) / 2 > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(kv_state) || !aligned16(z_state) ||
        !aligned16(out) || !aligned16(qw) || !aligned16(kw) || !aligned16(vw) || !aligned16(k_cache) ||
        !aligned16(v_cache) || !aligned16(out_w) || (reinterpret_cast<uintptr_t>(pos_state) & 7u))
        return BASED_ERR_ALIGNMENT;
    return BASED_OK;
}

based_status based_generation_step(const void* q, const void* k, const void* v, float* kv_state, float* z_state,
                                   void* out, const void* qw, const void* kw, const void* vw, void* k_cache,
                                   void* v_cache, void* out_w, int B, int H, int d_feat, int d_v, int H_w, int d_w,
                                   int window, int* pos_state, float softmax_scale, based_dtype io, int flags,
                                   void* cuda_stream) {
    const based_status st = generation_step_check(q, k, v, kv_state, z_state, out, qw, kw, vw, k_cache, v_cache, out_w, B, H, d_feat,
                                                  d_v, H_w, d_w, window, pos_state, io, flags);
    if (st != BASED_OK) return st;
    const float scale = softmax_scale > 0.f ? softmax_scale : 0.125f;   // 1/sqrt(64)
    return launch_generation_step(q, k, v, kv_state, z_state, out, B * H, d_v, (flags & BASED_STATE_SYM) != 0,
                                  (flags & BASED_NUMERATOR_ONLY) != 0, qw, kw, vw, k_cache, v_cache, out_w, B * H_w,
                                  window, pos_state, scale, io, static_cast<cudaStream_t>(cuda_stream));
}

// The step's arguments, and the order of its launches.  The kernel is launched as based_generation_step's is, not as a node of
// an instantiated graph: a dependent launch is on the SMs while the one before it drains, which graph launches, each behind
// the end of the one before, are not (16 heads x batch 8 / 16 / 32, 153 rows, d_v 128, on states from memory: 10.5 -> 8.3,
// 13.5 -> 10.2, 20.3 -> 16.8 us per step).  What a graph's launches give besides, an order among themselves whichever streams
// they are on, an event behind every step keeps.
struct based_generation_graph {
    std::vector<unsigned char> args;           // launch_generation_args
    void* buffers[6] = {};
    bool own_inputs = false;                   // the arguments point at inputs other than the buffers
    cudaEvent_t done = nullptr;                // behind the last step
    unsigned long long last_stream = 0;        // its stream's number, which no later stream is given again
    bool launched = false;
    std::mutex mu;
};

void based_generation_graph_destroy(based_generation_graph* g) {
    if (!g) return;
    if (g->done) cudaEventDestroy(g->done);
    delete g;
}

based_status based_generation_graph_create(void* q, void* k, void* v, float* kv_state, float* z_state, void* out, void* qw,
                                           void* kw, void* vw, void* k_cache, void* v_cache, void* out_w, int B, int H,
                                           int d_feat, int d_v, int H_w, int d_w, int window, int* pos_state,
                                           float softmax_scale, based_dtype io, int flags, based_generation_graph** graph) {
    if (!graph) return BASED_ERR_INVALID_ARG;
    *graph = nullptr;
    const based_status st = generation_step_check(q, k, v, kv_state, z_state, out, qw, kw, vw, k_cache, v_cache, out_w, B, H, d_feat,
                                                  d_v, H_w, d_w, window, pos_state, io, flags);
    if (st != BASED_OK) return st;
    based_generation_graph* g = new (std::nothrow) based_generation_graph;
    if (!g) return BASED_ERR_CUDA;
    const float scale = softmax_scale > 0.f ? softmax_scale : 0.125f;   // 1/sqrt(64)
    try {
        g->args.resize(generation_step_args_bytes());
    } catch (const std::bad_alloc&) {
        delete g;
        return BASED_ERR_CUDA;
    }
    if (make_generation_args(g->args.data(), q, k, v, kv_state, z_state, out, B * H, d_v, (flags & BASED_STATE_SYM) != 0,
                             (flags & BASED_NUMERATOR_ONLY) != 0, qw, kw, vw, k_cache, v_cache, out_w, B * H_w, window, pos_state,
                             scale, io) != BASED_OK ||
        cudaEventCreateWithFlags(&g->done, cudaEventDisableTiming) != cudaSuccess) {
        based_generation_graph_destroy(g);
        return BASED_ERR_CUDA;
    }
    void* const buffers[6] = {q, k, v, qw, kw, vw};
    for (int i = 0; i < 6; ++i) g->buffers[i] = buffers[i];
    *graph = g;
    return BASED_OK;
}

based_status based_generation_graph_step(based_generation_graph* g, const void* q, const void* k, const void* v, const void* qw,
                                         const void* kw, const void* vw, void* cuda_stream) {
    if (!g) return BASED_ERR_INVALID_ARG;
    const void* const in[6] = {q, k, v, qw, kw, vw};
    int given = 0;
    for (const void* p : in) {
        given += p != nullptr;
        if (!aligned16(p)) return BASED_ERR_ALIGNMENT;
    }
    if (given != 0 && given != 6) return BASED_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    // a stream under capture cannot take the order among the steps (nor could it take a graph launch)
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    unsigned long long id = 0;
    if (cudaStreamIsCapturing(stream, &capture) != cudaSuccess || capture != cudaStreamCaptureStatusNone ||
        cudaStreamGetId(stream, &id) != cudaSuccess)
        return BASED_ERR_CUDA;
    std::lock_guard<std::mutex> lock(g->mu);
    if (given || g->own_inputs) {
        generation_step_inputs(g->args.data(), in, g->buffers);
        g->own_inputs = given != 0;
    }
    if (g->launched && id != g->last_stream && cudaStreamWaitEvent(stream, g->done, 0) != cudaSuccess) return BASED_ERR_CUDA;
    const based_status st = launch_generation_args(g->args.data(), stream);
    if (st != BASED_OK) return st;
    g->launched = true;
    g->last_stream = id;
    return cudaEventRecord(g->done, stream) == cudaSuccess ? BASED_OK : BASED_ERR_CUDA;
}

static based_status baseconv_check(const void* a, const void* g, const float* h, const float* b2, const void* out,
                                   int B, int N, int C, int width, based_dtype io) {
    if (!a || !g || !h || !b2 || !out || B <= 0 || N <= 0 || C <= 0 || width <= 0) return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if (out == g) return BASED_ERR_INVALID_ARG;
    if (width > 4 || C % 8 != 0 || B > 65535 || (N + 63) / 64 > 65535) return BASED_ERR_UNSUPPORTED;
    if (!aligned16(a) || !aligned16(g) || !aligned16(h) || !aligned16(b2) || !aligned16(out)) return BASED_ERR_ALIGNMENT;
    return BASED_OK;
}

based_status baseconv_gate_forward(const void* a, const void* g, const float* h, const float* b2, void* out, int B,
                                   int N, int C, int width, based_dtype io, void* cuda_stream) {
    const based_status st = baseconv_check(a, g, h, b2, out, B, N, C, width, io);
    if (st != BASED_OK) return st;
    return launch_baseconv(a, g, h, b2, nullptr, out, B, N, C, width, false, io,
                           static_cast<cudaStream_t>(cuda_stream));
}

based_status baseconv_gate_step(const void* a, const void* g, const float* h, const float* b2, void* conv_state,
                                void* out, int B, int C, int width, based_dtype io, void* cuda_stream) {
    const based_status st = baseconv_check(a, g, h, b2, out, B, 1, C, width, io);
    if (st != BASED_OK) return st;
    if (width > 1 && !conv_state) return BASED_ERR_INVALID_ARG;
    if (!aligned16(conv_state)) return BASED_ERR_ALIGNMENT;
    return launch_baseconv(a, g, h, b2, conv_state, out, B, 1, C, width, true, io,
                           static_cast<cudaStream_t>(cuda_stream));
}

static inline bool is_one_of(const void* p, std::initializer_list<const void*> of) {
    for (const void* q : of)
        if (p && p == q) return true;
    return false;
}
static based_status tokens_check(const based_tokens& t, int B, int N, int C, based_dtype io) {
    const long long per16 = 16 / (long long)esize(io);
    if (N > 1 && t.token_stride < C) return BASED_ERR_INVALID_ARG;
    if (B > 1 && t.batch_stride < (N > 1 ? (N - 1) * t.token_stride : 0) + C) return BASED_ERR_INVALID_ARG;
    // (the copies' tensor maps hold strides below 2^40 bytes)
    if ((N > 1 && (t.token_stride % per16 != 0 || t.token_stride >= 1ll << 36)) || (B > 1 && (t.batch_stride % per16 != 0 || t.batch_stride >= 1ll << 37)))
        return BASED_ERR_UNSUPPORTED;
    return aligned16(t.data) ? BASED_OK : BASED_ERR_ALIGNMENT;
}
static based_status recurrence_check(const based_tokens& x, const based_tokens& r, const based_tokens& g, const float* rate, int B, int N, int C,
                                     based_dtype io) {
    if (!x.data || !r.data || !g.data || !rate || B <= 0 || N <= 0 || C <= 0) return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if (C % 8 != 0 || N > 0x7fff0000 || (long long)B * C > (1ll << 36) || gated_recurrence_blocks(B, C, io) > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    for (const based_tokens* t : {&x, &r, &g}) {
        const based_status st = tokens_check(*t, B, N, C, io);
        if (st != BASED_OK) return st;
    }
    return aligned16(rate) ? BASED_OK : BASED_ERR_ALIGNMENT;
}

based_status based_gated_recurrence_forward(based_tokens x, based_tokens r, based_tokens g, const float* rate, const float* state_in,
                                            void* out, float* state_out, int B, int N, int C, based_dtype io, void* cuda_stream) {
    if (!out || is_one_of(out, {x.data, r.data, g.data, rate, state_in, state_out}) || is_one_of(state_out, {x.data, r.data, g.data, rate}))
        return BASED_ERR_INVALID_ARG;
    const based_status st = recurrence_check(x, r, g, rate, B, N, C, io);
    if (st != BASED_OK) return st;
    if (!aligned16(out) || !aligned16(state_in) || !aligned16(state_out)) return BASED_ERR_ALIGNMENT;
    return launch_gated_recurrence(x, r, g, rate, state_in, out, state_out, B, N, C, io, static_cast<cudaStream_t>(cuda_stream));
}

based_status based_gated_recurrence_step(based_tokens x, based_tokens r, based_tokens g, const float* rate, const float* state_in,
                                         void* out, float* state_out, int B, int C, based_dtype io, void* cuda_stream) {
    if (!state_in || !state_out) return BASED_ERR_INVALID_ARG;
    return based_gated_recurrence_forward(x, r, g, rate, state_in, out, state_out, B, 1, C, io, cuda_stream);
}

size_t based_gated_recurrence_backward_workspace_bytes(int B, int N, int C, based_dtype io) {
    if (B <= 0 || N <= 0 || C <= 0 || (io != BASED_F32 && io != BASED_BF16)) return 0;
    return gated_recurrence_backward_bytes(B, N, C, io);
}

based_status based_gated_recurrence_backward(based_tokens x, based_tokens r, based_tokens g, const float* rate, const float* state_in,
                                             based_tokens out, based_tokens dout, const float* dstate_out, void* dx, void* dr, void* dg,
                                             float* drate, float* dstate_in, int B, int N, int C, based_dtype io, void* workspace,
                                             size_t workspace_bytes, void* cuda_stream) {
    if (!out.data || !dout.data || !dx || !dr || !dg || !drate) return BASED_ERR_INVALID_ARG;
    const void* outs[] = {dx, dr, dg, drate, dstate_in};
    for (int i = 0; i < 5; ++i) {
        if (is_one_of(outs[i], {x.data, r.data, g.data, rate, state_in, out.data, dout.data, workspace})) return BASED_ERR_INVALID_ARG;
        if (i < 4 && is_one_of(outs[i], {dstate_out})) return BASED_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (is_one_of(outs[i], {outs[j]})) return BASED_ERR_INVALID_ARG;
    }
    based_status st = recurrence_check(x, r, g, rate, B, N, C, io);
    if (st == BASED_OK) st = tokens_check(out, B, N, C, io);
    if (st == BASED_OK) st = tokens_check(dout, B, N, C, io);
    if (st != BASED_OK) return st;
    for (const void* p : {(const void*)state_in, (const void*)dstate_out, (const void*)dx, (const void*)dr, (const void*)dg,
                          (const void*)drate, (const void*)dstate_in, (const void*)workspace})
        if (!aligned16(p)) return BASED_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < gated_recurrence_backward_bytes(B, N, C, io)) return BASED_ERR_WORKSPACE;
    return launch_gated_recurrence_backward(x, r, g, rate, state_in, out, dout, dstate_out, dx, dr, dg, drate, dstate_in, B, N, C,
                                            static_cast<float*>(workspace), io, static_cast<cudaStream_t>(cuda_stream));
}

static based_status norm_rotate_check(const NormRotate& a, int positions_per_sequence, based_dtype io, int flags) {
    if (!a.q || !a.k || a.B <= 0 || a.L <= 0 || a.Hq <= 0 || a.Hk <= 0 || a.d <= 0 || a.n < 0 || !(a.eps >= 0.f)) return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if ((flags & ~BASED_ROTATE_PAIRS) || (a.n > 0) != (a.freqs != nullptr)) return BASED_ERR_INVALID_ARG;
    if (a.positions && positions_per_sequence != 1 && positions_per_sequence != a.L) return BASED_ERR_INVALID_ARG;
    const long long width_q = (long long)a.Hq * a.d, width_k = (long long)a.Hk * a.d, per16 = 16 / (long long)esize(io);
    if (a.q_stride < width_q || a.k_stride < width_k) return BASED_ERR_INVALID_ARG;
    if (a.d % 16 != 0 || a.d > 256 || a.n % 8 != 0 || 2 * a.n > a.d || a.q_stride % per16 != 0 || a.k_stride % per16 != 0 ||
        width_q > 0x7fffffffLL || width_k > 0x7fffffffLL || (long long)a.B * a.L > 0x7fffff00LL)
        return BASED_ERR_UNSUPPORTED;
    if (!aligned16(a.q) || !aligned16(a.k) || !aligned16(a.wq) || !aligned16(a.wk)) return BASED_ERR_ALIGNMENT;
    if ((reinterpret_cast<uintptr_t>(a.freqs) & 7u) || (reinterpret_cast<uintptr_t>(a.positions) & 3u)) return BASED_ERR_ALIGNMENT;
    return BASED_OK;
}

based_status based_qk_norm_rotate(const void* q, const void* k, long long q_token_stride, long long k_token_stride,
                                  const float* q_weight, const float* k_weight, const double* freqs, const int* positions,
                                  int positions_per_sequence, int start, void* out_q, void* out_k, int B, int L, int H_q, int H_k,
                                  int d, int n, float eps, based_dtype io, int flags, void* cuda_stream) {
    const NormRotate a{q, k, q_token_stride, k_token_stride, q_weight, k_weight, freqs, positions, positions_per_sequence != 1, start,
                       (flags & BASED_ROTATE_PAIRS) != 0, B, L, H_q, H_k, d, n, eps};
    if (!out_q || !out_k || out_q == out_k || is_one_of(out_q, {q, k, q_weight, k_weight, freqs, positions}) ||
        is_one_of(out_k, {q, k, q_weight, k_weight, freqs, positions}))
        return BASED_ERR_INVALID_ARG;
    const based_status st = norm_rotate_check(a, positions_per_sequence, io, flags);
    if (st != BASED_OK) return st;
    if (!aligned16(out_q) || !aligned16(out_k)) return BASED_ERR_ALIGNMENT;
    return launch_norm_rotate(a, out_q, out_k, io, static_cast<cudaStream_t>(cuda_stream));
}

size_t based_qk_norm_rotate_backward_workspace_bytes(int B, int L, int H_q, int H_k, int d, based_dtype io) {
    if (B <= 0 || L <= 0 || H_q <= 0 || H_k <= 0 || d <= 0 || d % 16 != 0 || d > 256 || (io != BASED_F32 && io != BASED_BF16)) return 0;
    return norm_rotate_backward_bytes(B, L, d, io);
}

based_status based_qk_norm_rotate_backward(const void* q, const void* k, long long q_token_stride, long long k_token_stride,
                                           const float* q_weight, const float* k_weight, const double* freqs, const int* positions,
                                           int positions_per_sequence, int start, const void* dout_q, const void* dout_k, void* dq,
                                           void* dk, long long dq_token_stride, long long dk_token_stride, float* dq_weight,
                                           float* dk_weight, int B, int L, int H_q, int H_k, int d, int n, float eps, based_dtype io,
                                           int flags, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const NormRotate a{q, k, q_token_stride, k_token_stride, q_weight, k_weight, freqs, positions, positions_per_sequence != 1, start,
                       (flags & BASED_ROTATE_PAIRS) != 0, B, L, H_q, H_k, d, n, eps};
    if (!dout_q || !dout_k || !dq || !dk || dq == dk || !dq_weight != !dk_weight || (dq_weight && dq_weight == dk_weight))
        return BASED_ERR_INVALID_ARG;
    for (const void* p : {(const void*)dq, (const void*)dk, (const void*)dq_weight, (const void*)dk_weight})
        if (is_one_of(p, {q, k, q_weight, k_weight, freqs, positions, dout_q, dout_k, workspace})) return BASED_ERR_INVALID_ARG;
    based_status st = norm_rotate_check(a, positions_per_sequence, io, flags);
    if (st != BASED_OK) return st;
    NormRotate to = a;                         // (the gradients' layout has the same rules)
    to.q_stride = dq_token_stride;
    to.k_stride = dk_token_stride;
    st = norm_rotate_check(to, positions_per_sequence, io, flags);
    if (st != BASED_OK) return st;
    for (const void* p : {dout_q, dout_k, (const void*)dq, (const void*)dk, (const void*)dq_weight, (const void*)dk_weight, (const void*)workspace})
        if (!aligned16(p)) return BASED_ERR_ALIGNMENT;
    if (dq_weight && (!workspace || workspace_bytes < norm_rotate_backward_bytes(B, L, d, io))) return BASED_ERR_WORKSPACE;
    return launch_norm_rotate_backward(a, dout_q, dout_k, dq, dq_token_stride, dk, dk_token_stride, dq_weight, dk_weight,
                                       static_cast<float*>(workspace), io, static_cast<cudaStream_t>(cuda_stream));
}

size_t swa_backward_workspace_bytes(int B, int H, int L, int window, based_dtype io) {
    if (B <= 0 || H <= 0 || L <= 0 || window <= 0 || window > 128 || (io != BASED_F32 && io != BASED_BF16)) return 0;
    if (io == BASED_BF16) return 0;
    const long long BH = (long long)B * H < kHeadSlab ? (long long)B * H : kHeadSlab;       // the largest slab of heads
    return (size_t)BH * L * 16;
}

based_status swa_backward(const void* q, const void* k, const void* v, const void* dout, void* dq, void* dk, void* dv, int B, int H,
                          int L, int d, int window, float softmax_scale, based_dtype io, void* workspace, size_t workspace_bytes,
                          void* cuda_stream) {
    if (!q || !k || !v || !dout || !dq || !dk || !dv || B <= 0 || H <= 0 || L <= 0 || window <= 0) return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if (dq == dk || dq == dv || dk == dv) return BASED_ERR_INVALID_ARG;
    for (const void* p : {(const void*)dq, (const void*)dk, (const void*)dv})
        if (is_one_of(p, {q, k, v, dout, workspace})) return BASED_ERR_INVALID_ARG;
    if (d != 64 || window > 128) return BASED_ERR_UNSUPPORTED;
    const long long BH = (long long)B * H;
    if (BH > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    for (const void* p : {q, k, v, dout, (const void*)dq, (const void*)dk, (const void*)dv, (const void*)workspace})
        if (!aligned16(p)) return BASED_ERR_ALIGNMENT;
    const size_t need = swa_backward_workspace_bytes(B, H, L, window, io);
    if (need && (!workspace || workspace_bytes < need)) return BASED_ERR_WORKSPACE;
    const float scale = softmax_scale > 0.f ? softmax_scale : 0.125f;   // 1/sqrt(64)
    const size_t hb = (size_t)L * d * esize(io);
    for (long long h0 = 0; h0 < BH; h0 += kHeadSlab) {
        const int n = (int)(BH - h0 < kHeadSlab ? BH - h0 : kHeadSlab);
        const size_t at = h0 * hb;
        const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
        const based_status st =
            io == BASED_BF16 ? launch_swa_backward_tc(off(q, at), off(k, at), off(v, at), off(dout, at), off(dq, at), off(dk, at), off(dv, at),
                                                      n, L, window, scale, stream)
                             : launch_swa_backward_f32(off(q, at), off(k, at), off(v, at), off(dout, at), off(dq, at), off(dk, at),
                                                       off(dv, at), static_cast<float*>(workspace), n, L, window, scale, stream);
        if (st != BASED_OK) return st;
    }
    return BASED_OK;
}

// a factor of scores: chosen here if not above 0; its reciprocal, and products with it, are to be in the range of fp32
static bool factor_ok(float x) { return !(x > 0.f) || (x >= 0x1p-60f && x <= 0x1p60f); }
static based_status heads_check(const based_heads& t, int B, int H, int L, int d, based_dtype io, bool written) {
    if (!t.data) return BASED_ERR_INVALID_ARG;
    const long long per16 = 16 / (long long)esize(io);
    struct { long long stride; int size; } dim[3] = {{t.token_stride, L}, {t.head_stride, H}, {t.batch_stride, B}};
    for (const auto& x : dim)
        if (x.size > 1 && x.stride < d) return BASED_ERR_INVALID_ARG;
    for (const auto& x : dim)      // (tensor maps hold strides below 2^40 bytes)
        if (x.size > 1 && (x.stride % per16 != 0 || x.stride >= 1ll << 37)) return BASED_ERR_UNSUPPORTED;
    if (written) {                 // from the smallest stride on, each steps over all that lies inside it
        long long extent = d;
        for (int turn = 0; turn < 3; ++turn) {
            int least = -1;
            for (int i = 0; i < 3; ++i)
                if (dim[i].size > 1 && (least < 0 || dim[i].stride < dim[least].stride)) least = i;
            if (least < 0) break;
            if (dim[least].stride < extent) return BASED_ERR_INVALID_ARG;
            extent += dim[least].stride * (dim[least].size - 1);
            dim[least].size = 0;
        }
    }
    return aligned16(t.data) ? BASED_OK : BASED_ERR_ALIGNMENT;
}
static based_status decay_sizes_check(int B, int H, int L, int d_k, int d_v, based_dtype io) {
    if (B <= 0 || H <= 0 || L <= 0 || d_k <= 0 || d_v <= 0 || (io != BASED_F32 && io != BASED_BF16)) return BASED_ERR_INVALID_ARG;
    if (d_k % 8 || d_v % 8 || d_k > kDecayMaxWidth || d_v > kDecayMaxWidth || L > 0x7fff0000 || (long long)B * H > 0x7fffffffLL ||
        (long long)B * ((L + 63) / 64) > 0x7fffffffLL || (long long)B * H * d_k * d_v > 1ll << 40)
        return BASED_ERR_UNSUPPORTED;
    return BASED_OK;
}
static DecayPlan decay_plan_of(const DecayCall& c, based_dtype io) { return io == BASED_F32 ? decay_plan_f32(c) : decay_plan_tc(c); }
// The calls that one is run as.  In bf16 the passes that return no state take operands in fewer parts and may have tiles twice as wide, so the
// others go by themselves where the plans say that it pays for the launches (8 x 16 heads x 4096 tokens, 128/128: 369 us for 476; but 1 x 8 x
// 4096: 90 for 56)
static int decay_parts(const DecayCall& c, based_dtype io, DecayCall (&part)[2]) {
    part[0] = part[1] = c;
    if (io != BASED_BF16 || c.passes != 3 || !c.pass[2].state_out) return 1;
    part[0].passes = 2;
    part[1].passes = 1;
    part[1].pass[0] = c.pass[2];
    const double launch = 2.5;             // in blocks, as in decay_plan_tc
    if (decay_plan_of(part[0], io).time + decay_plan_of(part[1], io).time + launch < decay_plan_of(c, io).time) return 2;
    part[0] = c;
    return 1;
}
static size_t decay_parts_bytes(const DecayCall& c, based_dtype io) {
    DecayCall part[2];
    size_t most = 0;
    for (int i = 0, n = decay_parts(c, io, part); i < n; ++i) {
        const size_t bytes = decay_plan_of(part[i], io).bytes();
        most = bytes > most ? bytes : most;
    }
    return most;
}
// what a call of these sizes takes, whether it returns a state or not
static size_t decay_bytes(int passes, int B, int H, int L, int d_k, int d_v, bool documents, based_dtype io) {
    if (decay_sizes_check(B, H, L, d_k, d_v, io) != BASED_OK) return 0;
    static const int given = 0;
    static float wanted = 0.f;
    DecayCall c{};
    c.passes = passes;
    c.B = B; c.H = H; c.L = L;
    c.documents = documents ? &given : nullptr;
    const int dc[2][3] = {{d_k, 0, 0}, {d_v, d_v, d_k}}, de[2][3] = {{d_v, 0, 0}, {d_k, d_k, d_v}};
    for (int i = 0; i < passes; ++i) {
        c.pass[i].dc = dc[passes == 3][i];
        c.pass[i].de = de[passes == 3][i];
    }
    const size_t without = decay_parts_bytes(c, io);
    c.pass[passes - 1].state_out = &wanted;
    const size_t with = decay_parts_bytes(c, io);
    return with > without ? with : without;
}
static based_status decay_run(const DecayCall& c, based_dtype io, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    DecayCall part[2];
    const int n = decay_parts(c, io, part);
    DecayPlan plan[2];
    if (!aligned16(workspace)) return BASED_ERR_ALIGNMENT;
    for (int i = 0; i < n; ++i) {
        plan[i] = decay_plan_of(part[i], io);
        if (plan[i].ctas > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
        if (plan[i].bytes() && (!workspace || workspace_bytes < plan[i].bytes())) return BASED_ERR_WORKSPACE;
    }
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    based_status st = BASED_OK;
    for (int i = 0; i < n && st == BASED_OK; ++i)
        st = io == BASED_F32 ? launch_decay_f32(part[i], plan[i], workspace, stream) : launch_decay_tc(part[i], plan[i], workspace, stream);
    return st;
}

size_t based_decay_attention_workspace_bytes(int B, int H, int L, int d_k, int d_v, int with_documents, based_dtype io) {
    return decay_bytes(1, B, H, L, d_k, d_v, with_documents != 0, io);
}
size_t based_decay_attention_backward_workspace_bytes(int B, int H, int L, int d_k, int d_v, int with_documents, based_dtype io) {
    return decay_bytes(3, B, H, L, d_k, d_v, with_documents != 0, io);
}

based_status based_decay_attention_forward(based_heads q, based_heads k, based_heads v, const float* rate, const int* documents,
                                           const float* state_in, based_heads out, float* state_out, int B, int H, int L, int d_k, int d_v,
                                           float scale, based_dtype io, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!q.data || !k.data || !v.data || !out.data || !rate) return BASED_ERR_INVALID_ARG;
    based_status st = decay_sizes_check(B, H, L, d_k, d_v, io);
    if (st == BASED_OK && !factor_ok(scale)) st = BASED_ERR_UNSUPPORTED;
    if (st != BASED_OK) return st;
    if (is_one_of(out.data, {q.data, k.data, v.data, rate, documents, state_in, state_out, workspace}) ||
        is_one_of(state_out, {q.data, k.data, v.data, rate, documents, state_in, workspace}))
        return BASED_ERR_INVALID_ARG;
    st = heads_check(q, B, H, L, d_k, io, false);
    if (st == BASED_OK) st = heads_check(k, B, H, L, d_k, io, false);
    if (st == BASED_OK) st = heads_check(v, B, H, L, d_v, io, false);
    if (st == BASED_OK) st = heads_check(out, B, H, L, d_v, io, true);
    if (st != BASED_OK) return st;
    if (!aligned16(rate) || !aligned16(state_in) || !aligned16(state_out) || (reinterpret_cast<uintptr_t>(documents) & 3)) return BASED_ERR_ALIGNMENT;
    DecayCall c{};
    c.passes = 1;
    c.pass[0] = {q, k, v, out, d_k, d_v, state_in, state_out, 0, 0, 1.f, 1.f};
    c.rate = rate;
    c.documents = documents;
    c.B = B; c.H = H; c.L = L;
    c.factor = scale > 0.f ? scale : 1.f / sqrtf((float)d_k);
    return decay_run(c, io, workspace, workspace_bytes, cuda_stream);
}

based_status based_decay_attention_step(const void* q, const void* k, const void* v, const float* rate, const float* state_in, void* out,
                                        float* state_out, int B, int H, int d_k, int d_v, float scale, based_dtype io, void* cuda_stream) {
    if (!q || !k || !v || !rate || !state_in || !out || !state_out) return BASED_ERR_INVALID_ARG;
    based_status st = decay_sizes_check(B, H, 1, d_k, d_v, io);
    if (st == BASED_OK && !factor_ok(scale)) st = BASED_ERR_UNSUPPORTED;
    if (st != BASED_OK) return st;
    if (is_one_of(out, {q, k, v, rate, state_in, state_out}) || is_one_of(state_out, {q, k, v, rate})) return BASED_ERR_INVALID_ARG;
    for (const void* p : {q, k, v, (const void*)rate, (const void*)state_in, (const void*)out, (const void*)state_out})
        if (!aligned16(p)) return BASED_ERR_ALIGNMENT;
    return launch_decay_step(q, k, v, rate, state_in, out, state_out, (long long)B * H, H, d_k, d_v,
                             scale > 0.f ? scale : 1.f / sqrtf((float)d_k), io, static_cast<cudaStream_t>(cuda_stream));
}

based_status based_decay_attention_backward(based_heads q, based_heads k, based_heads v, const float* rate, const int* documents,
                                            const float* state_in, based_heads dout, const float* dstate_out, based_heads dq, based_heads dk,
                                            based_heads dv, float* dstate_in, int B, int H, int L, int d_k, int d_v, float scale,
                                            based_dtype io, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!q.data || !k.data || !v.data || !dout.data || !dq.data || !dk.data || !dv.data || !rate) return BASED_ERR_INVALID_ARG;
    based_status st = decay_sizes_check(B, H, L, d_k, d_v, io);
    if (st == BASED_OK && !factor_ok(scale)) st = BASED_ERR_UNSUPPORTED;
    if (st != BASED_OK) return st;
    const void* outs[] = {dq.data, dk.data, dv.data, dstate_in};
    for (int i = 0; i < 4; ++i) {
        if (is_one_of(outs[i], {q.data, k.data, v.data, dout.data, rate, documents, state_in, dstate_out, workspace})) return BASED_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (is_one_of(outs[i], {outs[j]})) return BASED_ERR_INVALID_ARG;
    }
    const struct { const based_heads* t; int d; bool written; } all[] = {{&q, d_k, false}, {&k, d_k, false}, {&v, d_v, false}, {&dout, d_v, false},
                                                                         {&dq, d_k, true}, {&dk, d_k, true}, {&dv, d_v, true}};
    for (const auto& x : all) {
        st = heads_check(*x.t, B, H, L, x.d, io, x.written);
        if (st != BASED_OK) return st;
    }
    for (const void* p : {(const void*)rate, (const void*)state_in, (const void*)dstate_out, (const void*)dstate_in})
        if (!aligned16(p)) return BASED_ERR_ALIGNMENT;
    if (reinterpret_cast<uintptr_t>(documents) & 3) return BASED_ERR_ALIGNMENT;
    DecayCall c{};
    c.passes = 3;
    c.factor = scale > 0.f ? scale : 1.f / sqrtf((float)d_k);
    // R of the backward passes is kept without the scale
    c.pass[0] = {dout, v, k, dq, d_v, d_k, state_in, nullptr, 1, 0, 1.f, 1.f};
    c.pass[1] = {v, dout, q, dk, d_v, d_k, dstate_out, nullptr, 1, 1, 1.f / c.factor, c.factor};
    c.pass[2] = {k, q, dout, dv, d_k, d_v, dstate_out, dstate_in, 0, 1, 1.f / c.factor, c.factor};
    c.rate = rate;
    c.documents = documents;
    c.B = B; c.H = H; c.L = L;
    return decay_run(c, io, workspace, workspace_bytes, cuda_stream);
}

static based_status pages_check(const based_pages& c, const int* page_table, const int* pos, int B, int H, int d, int max_pages, based_dtype io) {
    if (!c.k || !c.v || c.k == c.v || !page_table || !pos || B <= 0 || H <= 0 || d <= 0 || c.pages <= 0 || c.page_size <= 0 || max_pages <= 0 ||
        (io != BASED_F32 && io != BASED_BF16))
        return BASED_ERR_INVALID_ARG;
    if (d % 8 || d > 128 || (long long)max_pages * c.page_size > 0x7fffffffLL || (long long)B * H > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    const long long per16 = 16 / (long long)esize(io);
    struct { long long stride; int size; } dim[3] = {{c.page_stride, c.pages}, {c.head_stride, H}, {c.token_stride, c.page_size}};
    for (const auto& x : dim)
        if (x.size > 1 && x.stride < d) return BASED_ERR_INVALID_ARG;
    for (const auto& x : dim)
        if (x.size > 1 && (x.stride % per16 != 0 || x.stride >= 1ll << 40)) return BASED_ERR_UNSUPPORTED;
    long long extent = d;                  // no slot lies in another, as with outputs given by strides
    for (int turn = 0; turn < 3; ++turn) {
        int least = -1;
        for (int i = 0; i < 3; ++i)
            if (dim[i].size > 1 && (least < 0 || dim[i].stride < dim[least].stride)) least = i;
        if (least < 0) break;
        if (dim[least].stride < extent) return BASED_ERR_INVALID_ARG;
        extent += dim[least].stride * (dim[least].size - 1);
        dim[least].size = 0;
    }
    if (!aligned16(c.k) || !aligned16(c.v) || (reinterpret_cast<uintptr_t>(page_table) & 3) || (reinterpret_cast<uintptr_t>(pos) & 3)) return BASED_ERR_ALIGNMENT;
    return BASED_OK;
}

size_t based_paged_decode_step_workspace_bytes(int B, int H_q, int H_k, int d, int page_size, int max_pages, based_dtype io) {
    if (B <= 0 || H_q <= 0 || H_k <= 0 || H_q % H_k || d <= 0 || d % 8 || d > 128 || page_size <= 0 || max_pages <= 0 ||
        (long long)max_pages * page_size > 0x7fffffffLL || (io != BASED_F32 && io != BASED_BF16))
        return 0;
    return paged_decode_bytes(B, H_q, H_k, d, page_size, max_pages, io);
}

based_status based_paged_decode_step(const void* q, const void* k, const void* v, based_pages cache, const int* page_table, const int* pos,
                               const float* slopes, void* out, int B, int H_q, int H_k, int d, int max_pages, int window, float softmax_scale,
                               float softcap, based_dtype io, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!q || !k || !v || !out || H_q <= 0 || H_k <= 0 || H_q % H_k || window < 0 || !(softcap >= 0.f)) return BASED_ERR_INVALID_ARG;
    based_status st = pages_check(cache, page_table, pos, B, H_k, d, max_pages, io);
    if (st == BASED_OK && !(factor_ok(softmax_scale) && factor_ok(softcap))) st = BASED_ERR_UNSUPPORTED;
    if (st != BASED_OK) return st;
    if (is_one_of(out, {q, k, v, cache.k, cache.v, page_table, pos, slopes, workspace}) || is_one_of(workspace, {q, k, v, cache.k, cache.v, page_table, pos, slopes}))
        return BASED_ERR_INVALID_ARG;
    if ((long long)B * H_q > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    for (const void* p : {q, k, v, (const void*)out, (const void*)workspace})
        if (!aligned16(p)) return BASED_ERR_ALIGNMENT;
    if (reinterpret_cast<uintptr_t>(slopes) & 3) return BASED_ERR_ALIGNMENT;
    const size_t need = paged_decode_bytes(B, H_q, H_k, d, cache.page_size, max_pages, io);
    if (need && (!workspace || workspace_bytes < need)) return BASED_ERR_WORKSPACE;
    const PagedCall c{q, k, v, cache.k, cache.v, cache.page_stride, cache.head_stride, cache.token_stride, page_table, pos, slopes, out, B, H_q, H_k, d,
                      cache.pages, cache.page_size, max_pages, window, softmax_scale > 0.f ? softmax_scale : 1.f / sqrtf((float)d), softcap};
    return launch_paged_decode(c, workspace, io, static_cast<cudaStream_t>(cuda_stream));
}

based_status based_paged_cache_write(based_heads k, based_heads v, based_pages cache, const int* page_table, const int* pos, const int* counts, int B,
                               int H, int L, int d, int max_pages, based_dtype io, void* cuda_stream) {
    if (!k.data || !v.data || L <= 0) return BASED_ERR_INVALID_ARG;
    based_status st = pages_check(cache, page_table, pos, B, H, d, max_pages, io);
    if (st == BASED_OK) st = heads_check(k, B, H, L, d, io, false);
    if (st == BASED_OK) st = heads_check(v, B, H, L, d, io, false);
    if (st != BASED_OK) return st;
    if (is_one_of(cache.k, {k.data, v.data}) || is_one_of(cache.v, {k.data, v.data})) return BASED_ERR_INVALID_ARG;
    if (L > 0x7fff0000 || (long long)B * H * (((long long)L + 63) / 64) > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(counts) & 3) return BASED_ERR_ALIGNMENT;
    const PagedWrite c{k, v, cache.k, cache.v, cache.page_stride, cache.head_stride, cache.token_stride, page_table, pos, counts, B, H, L, d, cache.pages,
                       cache.page_size, max_pages};
    return launch_paged_write(c, io, static_cast<cudaStream_t>(cuda_stream));
}

size_t based_prefill_backward_workspace_bytes(int B, int H, int L, int d_v, based_dtype io) {
    if (B <= 0 || H <= 0 || L <= 0 || !dv_ok(d_v)) return 0;
    const int heads = (long long)B * H > kHeadSlab ? (int)kHeadSlab : B * H;       // the largest slab of heads
    if (io == BASED_BF16) return backward_tc_workspace_bytes(heads, L, d_v);
    return (size_t)heads * L * 2 * sizeof(float);
}

int based_prefill_backward_block_tokens(int B, int H, int L, int d_feat, int d_v, based_dtype io, int flags,
                                        int with_out) {
    if (B <= 0 || H <= 0 || L <= 0 || !dv_ok(d_v) || io != BASED_BF16) return 0;
    return backward_tc_block_tokens(B * H, L, d_feat, d_v, (with_out || (flags & BASED_NUMERATOR_ONLY)) ? 1 : 0);
}

// fp32 io, one slab of heads, checked arguments; dout_H: 0, or H where dout lies [B, L, H, d_v]
static based_status backward_f32(const void* q, const void* k, const void* v, const void* dout, int dout_H, void* dq, void* dk,
                                 void* dv, int B, int H, int L, int d_v, int flags, void* workspace, size_t workspace_bytes,
                                 void* cuda_stream) {
    auto in = [](const void* p) { return static_cast<const float*>(p); };
    auto out = [](void* p) { return static_cast<float*>(p); };
    const int numerator_only = (flags & BASED_NUMERATOR_ONLY) ? 1 : 0;
    const size_t parts = based_f32_parts_bytes(B, H, L, kDFeat, d_v, 1);
    if (parts > 0 && workspace_bytes >= parts)
        return launch_quadratic_backward_f32(in(q), in(k), in(v), in(dout), dout_H, out(dq), out(dk), out(dv), workspace, B * H, L,
                                             numerator_only, static_cast<cudaStream_t>(cuda_stream));
    return launch_prefill_backward_f32(in(q), in(k), in(v), in(dout), dout_H, out(dq), out(dk), out(dv), out(workspace), B * H, L,
                                       d_v, numerator_only, static_cast<cudaStream_t>(cuda_stream));
}

static based_status prefill_backward(const void* q, const void* k, const void* v, const void* out, const void* dout,
                                     void* dq, void* dk, void* dv, int B, int H, int L, int d_feat, int d_v,
                                     based_dtype io, int flags, void* workspace, size_t workspace_bytes,
                                     void* cuda_stream) {
    if (!q || !k || !v || !dout || !dq || !dk || !dv || B <= 0 || H <= 0 || L <= 0) return BASED_ERR_INVALID_ARG;
    if (io != BASED_F32 && io != BASED_BF16) return BASED_ERR_INVALID_ARG;
    if (flags & ~BASED_NUMERATOR_ONLY) return BASED_ERR_INVALID_ARG;
    if (dq == q || dq == k || dk == q || dk == k || dv == v || dv == dout) return BASED_ERR_INVALID_ARG;
    // the other feature dimensions: bf16 io only (the tensor-core kernels take d' as a parameter)
    if (!(d_feat == kDFeat || (df_generic(d_feat) && io == BASED_BF16)) || !dv_ok(d_v)) return BASED_ERR_UNSUPPORTED;
    if ((long long)B * H > 0x7fffffffLL) return BASED_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(dout) || !aligned16(dq) || !aligned16(dk) ||
        !aligned16(dv) || !aligned16(workspace) || !aligned16(out))
        return BASED_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < based_prefill_backward_workspace_bytes(B, H, L, d_v, io))
        return BASED_ERR_WORKSPACE;
    if ((long long)B * H > kHeadSlab) {
        const size_t qb = (size_t)L * d_feat * esize(io), vb = (size_t)L * d_v * esize(io);
        for (long long h0 = 0; h0 < (long long)B * H; h0 += kHeadSlab) {
            const int n = (int)((long long)B * H - h0 < kHeadSlab ? (long long)B * H - h0 : kHeadSlab);
            const based_status st = prefill_backward(off(q, h0 * qb), off(k, h0 * qb), off(v, h0 * vb), off(out, h0 * vb),
                                                     off(dout, h0 * vb), off(dq, h0 * qb), off(dk, h0 * qb), off(dv, h0 * vb), 1,
                                                     n, L, d_feat, d_v, io, flags, workspace, workspace_bytes, cuda_stream);
            if (st != BASED_OK) return st;
        }
        return BASED_OK;
    }
    if (io == BASED_BF16)
        return launch_prefill_backward_tc(q, k, v, out, dout, 0, dq, dk, dv, static_cast<float*>(workspace), B * H, L,
                                          d_feat, d_v, (flags & BASED_NUMERATOR_ONLY) ? 1 : 0,
                                          static_cast<cudaStream_t>(cuda_stream));
    return backward_f32(q, k, v, dout, 0, dq, dk, dv, B, H, L, d_v, flags, workspace, workspace_bytes, cuda_stream);
}

based_status based_prefill_backward(const void* q, const void* k, const void* v, const void* dout, void* dq,
                                    void* dk, void* dv, int B, int H, int L, int d_feat, int d_v, based_dtype io,
                                    int flags, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return prefill_backward(q, k, v, nullptr, dout, dq, dk, dv, B, H, L, d_feat, d_v, io, flags, workspace,
                            workspace_bytes, cuda_stream);
}

based_status based_prefill_backward_with_out(const void* q, const void* k, const void* v, const void* out,
                                             const void* dout, void* dq, void* dk, void* dv, int B, int H, int L,
                                             int d_feat, int d_v, based_dtype io, int flags, void* workspace,
                                             size_t workspace_bytes, void* cuda_stream) {
    if (!out || out == dq || out == dk || out == dv) return BASED_ERR_INVALID_ARG;
    return prefill_backward(q, k, v, out, dout, dq, dk, dv, B, H, L, d_feat, d_v, io, flags, workspace,
                            workspace_bytes, cuda_stream);
}

based_status based_prefill_backward_tokens_first(const void* q, const void* k, const void* v, const void* dout, void* dq, void* dk,
                                                 void* dv, int B, int H, int L, int d_feat, int d_v, based_dtype io, int flags,
                                                 void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (!q || !k || !v || !dout || !dq || !dk || !dv || B <= 0 || H <= 0 || L <= 0) return BASED_ERR_INVALID_ARG;
    if (flags & ~BASED_NUMERATOR_ONLY) return BASED_ERR_INVALID_ARG;
    if (dq == q || dq == k || dk == q || dk == k || dv == v || dv == dout) return BASED_ERR_INVALID_ARG;
    // one slab of heads, rows counted in 32 bits
    if (io != BASED_F32 || d_feat != kDFeat || !dv_ok(d_v) || (long long)B * H > kHeadSlab || (long long)B * H * L > 0x7fffffffLL)
        return BASED_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(dout) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv) ||
        !aligned16(workspace))
        return BASED_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < based_prefill_backward_workspace_bytes(B, H, L, d_v, io)) return BASED_ERR_WORKSPACE;
    return backward_f32(q, k, v, dout, H, dq, dk, dv, B, H, L, d_v, flags, workspace, workspace_bytes, cuda_stream);
}

based_status based_prefill_backward_tokens_first_with_out(const void* q, const void* k, const void* v, const void* out,
                                                          const void* dout, void* dq, void* dk, void* dv, int B, int H, int L,
                                                          int d_feat, int d_v, based_dtype io, int flags, void* workspace,
                                                          size_t workspace_bytes, void* cuda_stream) {
    if (!q || !k || !v || !out || !dout || !dq || !dk || !dv || B <= 0 || H <= 0 || L <= 0) return BASED_ERR_INVALID_ARG;
    if (flags & ~BASED_NUMERATOR_ONLY) return BASED_ERR_INVALID_ARG;
    if (dq == q || dq == k || dk == q || dk == k || dv == v || dv == dout || out == dq || out == dk || out == dv) return BASED_ERR_INVALID_ARG;
    // one slab of heads, rows counted in 32 bits
    if (io != BASED_BF16 || !(d_feat == kDFeat || df_generic(d_feat)) || !dv_ok(d_v) || (long long)B * H > kHeadSlab ||
        (long long)B * H * L > 0x7fffffffLL)
        return BASED_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(dout) || !aligned16(dq) || !aligned16(dk) ||
        !aligned16(dv) || !aligned16(workspace))
        return BASED_ERR_ALIGNMENT;
    if (!workspace || workspace_bytes < based_prefill_backward_workspace_bytes(B, H, L, d_v, io)) return BASED_ERR_WORKSPACE;
    return launch_prefill_backward_tc(q, k, v, out, dout, H, dq, dk, dv, static_cast<float*>(workspace), B * H, L, d_feat, d_v,
                                      (flags & BASED_NUMERATOR_ONLY) ? 1 : 0, static_cast<cudaStream_t>(cuda_stream));
}

based_status based_tokens_to_heads(const void* src, void* dst, int B, int H, int L, int row_bytes, void* cuda_stream) {
    if (!src || !dst || src == dst || B <= 0 || H <= 0 || L <= 0 || row_bytes <= 0) return BASED_ERR_INVALID_ARG;
    // one head of one sequence is indexed with 32 bits, heads and sequences by the grid's y and z
    if (row_bytes % 16 || (long long)L * (row_bytes / 16) > 0x7fffffffLL || B > 65535 || H > 65535) return BASED_ERR_UNSUPPORTED;
    if (!aligned16(src) || !aligned16(dst)) return BASED_ERR_ALIGNMENT;
    return launch_tokens_to_heads(src, dst, B, H, L, row_bytes, static_cast<cudaStream_t>(cuda_stream));
}

based_status based_preload_decode(void) {
    unsigned int* err = nullptr;
    based_status st = error_word_ptr(&err);
    if (st == BASED_OK) st = preload_decode();
    if (st == BASED_OK) st = preload_swa_decode();
    if (st == BASED_OK) st = preload_generation_step();
    return st;
}

based_status based_poll_error(void* cuda_stream) {
    if (cudaStreamSynchronize(static_cast<cudaStream_t>(cuda_stream)) != cudaSuccess) return BASED_ERR_CUDA;
    unsigned int word = 0;
    if (cudaMemcpyFromSymbol(&word, g_error_word, sizeof(word)) != cudaSuccess) return BASED_ERR_CUDA;
    if (word != 0) {
        const unsigned int zero = 0;
        if (cudaMemcpyToSymbol(g_error_word, &zero, sizeof(zero)) != cudaSuccess) return BASED_ERR_CUDA;
        return word & 1u ? BASED_ERR_DEVICE_TIMEOUT : BASED_ERR_INVALID_ARG;
    }
    return BASED_OK;
}

}  // extern "C"

namespace based {
based_status prefill_fit_workspace(const void* q, const void* k, const void* v, void* out, float* kv_state, float* z_state,
                                   int B, int H, int L, int d_feat, int d_v, based_dtype io, int flags, void* workspace,
                                   size_t workspace_bytes, void* cuda_stream) {
    return ::prefill_impl(q, k, v, out, kv_state, z_state, B, H, L, d_feat, d_v, io, flags, workspace, workspace_bytes,
                          cuda_stream, true);
}
}  // namespace based
