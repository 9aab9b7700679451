// Internal declarations of the operators between a decoder layer's projections: rotary positions, the paged cache,
// causal attention.  Not part of the C ABI (that is include/commfuse.h).
#pragma once
#include "cf_internal.h"

namespace cf {

// What the entry points of every translation unit share with commfuse_api.hip.
int fail(int status, const char *fmt, ...);         // sets the calling thread's last error, returns `status`
int num_cu();                                       // compute units of the current device
struct WorkspaceView {                              // the workspace registered for a stream (all null without one)
    unsigned *counters = nullptr;                   // max_counters words, zero between launches
    float *parts = nullptr;
    size_t bytes = 0;                               // of parts
    int max_counters = 0;
};
WorkspaceView workspace_view(hipStream_t s);
constexpr size_t WORKSPACE_HEAD_BYTES = 64 * 1024;  // counters, flags, status word

struct RopeParams {
    uint64_t turn[128];
    int head_dim, rot_dim;
    bool interleaved;
    float cos_factor, sin_factor;                   // magnitude, and with the direction's sign
    const void *x;
    const int32_t *positions;
    void *out;
    unsigned tokens, heads, groups;                 // a thread takes heads g, g + groups, ...
    int64_t x_token, x_head, o_token, o_head;
};
hipError_t launch_rope(const RopeParams &p, bool bf16, hipStream_t s, int num_cu);

// Strides of the pool in elements; *_exp packed [n_pages][kv_heads][page_size].
struct CachePool {
    void *k, *v;
    uint8_t *k_exp, *v_exp;
    bool e4m3;
    int page_shift;                                 // page_size = 1 << page_shift
    int kv_heads, head_dim;
    int64_t n_pages, page_stride, head_stride, token_stride;
};

struct CacheRows {
    const void *q, *k, *v;                          // q: null = none
    void *q_out;
    unsigned tokens, heads;
    int64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;
    const int32_t *positions;
    const int64_t *slots;
    int rot_dim;                                    // 0: no rotation
    bool interleaved;
    float magnitude;
    unsigned groups;                                // a thread takes rows g, g + groups, ... of its token
    uint64_t turn[128];
};
hipError_t launch_cache_write(const CachePool &c, const CacheRows &r, hipStream_t s, int num_cu);
hipError_t launch_cache_read(const CachePool &c, const CacheRows &r, void *K, void *V, hipStream_t s);

}  // namespace cf
