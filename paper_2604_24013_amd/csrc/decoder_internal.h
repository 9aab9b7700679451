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

// Positions on up to four axes, and the weights of heads that are divided by their root mean square.
struct AxesRotation {
    uint64_t turn[128];
    uint32_t axis_bits[8];                          // of pair j: bits 2 (j % 16), .. + 1 of word j / 16
    int n_axes;
    int rot_dim;                                    // 0: no rotation
    bool interleaved;
    float magnitude;
    int64_t position_axis;                          // between two axes' positions of a token
};
struct NormParams {
    const void *wq, *wk;                            // null: a factor of 1
    bool on, weight_bf16;
    float eps, offset;
};
struct HeadParams {
    AxesRotation rot;
    NormParams norm;
    int head_dim;
    unsigned tokens, heads, kv_heads;
    unsigned lanes, groups, subs_shift;             // lanes of a head; workgroups that share out the heads of some tokens; jobs of a head (their logarithm)
    const void *q, *k;
    void *q_out, *k_out;
    const int32_t *positions;
    int64_t q_token, q_head, k_token, k_head, oq_token, oq_head, ok_token, ok_head;
};
hipError_t launch_norm_rope(const HeadParams &p, bool bf16, hipStream_t s, int num_cu);
// dq_out, dk_out with the strides of q_out, k_out; dq, dk with those of q, k; dwq, dwk: null = not wanted
hipError_t launch_norm_rope_grad(const HeadParams &p, const void *dq_out, const void *dk_out, void *dq, void *dk, float *dwq, float *dwk, float *scratch,
                                 bool bf16, hipStream_t s, int num_cu);
size_t norm_rope_scratch_bytes(int head_dim, unsigned heads);
hipError_t launch_cache_write_norm(const CachePool &c, const CacheRows &r, const AxesRotation &a, const NormParams &n, hipStream_t s, int num_cu);

// A serving step's tables (cf_tables, with the counts resolved).
constexpr int MAX_TABLE_SEQS = 4096;
struct TableParams {
    int n_seqs, page_shift, max_pages, n_pages, max_tokens;
    bool clear_back;
    const int32_t *held, *new_tokens, *back_from, *back_to, *free_count;
    int32_t *page_table, *free_pages, *free_left, *q_start, *kv_len, *positions;
    int64_t *slots;
};
hipError_t launch_step_tables(const TableParams &p, hipStream_t s);

// Causal attention of rows (token, query head of one key head's group) over keys that lie packed (a prompt's own) or in a
// paged cache.  Strides in elements.
struct CausalParams {
    const void *Q;
    void *out;
    float *lse;                                     // [heads][lse_stride], nullable
    int64_t lse_stride;
    int64_t q_token, q_head, o_token, o_head;
    int heads, kv_heads, group;                     // group = heads / kv_heads
    float scale;
    // packed: K, V [tokens], sequences at starts[0 .. n_seqs]
    const void *K, *V;
    int64_t k_token, k_head, v_token, v_head;
    int tokens, n_seqs;
    const int32_t *starts;                          // (paged: of the query rows)
    bool paged;                                     // keys in a cache; else packed
    CachePool pool;
    const int32_t *kv_len, *table;
    int max_q, max_kv, max_pages;
    int window = 0, sinks = 0;                      // a row sees the last `window` keys up to its own and the first `sinks` (0: all up to its own)
    // a walk's tiles split over workgroups
    int items = 0;                                  // workgroups of the launch at the most (0: one for each block and key head)
    int chunk = 0;                                  // tiles of a split (0: as few as the items allow)
    int slots = 0;                                  // where only some walks are long: what is parked at the most
    int whole_from = 0;                             // blocks of a key head that have rows, of which as many are left whole (0: none)
    int num_cu = 0;
    float *parts = nullptr;
    unsigned *counters = nullptr;
    size_t part_bytes = 0;
    int max_counters = 0;
};
// Workgroups of a launch over `blocks` blocks of one key head whose walks are of up to `longest` tiles, and P.items and P.chunk to go with it:
// as many as fit the compute units the least number of times that leaves a third of them over for splits.  `least`: tiles of a split at
// the least (where no walk has half as many more, none is cut); `part`: bytes that a split parks; `counted`: every block needs a counter.
// Without workspace for that, with blocks enough, with more blocks (512) or packed sequences (64) than are looked at, or with walks of more
// than 2^31 tiles together: one workgroup a block.
int64_t plan_items(CausalParams &p, int64_t blocks, int64_t longest, int64_t least, size_t part, bool counted, int num_cu);
// The same for packed rows or keys where there may be a window, whose walks are alike: three quarters or more of the `resident` workgroups that fit the chip
// at once are left whole.  (Of a paged batch's blocks only the tables tell which have rows: `whole_from`.)
int64_t plan_alike(CausalParams &p, int64_t blocks, int64_t longest, int64_t least, size_t part, bool counted, int num_cu, int64_t resident);
hipError_t launch_attn_prompt(const CausalParams &p, hipStream_t s, int num_cu);
hipError_t launch_attn_paged_blocks(const CausalParams &p, hipStream_t s, int num_cu);
bool attn_few_takes(const CausalParams &p);         // few rows of a sequence and key head: the kernel that splits keys over waves
hipError_t launch_attn_few(const CausalParams &p, hipStream_t s, int num_cu);
// The gradient of packed prompts; c.out and c.lse as the forward call left them, dq, dk, dv with the strides of Q, K, V.
struct GradParams {
    CausalParams c;
    const void *dout;
    float *delta;                                   // [heads][lse_stride]
    void *dq, *dk, *dv;
};
hipError_t launch_attn_prompt_grad(const GradParams &p, hipStream_t s, int num_cu);
// Bytes of the partial results that the kernels park for their choice of splits.
size_t attn_prompt_part_bytes(const CausalParams &p, int num_cu);
size_t attn_grad_part_bytes(const CausalParams &p, int num_cu);
size_t attn_few_part_bytes(const CausalParams &p, int num_cu);
size_t attn_paged_blocks_part_bytes(const CausalParams &p, int num_cu);

}  // namespace cf
