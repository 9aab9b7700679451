// Entry points of the operators between a decoder layer's projections: argument checking and dispatch.
// The contract of every entry point is stated in include/commfuse.h.
#include "../../include/commfuse.h"
#include "decoder_internal.h"

#include <climits>
#include <cmath>
#include <cstring>

namespace {

using cf::fail;

#define CF_FAIL(...) static_cast<cf_status>(fail(__VA_ARGS__))

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// No element twice: n dimensions (count, stride) around rows of `row` elements.
struct Dim {
    int64_t count, stride;
};
bool disjoint(Dim *d, int n, int64_t row)
{
    for (int i = 1; i < n; ++i)                                  // by stride
        for (int j = i; j > 0 && d[j].stride < d[j - 1].stride; --j) {
            const Dim t = d[j];
            d[j] = d[j - 1];
            d[j - 1] = t;
        }
    __int128 extent = row;
    for (int i = 0; i < n; ++i) {
        if (d[i].count <= 1)
            continue;
        if (d[i].stride < extent)
            return false;
        extent += (__int128)(d[i].count - 1) * d[i].stride;
    }
    return extent <= INT64_MAX / 8;
}

// Strides of rows [tokens][heads][head_dim]: 0 = packed.  `mult`: elements of a 16-byte line.
cf_status resolve_rows(const char *what, int64_t *token, int64_t *head, int64_t tokens, int64_t heads, int64_t head_dim, int64_t mult)
{
    if (*token < 0 || *head < 0)
        return CF_FAIL(CF_ERR_INVALID_ARG, "%s: negative stride", what);
    *head = *head ? *head : head_dim;
    *token = *token ? *token : heads * *head;
    Dim d[2] = {{heads, *head}, {tokens, *token}};
    if (tokens > 0 && heads > 0 && !disjoint(d, 2, head_dim))
        return CF_FAIL(CF_ERR_INVALID_ARG, "%s: rows overlap (token stride %lld, head stride %lld)", what, (long long)*token, (long long)*head);
    if (*token % mult || *head % mult)
        return CF_FAIL(CF_ERR_MISALIGNED, "%s: strides must be multiples of %lld elements", what, (long long)mult);
    return CF_OK;
}

cf_status check_rope(const cf_rope *rope)
{
    if (rope == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "rope is NULL");
    if (rope->head_dim < 8 || rope->head_dim > 256 || rope->head_dim % 8 || rope->rot_dim < 2 || rope->rot_dim > rope->head_dim || rope->rot_dim % 2 ||
        (rope->layout != CF_ROPE_HALF && rope->layout != CF_ROPE_INTERLEAVED) || !(rope->magnitude > 0.0f) || !std::isfinite(rope->magnitude))
        return CF_FAIL(CF_ERR_INVALID_ARG, "rope was not filled in by commfuse_rope_make");
    return CF_OK;
}

// The pool with its strides filled in.
cf_status resolve_cache(const cf_cache_desc *d, const cf_cache *c, cf::CachePool *out)
{
    if (d == nullptr || c == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "cache descriptor or cache is NULL");
    if (d->dtype != CF_BF16 && d->dtype != CF_E4M3)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "cache dtype %d", d->dtype);
    if (d->page_size < 16 || d->page_size > 1024 || (d->page_size & (d->page_size - 1)))
        return CF_FAIL(CF_ERR_INVALID_ARG, "page_size = %d must be a power of two in [16, 1024]", d->page_size);
    if (d->kv_heads < 1 || d->kv_heads > 65535 || d->n_pages < 0 || d->n_pages > INT32_MAX)
        return CF_FAIL(CF_ERR_INVALID_ARG, "kv_heads = %d, n_pages = %lld out of range", d->kv_heads, (long long)d->n_pages);
    if (d->head_dim < 16 || d->head_dim > 256 || d->head_dim % 16)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "head_dim %d: the cache takes multiples of 16 up to 256", d->head_dim);
    cf::CachePool p;
    p.e4m3 = d->dtype == CF_E4M3;
    p.page_shift = __builtin_ctz((unsigned)d->page_size);
    p.kv_heads = d->kv_heads;
    p.head_dim = d->head_dim;
    p.n_pages = d->n_pages;
    if (d->page_stride == 0 && d->head_stride == 0 && d->token_stride == 0) {
        p.token_stride = d->head_dim;
        p.head_stride = (int64_t)d->page_size * d->head_dim;
        p.page_stride = p.head_stride * d->kv_heads;
    } else {
        p.page_stride = d->page_stride;
        p.head_stride = d->head_stride;
        p.token_stride = d->token_stride;
    }
    Dim dims[3] = {{d->page_size, p.token_stride}, {d->kv_heads, p.head_stride}, {d->n_pages, p.page_stride}};
    if (p.token_stride < 0 || p.head_stride < 0 || p.page_stride < 0 || !disjoint(dims, 3, d->head_dim))
        return CF_FAIL(CF_ERR_INVALID_ARG, "cache rows overlap (strides: page %lld, head %lld, token %lld)", (long long)p.page_stride,
                       (long long)p.head_stride, (long long)p.token_stride);
    const int64_t mult = p.e4m3 ? 16 : 8;
    if (p.page_stride % mult || p.head_stride % mult || p.token_stride % mult)
        return CF_FAIL(CF_ERR_MISALIGNED, "cache strides must be multiples of %lld elements", (long long)mult);
    // a page of one head is addressed with 32-bit offsets from its first token
    if (p.token_stride > (int64_t)INT32_MAX / 2 / 1024)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "cache token stride %lld", (long long)p.token_stride);
    p.k = c->k;
    p.v = c->v;
    p.k_exp = c->k_exp;
    p.v_exp = c->v_exp;
    if (p.k == nullptr || p.v == nullptr || (p.e4m3 && (p.k_exp == nullptr || p.v_exp == nullptr)))
        return CF_FAIL(CF_ERR_NULL_PTR, "cache tensors must not be NULL");
    if (!aligned(p.k, 16) || !aligned(p.v, 16) || (p.e4m3 && (!aligned(p.k_exp, 8) || !aligned(p.v_exp, 8))))
        return CF_FAIL(CF_ERR_MISALIGNED, "cache tensors must be 16-byte aligned, their exponents 8-byte");
    *out = p;
    return CF_OK;
}

// Tokens and rows of one head in a call, so that the kernels count them in 32 bits.
cf_status check_tokens(int64_t tokens, int64_t rows_of_a_token)
{
    if (tokens < 0)
        return CF_FAIL(CF_ERR_INVALID_ARG, "tokens = %lld", (long long)tokens);
    if (tokens > INT32_MAX / (rows_of_a_token > 0 ? rows_of_a_token : 1))
        return CF_FAIL(CF_ERR_INVALID_ARG, "%lld tokens of %lld rows exceed the 32-bit index range of the kernels", (long long)tokens, (long long)rows_of_a_token);
    return CF_OK;
}

// A tile of 64 rows is addressed with 32-bit offsets from its first.
constexpr int64_t MAX_TOKEN_STRIDE = (int64_t)1 << 23;

cf_status check_scale(float scale)
{
    if (!(scale > 0.0f) || !(scale < 1e30f))
        return CF_FAIL(CF_ERR_INVALID_ARG, "scale must be a positive finite number");
    return CF_OK;
}

void use_workspace(cf::CausalParams &p, hipStream_t s)
{
    const cf::WorkspaceView v = cf::workspace_view(s);
    p.parts = v.parts;
    p.counters = v.counters;
    p.part_bytes = v.bytes;
    p.max_counters = v.max_counters;
}

// The strides of the rows that go into the cache.  `nothing`: no token.
cf_status resolve_cache_rows(const cf::CachePool &c, const cf_cache_rows *rows, bool q_given, cf::CacheRows *out, bool *nothing)
{
    if (rows == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "rows is NULL");
    if (rows->heads < 0 || rows->reserved != 0)
        return CF_FAIL(CF_ERR_INVALID_ARG, "heads = %d, reserved = %d", rows->heads, rows->reserved);
    if (cf_status st = check_tokens(rows->tokens, (int64_t)rows->heads + 2 * c.kv_heads))
        return st;
    cf::CacheRows r = {};
    r.q_token = rows->q_token, r.q_head = rows->q_head, r.k_token = rows->k_token, r.k_head = rows->k_head;
    r.v_token = rows->v_token, r.v_head = rows->v_head, r.o_token = rows->o_token, r.o_head = rows->o_head;
    if (cf_status st = resolve_rows("K", &r.k_token, &r.k_head, rows->tokens, c.kv_heads, c.head_dim, 8))
        return st;
    if (cf_status st = resolve_rows("V", &r.v_token, &r.v_head, rows->tokens, c.kv_heads, c.head_dim, 8))
        return st;
    if (q_given && rows->heads > 0) {
        if (cf_status st = resolve_rows("Q", &r.q_token, &r.q_head, rows->tokens, rows->heads, c.head_dim, 8))
            return st;
        if (cf_status st = resolve_rows("q_out", &r.o_token, &r.o_head, rows->tokens, rows->heads, c.head_dim, 8))
            return st;
    }
    *nothing = rows->tokens == 0;
    *out = r;
    return CF_OK;
}

// ... and their pointers.
cf_status take_cache_rows(const void *Q, const void *K, const void *V, bool rotated, const int32_t *positions, const int64_t *slots, void *q_out,
                          const cf_cache_rows *rows, cf::CacheRows *r)
{
    const bool with_q = Q != nullptr && rows->heads > 0;
    if (K == nullptr || V == nullptr || slots == nullptr || (rotated && positions == nullptr) || (with_q && q_out == nullptr))
        return CF_FAIL(CF_ERR_NULL_PTR, "K, V, slots, with rope positions, with Q q_out must not be NULL");
    if (!aligned(K, 16) || !aligned(V, 16) || (with_q && (!aligned(Q, 16) || !aligned(q_out, 16))) || !aligned(slots, 8) || (rotated && !aligned(positions, 4)))
        return CF_FAIL(CF_ERR_MISALIGNED, "tensor pointers must be 16-byte aligned, slots 8-byte, positions 4-byte");
    if (with_q && Q == q_out && (r->q_token != r->o_token || r->q_head != r->o_head))
        return CF_FAIL(CF_ERR_INVALID_ARG, "in place, Q and q_out must have the same strides");
    r->q = with_q ? Q : nullptr;
    r->k = K;
    r->v = V;
    r->q_out = q_out;
    r->tokens = (unsigned)rows->tokens;
    r->heads = (unsigned)rows->heads;
    r->positions = positions;
    r->slots = slots;
    return CF_OK;
}

// Turns per position, in units of 2^-64, of pair j of a spectrum over `dim` features.
uint64_t turns_of(const cf_rope_desc &d, int dim, int j)
{
    const long double two_pi = 6.283185307179586476925286766559005768L;
    const long double f = powl((long double)d.base, -2.0L * j / dim);
    double r = 0.0;
    if (d.scaling == CF_ROPE_WAVELENGTH) {
        r = ((double)(d.trained_len * f / two_pi) - d.low) / (d.high - d.low);
    } else if (d.scaling == CF_ROPE_INDEX) {
        const double per = dim / (2.0 * std::log(d.base));           // the ramp's ends
        double first = std::floor(per * std::log(d.trained_len / ((double)two_pi * d.high)));
        double last = std::ceil(per * std::log(d.trained_len / ((double)two_pi * d.low)));
        first = first > 0.0 ? first : 0.0;
        last = last < dim - 1 ? last : dim - 1;                      // (it may lie behind the last pair)
        r = 1.0 - (j - first) / (last - first > 0.001 ? last - first : 0.001);
    }
    r = r < 0.0 ? 0.0 : r > 1.0 ? 1.0 : r;
    const long double turns = f * (r + (1.0L - r) / d.factor) / two_pi;              // below 0.16
    return (uint64_t)(turns * 18446744073709551616.0L + 0.5L);
}

// What the kernels take of a rotation by several axes (nullptr: none).
cf_status resolve_axes(const cf_rope_axes *rope, int head_dim, int64_t tokens, int64_t position_axis, cf::AxesRotation *out)
{
    cf::AxesRotation r = {};
    if (rope != nullptr) {
        if (cf_status st = check_rope(&rope->rope))
            return st;
        if (rope->n_axes < 1 || rope->n_axes > 4)
            return CF_FAIL(CF_ERR_INVALID_ARG, "rope was not filled in by commfuse_rope_axes_make");
        if (rope->rope.head_dim != head_dim)
            return CF_FAIL(CF_ERR_INVALID_ARG, "rope turns heads of %d features, these have %d", rope->rope.head_dim, head_dim);
        if (position_axis < 0 || (position_axis > 0 && position_axis < tokens && rope->n_axes > 1))
            return CF_FAIL(CF_ERR_INVALID_ARG, "position_axis = %lld: 0, or at least the %lld tokens", (long long)position_axis, (long long)tokens);
        if (position_axis > INT64_MAX / 32)
            return CF_FAIL(CF_ERR_INVALID_ARG, "position_axis = %lld", (long long)position_axis);
        memcpy(r.turn, rope->rope.turn, sizeof(r.turn));
        for (int j = 0; j < rope->rope.rot_dim / 2; ++j) {
            if (rope->axis[j] >= rope->n_axes)
                return CF_FAIL(CF_ERR_INVALID_ARG, "rope was not filled in by commfuse_rope_axes_make");
            r.axis_bits[j / 16] |= (uint32_t)rope->axis[j] << 2 * (j % 16);
        }
        r.n_axes = rope->n_axes;
        r.rot_dim = rope->rope.rot_dim;
        r.interleaved = rope->rope.layout == CF_ROPE_INTERLEAVED;
        r.magnitude = rope->rope.magnitude;
        r.position_axis = position_axis;
    }
    *out = r;
    return CF_OK;
}

cf_status resolve_norm(const cf_head_norm *norm, const void *wq, const void *wk, cf::NormParams *out)
{
    cf::NormParams n = {};
    if (norm != nullptr) {
        if (norm->weight_dtype != CF_BF16 && norm->weight_dtype != CF_F32)
            return CF_FAIL(CF_ERR_UNSUPPORTED, "weight dtype %d", norm->weight_dtype);
        if (norm->reserved != 0)
            return CF_FAIL(CF_ERR_INVALID_ARG, "reserved = %d", norm->reserved);
        if (!(norm->eps >= 1e-30f) || !std::isfinite(norm->eps) || !std::isfinite(norm->offset))
            return CF_FAIL(CF_ERR_INVALID_ARG, "need a finite eps of at least 1e-30 and a finite offset");
        if (!aligned(wq, 16) || !aligned(wk, 16))
            return CF_FAIL(CF_ERR_MISALIGNED, "weights must be 16-byte aligned");
        n.on = true;
        n.wq = wq;
        n.wk = wk;
        n.weight_bf16 = norm->weight_dtype == CF_BF16;
        n.eps = norm->eps;
        n.offset = norm->offset;
    }
    *out = n;
    return CF_OK;
}

// The rows of commfuse_norm_rope and its gradient.  `nothing`: no row.
cf_status resolve_heads(const cf_rope_axes *rope, const cf_head_norm *norm, const cf_head_rows *rows, const void *wq, const void *wk, int64_t position_axis,
                        cf::HeadParams *out, bool *nothing)
{
    if (rows == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "rows is NULL");
    if (rope == nullptr && norm == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "neither rope nor norm is given");
    if (rows->dtype != CF_BF16 && rows->dtype != CF_F32)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "dtype %d", rows->dtype);
    if (rows->head_dim < 8 || rows->head_dim > 256 || rows->head_dim % 8)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "head_dim %d: multiples of 8 up to 256", rows->head_dim);
    if (rows->heads < 0 || rows->kv_heads < 0)
        return CF_FAIL(CF_ERR_INVALID_ARG, "heads = %d, kv_heads = %d", rows->heads, rows->kv_heads);
    if (cf_status st = check_tokens(rows->tokens, (int64_t)rows->heads + rows->kv_heads))
        return st;
    cf::HeadParams p = {};
    if (cf_status st = resolve_axes(rope, rows->head_dim, rows->tokens, position_axis, &p.rot))
        return st;
    if (cf_status st = resolve_norm(norm, wq, wk, &p.norm))
        return st;
    p.q_token = rows->q_token, p.q_head = rows->q_head, p.k_token = rows->k_token, p.k_head = rows->k_head;
    p.oq_token = rows->oq_token, p.oq_head = rows->oq_head, p.ok_token = rows->ok_token, p.ok_head = rows->ok_head;
    const int64_t mult = rows->dtype == CF_BF16 ? 8 : 4;
    if (cf_status st = resolve_rows("Q", &p.q_token, &p.q_head, rows->tokens, rows->heads, rows->head_dim, mult))
        return st;
    if (cf_status st = resolve_rows("K", &p.k_token, &p.k_head, rows->tokens, rows->kv_heads, rows->head_dim, mult))
        return st;
    if (cf_status st = resolve_rows("q_out", &p.oq_token, &p.oq_head, rows->tokens, rows->heads, rows->head_dim, mult))
        return st;
    if (cf_status st = resolve_rows("k_out", &p.ok_token, &p.ok_head, rows->tokens, rows->kv_heads, rows->head_dim, mult))
        return st;
    p.head_dim = rows->head_dim;
    p.tokens = (unsigned)rows->tokens;
    p.heads = (unsigned)rows->heads;
    p.kv_heads = (unsigned)rows->kv_heads;
    *nothing = rows->tokens == 0 || rows->heads + rows->kv_heads == 0;
    *out = p;
    return CF_OK;
}

// Pointers of the rows of some heads: all there and aligned, and in place only with the same strides.
cf_status check_rows(const char *what, int heads, const void *in, int64_t in_token, int64_t in_head, const void *out, int64_t out_token, int64_t out_head)
{
    if (heads == 0)
        return CF_OK;
    if (in == nullptr || out == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "%s must not be NULL", what);
    if (!aligned(in, 16) || !aligned(out, 16))
        return CF_FAIL(CF_ERR_MISALIGNED, "%s must be 16-byte aligned", what);
    if (in == out && (in_token != out_token || in_head != out_head))
        return CF_FAIL(CF_ERR_INVALID_ARG, "%s: in place, both must have the same strides", what);
    return CF_OK;
}

// The packed prompts' geometry.  `nothing`: no row to compute.
cf_status resolve_prompt(const cf_prompt_desc *d, cf::CausalParams *out, bool *nothing)
{
    if (d == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "descriptor is NULL");
    if (d->n_seqs < 0 || d->heads < 1 || d->kv_heads < 1 || d->reserved != 0)
        return CF_FAIL(CF_ERR_INVALID_ARG, "n_seqs = %d, heads = %d, kv_heads = %d, reserved = %d", d->n_seqs, d->heads, d->kv_heads, d->reserved);
    if (d->heads % d->kv_heads)
        return CF_FAIL(CF_ERR_INVALID_ARG, "kv_heads = %d must divide heads = %d", d->kv_heads, d->heads);
    if (d->head_dim != 128)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "head_dim %d: the attention kernel is written for 128", d->head_dim);
    if (cf_status st = check_tokens(d->tokens, d->heads))
        return st;
    if (d->tokens * d->heads > INT32_MAX - 65536)                // (rows are counted beyond the last by less than this)
        return CF_FAIL(CF_ERR_INVALID_ARG, "%lld tokens of %d heads exceed the 32-bit index range of the kernels", (long long)d->tokens, d->heads);
    if (cf_status st = check_scale(d->scale))
        return st;
    cf::CausalParams p = {};
    p.q_token = d->q_token, p.q_head = d->q_head, p.k_token = d->k_token, p.k_head = d->k_head;
    p.v_token = d->v_token, p.v_head = d->v_head, p.o_token = d->o_token, p.o_head = d->o_head;
    if (cf_status st = resolve_rows("Q", &p.q_token, &p.q_head, d->tokens, d->heads, 128, 8))
        return st;
    if (cf_status st = resolve_rows("K", &p.k_token, &p.k_head, d->tokens, d->kv_heads, 128, 8))
        return st;
    if (cf_status st = resolve_rows("V", &p.v_token, &p.v_head, d->tokens, d->kv_heads, 128, 8))
        return st;
    if (cf_status st = resolve_rows("out", &p.o_token, &p.o_head, d->tokens, d->heads, 128, 8))
        return st;
    if (p.q_token > MAX_TOKEN_STRIDE || p.k_token > MAX_TOKEN_STRIDE || p.v_token > MAX_TOKEN_STRIDE || p.o_token > MAX_TOKEN_STRIDE)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "token strides of more than %lld elements", (long long)MAX_TOKEN_STRIDE);
    p.heads = d->heads;
    p.kv_heads = d->kv_heads;
    p.group = d->heads / d->kv_heads;
    p.scale = d->scale;
    p.tokens = (int)d->tokens;
    p.n_seqs = d->n_seqs;
    p.lse_stride = d->tokens;
    *nothing = d->tokens == 0 || d->n_seqs == 0;
    *out = p;
    return CF_OK;
}

cf_status resolve_paged(const cf_cache_desc *cd, const cf_cache *c, const cf_paged_desc *d, cf::CausalParams *out, bool *nothing)
{
    cf::CausalParams p = {};
    p.paged = true;
    if (cf_status st = resolve_cache(cd, c, &p.pool))
        return st;
    if (d == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "descriptor is NULL");
    if (p.pool.head_dim != 128)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "head_dim %d: the attention kernel is written for 128", p.pool.head_dim);
    if (d->n_seqs < 0 || d->heads < 1 || d->max_q < 0 || d->max_kv < 0 || d->max_pages < 0)
        return CF_FAIL(CF_ERR_INVALID_ARG, "n_seqs = %d, heads = %d, max_q = %d, max_kv = %d, max_pages = %d", d->n_seqs, d->heads, d->max_q, d->max_kv, d->max_pages);
    if (d->heads % p.pool.kv_heads)
        return CF_FAIL(CF_ERR_INVALID_ARG, "the cache's %d key heads must divide heads = %d", p.pool.kv_heads, d->heads);
    if (cf_status st = check_tokens(d->total_q, d->heads))
        return st;
    if (cf_status st = check_scale(d->scale))
        return st;
    if ((int64_t)d->max_q * d->heads > INT32_MAX || d->max_kv > INT32_MAX - 4096)
        return CF_FAIL(CF_ERR_INVALID_ARG, "max_q = %d, max_kv = %d exceed the 32-bit index range of the kernels", d->max_q, d->max_kv);
    p.q_token = d->q_token, p.q_head = d->q_head, p.o_token = d->o_token, p.o_head = d->o_head;
    if (cf_status st = resolve_rows("Q", &p.q_token, &p.q_head, d->total_q, d->heads, 128, 8))
        return st;
    if (cf_status st = resolve_rows("out", &p.o_token, &p.o_head, d->total_q, d->heads, 128, 8))
        return st;
    p.heads = d->heads;
    p.kv_heads = p.pool.kv_heads;
    p.group = d->heads / p.kv_heads;
    p.scale = d->scale;
    p.tokens = (int)d->total_q;
    p.n_seqs = d->n_seqs;
    p.lse_stride = d->total_q;
    p.max_q = d->max_q;
    p.max_pages = d->max_pages;
    const int64_t room = (int64_t)d->max_pages * cd->page_size;
    p.max_kv = p.pool.n_pages == 0 ? 0 : room < d->max_kv ? (int)room : d->max_kv;
    *nothing = d->total_q == 0 || d->n_seqs == 0 || d->max_q == 0;
    *out = p;
    return CF_OK;
}

// The window (nullptr: none) of sequences of up to `longest` tokens; where it hides none of them, the kernels without one.
cf_status resolve_window(const cf_window *w, int64_t longest, cf::CausalParams *p)
{
    if (w == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "window is NULL");
    if (w->window < 1 || w->sinks < 0)
        return CF_FAIL(CF_ERR_INVALID_ARG, "window = %d must be at least 1, sinks = %d at least 0", w->window, w->sinks);
    const bool hides = (int64_t)w->window + w->sinks < longest;
    p->window = hides ? w->window : 0;
    p->sinks = hides ? w->sinks : 0;
    return CF_OK;
}

cf_status launched(hipError_t e, const char *what)
{
    return e == hipSuccess ? CF_OK : CF_FAIL(CF_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace

extern "C" {

cf_status commfuse_rope_make(const cf_rope_desc *d, cf_rope *rope)
{
    if (d == nullptr || rope == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "descriptor or rope is NULL");
    if (d->head_dim < 8 || d->head_dim > 256 || d->head_dim % 8)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "head_dim %d: rotation takes multiples of 8 up to 256", d->head_dim);
    if (d->rot_dim < 2 || d->rot_dim > d->head_dim || d->rot_dim % 2)
        return CF_FAIL(CF_ERR_INVALID_ARG, "rot_dim = %d must be even, in [2, head_dim]", d->rot_dim);
    if (d->layout != CF_ROPE_HALF && d->layout != CF_ROPE_INTERLEAVED)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "layout %d", d->layout);
    if (d->scaling != CF_ROPE_LINEAR && d->scaling != CF_ROPE_WAVELENGTH && d->scaling != CF_ROPE_INDEX)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "scaling %d", d->scaling);
    if (!(d->base > 1.0) || !(d->base <= 1e18) || !(d->factor >= 1.0) || !(d->factor <= 1e9) || !(d->magnitude > 0.0) || !(d->magnitude <= 1e9))
        return CF_FAIL(CF_ERR_INVALID_ARG, "need base in (1, 1e18], factor in [1, 1e9], magnitude in (0, 1e9]");
    if (d->scaling != CF_ROPE_LINEAR && (d->trained_len < 1 || !(d->low > 0.0) || !(d->high > d->low) || !std::isfinite(d->high)))
        return CF_FAIL(CF_ERR_INVALID_ARG, "the ramp needs trained_len >= 1 and 0 < low < high");
    memset(rope, 0, sizeof(*rope));
    rope->head_dim = d->head_dim;
    rope->rot_dim = d->rot_dim;
    rope->layout = d->layout;
    rope->magnitude = (float)d->magnitude;
    for (int j = 0; j < d->rot_dim / 2; ++j)
        rope->turn[j] = turns_of(*d, d->rot_dim, j);
    return CF_OK;
}

cf_status commfuse_rope_axes_make(const cf_rope_desc *d, const cf_axes_desc *axes, cf_rope_axes *rope)
{
    if (axes == nullptr || rope == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "axes or rope is NULL");
    if (axes->n_axes < 1 || axes->n_axes > 4)
        return CF_FAIL(CF_ERR_INVALID_ARG, "n_axes = %d must be in [1, 4]", axes->n_axes);
    if (axes->order != CF_AXES_SECTIONS && axes->order != CF_AXES_INTERLEAVED)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "order %d", axes->order);
    if (axes->spectrum != CF_SPECTRUM_SHARED && axes->spectrum != CF_SPECTRUM_OWN)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "spectrum %d", axes->spectrum);
    cf_rope_axes r;
    memset(&r, 0, sizeof(r));
    if (cf_status st = commfuse_rope_make(d, &r.rope))
        return st;
    const int pairs = d->rot_dim / 2, n = axes->n_axes;
    int64_t all = 0;
    for (int a = 0; a < n; ++a) {
        if (axes->sections[a] < 1)
            return CF_FAIL(CF_ERR_INVALID_ARG, "section %d has %d pairs", a, axes->sections[a]);
        if (a > 0 && axes->order == CF_AXES_INTERLEAVED && axes->sections[a] > pairs / n)
            return CF_FAIL(CF_ERR_INVALID_ARG, "section %d: of %d pairs that %d axes take in turn it cannot have %d", a, pairs, n, axes->sections[a]);
        all += axes->sections[a];
    }
    if (all != pairs)
        return CF_FAIL(CF_ERR_INVALID_ARG, "the sections have %lld pairs, rot_dim %d has %d", (long long)all, d->rot_dim, pairs);
    r.n_axes = n;
    int used[4] = {};
    for (int j = 0, section = 0; j < pairs; ++j) {
        int a = 0;
        if (axes->order == CF_AXES_INTERLEAVED) {
            a = j / n < axes->sections[j % n] ? j % n : 0;
        } else {
            while (used[section] == axes->sections[section])
                ++section;
            a = section;
        }
        r.axis[j] = (uint8_t)a;
        if (axes->spectrum == CF_SPECTRUM_OWN)
            r.rope.turn[j] = turns_of(*d, 2 * axes->sections[a], used[a]);
        ++used[a];
    }
    *rope = r;
    return CF_OK;
}

cf_status commfuse_rope(const cf_rope *rope, const cf_rope_rows *rows, const void *x, const int32_t *positions, void *out, int gradient,
                        void *hip_stream)
{
    if (cf_status st = check_rope(rope))
        return st;
    if (rows == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "rows is NULL");
    if (rows->dtype != CF_BF16 && rows->dtype != CF_F32)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "dtype %d", rows->dtype);
    if (rows->heads < 0)
        return CF_FAIL(CF_ERR_INVALID_ARG, "heads = %d", rows->heads);
    if (cf_status st = check_tokens(rows->tokens, rows->heads))
        return st;
    const bool bf16 = rows->dtype == CF_BF16;
    cf::RopeParams p;
    p.x_token = rows->x_token;
    p.x_head = rows->x_head;
    p.o_token = rows->o_token;
    p.o_head = rows->o_head;
    if (cf_status st = resolve_rows("x", &p.x_token, &p.x_head, rows->tokens, rows->heads, rope->head_dim, bf16 ? 8 : 4))
        return st;
    if (cf_status st = resolve_rows("out", &p.o_token, &p.o_head, rows->tokens, rows->heads, rope->head_dim, bf16 ? 8 : 4))
        return st;
    if (rows->tokens == 0 || rows->heads == 0)
        return CF_OK;
    if (x == nullptr || positions == nullptr || out == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "x, positions and out must not be NULL");
    if (!aligned(x, 16) || !aligned(out, 16) || !aligned(positions, 4))
        return CF_FAIL(CF_ERR_MISALIGNED, "tensor pointers must be 16-byte aligned, positions 4-byte");
    if (x == out && (p.x_token != p.o_token || p.x_head != p.o_head))
        return CF_FAIL(CF_ERR_INVALID_ARG, "in place, x and out must have the same strides");
    memcpy(p.turn, rope->turn, sizeof(p.turn));
    p.head_dim = rope->head_dim;
    p.rot_dim = rope->rot_dim;
    p.interleaved = rope->layout == CF_ROPE_INTERLEAVED;
    p.cos_factor = rope->magnitude;
    p.sin_factor = gradient ? -rope->magnitude : rope->magnitude;
    p.x = x;
    p.positions = positions;
    p.out = out;
    p.tokens = (unsigned)rows->tokens;
    p.heads = (unsigned)rows->heads;
    return launched(cf::launch_rope(p, bf16, static_cast<hipStream_t>(hip_stream), cf::num_cu()), "rotation launch");
}

cf_status commfuse_cache_write(const cf_cache_desc *desc, const cf_cache *cache, const cf_cache_rows *rows, const cf_rope *rope,
                               const void *Q, const void *K, const void *V, const int32_t *positions, const int64_t *slots,
                               void *q_out, void *hip_stream)
{
    cf::CachePool c;
    cf::CacheRows r;
    bool nothing;
    if (cf_status st = resolve_cache(desc, cache, &c))
        return st;
    if (rope != nullptr) {
        if (cf_status st = check_rope(rope))
            return st;
        if (rope->head_dim != c.head_dim)
            return CF_FAIL(CF_ERR_INVALID_ARG, "rope turns heads of %d features, the cache has %d", rope->head_dim, c.head_dim);
        if (rope->rot_dim % 16)
            return CF_FAIL(CF_ERR_UNSUPPORTED, "rot_dim %d: the cache's writer takes multiples of 16 (rotate with commfuse_rope first)", rope->rot_dim);
    }
    if (cf_status st = resolve_cache_rows(c, rows, Q != nullptr, &r, &nothing))
        return st;
    if (Q != nullptr && rows->heads > 0 && rope == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "Q is given, but no rope to rotate it by");
    if (nothing)
        return CF_OK;
    if (cf_status st = take_cache_rows(Q, K, V, rope != nullptr, positions, slots, q_out, rows, &r))
        return st;
    if (rope != nullptr) {
        r.rot_dim = rope->rot_dim;
        r.interleaved = rope->layout == CF_ROPE_INTERLEAVED;
        r.magnitude = rope->magnitude;
        memcpy(r.turn, rope->turn, sizeof(r.turn));
    }
    return launched(cf::launch_cache_write(c, r, static_cast<hipStream_t>(hip_stream), cf::num_cu()), "cache write launch");
}

cf_status commfuse_cache_read(const cf_cache_desc *desc, const cf_cache *cache, const cf_cache_rows *rows, const int64_t *slots,
                              void *K, void *V, void *hip_stream)
{
    cf::CachePool c;
    if (cf_status st = resolve_cache(desc, cache, &c))
        return st;
    if (rows == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "rows is NULL");
    if (rows->reserved != 0)
        return CF_FAIL(CF_ERR_INVALID_ARG, "reserved = %d", rows->reserved);
    if (cf_status st = check_tokens(rows->tokens, 2 * c.kv_heads))
        return st;
    cf::CacheRows r = {};
    r.k_token = rows->k_token, r.k_head = rows->k_head, r.v_token = rows->v_token, r.v_head = rows->v_head;
    if (cf_status st = resolve_rows("K", &r.k_token, &r.k_head, rows->tokens, c.kv_heads, c.head_dim, 8))
        return st;
    if (cf_status st = resolve_rows("V", &r.v_token, &r.v_head, rows->tokens, c.kv_heads, c.head_dim, 8))
        return st;
    if (rows->tokens == 0)
        return CF_OK;
    if (K == nullptr || V == nullptr || slots == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "K, V and slots must not be NULL");
    if (!aligned(K, 16) || !aligned(V, 16) || !aligned(slots, 8))
        return CF_FAIL(CF_ERR_MISALIGNED, "tensor pointers must be 16-byte aligned, slots 8-byte");
    r.tokens = (unsigned)rows->tokens;
    r.slots = slots;
    return launched(cf::launch_cache_read(c, r, K, V, static_cast<hipStream_t>(hip_stream)), "cache read launch");
}

cf_status commfuse_norm_rope(const cf_rope_axes *rope, const cf_head_norm *norm, const cf_head_rows *rows, const void *Q, const void *K, const void *wq,
                             const void *wk, const int32_t *positions, int64_t position_axis, void *q_out, void *k_out, void *hip_stream)
{
    cf::HeadParams p;
    bool nothing;
    if (cf_status st = resolve_heads(rope, norm, rows, wq, wk, position_axis, &p, &nothing))
        return st;
    if (nothing)
        return CF_OK;
    if (rope != nullptr && (positions == nullptr || !aligned(positions, 4)))
        return CF_FAIL(positions == nullptr ? CF_ERR_NULL_PTR : CF_ERR_MISALIGNED, "positions must not be NULL, and 4-byte aligned");
    if (cf_status st = check_rows("Q and q_out", rows->heads, Q, p.q_token, p.q_head, q_out, p.oq_token, p.oq_head))
        return st;
    if (cf_status st = check_rows("K and k_out", rows->kv_heads, K, p.k_token, p.k_head, k_out, p.ok_token, p.ok_head))
        return st;
    p.q = Q;
    p.k = K;
    p.q_out = q_out;
    p.k_out = k_out;
    p.positions = positions;
    return launched(cf::launch_norm_rope(p, rows->dtype == CF_BF16, static_cast<hipStream_t>(hip_stream), cf::num_cu()), "norm and rotation launch");
}

size_t commfuse_norm_rope_scratch_bytes(const cf_head_rows *rows)
{
    if (rows == nullptr || rows->head_dim < 8 || rows->head_dim > 256 || rows->heads < 0 || rows->kv_heads < 0)
        return 0;
    return cf::norm_rope_scratch_bytes(rows->head_dim, (unsigned)rows->heads + (unsigned)rows->kv_heads);
}

cf_status commfuse_norm_rope_grad(const cf_rope_axes *rope, const cf_head_norm *norm, const cf_head_rows *rows, const void *Q, const void *K, const void *wq,
                                  const void *wk, const int32_t *positions, int64_t position_axis, const void *dq_out, const void *dk_out, void *dQ, void *dK,
                                  float *dwq, float *dwk, void *scratch, void *hip_stream)
{
    cf::HeadParams p;
    bool nothing;
    if (cf_status st = resolve_heads(rope, norm, rows, wq, wk, position_axis, &p, &nothing))
        return st;
    if (norm == nullptr && (dwq != nullptr || dwk != nullptr))
        return CF_FAIL(CF_ERR_INVALID_ARG, "without norm there are no weights: dwq and dwk must be NULL");
    if (!aligned(dwq, 4) || !aligned(dwk, 4) || !aligned(scratch, 16))
        return CF_FAIL(CF_ERR_MISALIGNED, "dwq and dwk must be 4-byte aligned, scratch 16-byte");
    if ((dwq != nullptr || dwk != nullptr) && scratch == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "dwq and dwk need scratch");
    if (dwq != nullptr && dwq == dwk)
        return CF_FAIL(CF_ERR_INVALID_ARG, "dwq and dwk may not alias each other");
    if (nothing && dwq == nullptr && dwk == nullptr)
        return CF_OK;
    if (!nothing) {
        if (rope != nullptr && (positions == nullptr || !aligned(positions, 4)))
            return CF_FAIL(positions == nullptr ? CF_ERR_NULL_PTR : CF_ERR_MISALIGNED, "positions must not be NULL, and 4-byte aligned");
        if (cf_status st = check_rows("dq_out and dQ", rows->heads, dq_out, p.oq_token, p.oq_head, dQ, p.q_token, p.q_head))
            return st;
        if (cf_status st = check_rows("dk_out and dK", rows->kv_heads, dk_out, p.ok_token, p.ok_head, dK, p.k_token, p.k_head))
            return st;
        if (norm != nullptr) {
            if (cf_status st = check_rows("Q and dQ", rows->heads, Q, p.q_token, p.q_head, dQ, p.q_token, p.q_head))
                return st;
            if (cf_status st = check_rows("K and dK", rows->kv_heads, K, p.k_token, p.k_head, dK, p.k_token, p.k_head))
                return st;
        }
    }
    p.q = Q;
    p.k = K;
    p.positions = positions;
    return launched(cf::launch_norm_rope_grad(p, dq_out, dk_out, dQ, dK, dwq, dwk, static_cast<float *>(scratch), rows->dtype == CF_BF16,
                                              static_cast<hipStream_t>(hip_stream), cf::num_cu()), "norm and rotation gradient launch");
}

cf_status commfuse_cache_write_norm(const cf_cache_desc *desc, const cf_cache *cache, const cf_cache_rows *rows, const cf_rope_axes *rope,
                                    const cf_head_norm *norm, const void *Q, const void *K, const void *V, const void *wq, const void *wk,
                                    const int32_t *positions, int64_t position_axis, const int64_t *slots, void *q_out, void *hip_stream)
{
    cf::CachePool c;
    cf::CacheRows r;
    bool nothing;
    if (cf_status st = resolve_cache(desc, cache, &c))
        return st;
    if (rope == nullptr && norm == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "neither rope nor norm is given");
    if (cf_status st = resolve_cache_rows(c, rows, Q != nullptr, &r, &nothing))
        return st;
    cf::AxesRotation a;
    cf::NormParams n;
    if (cf_status st = resolve_axes(rope, c.head_dim, rows->tokens, position_axis, &a))
        return st;
    if (a.rot_dim % 16)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "rot_dim %d: the cache's writer takes multiples of 16 (rotate with commfuse_norm_rope first)", a.rot_dim);
    if (cf_status st = resolve_norm(norm, wq, wk, &n))
        return st;
    if (nothing)
        return CF_OK;
    if (cf_status st = take_cache_rows(Q, K, V, rope != nullptr, positions, slots, q_out, rows, &r))
        return st;
    return launched(cf::launch_cache_write_norm(c, r, a, n, static_cast<hipStream_t>(hip_stream), cf::num_cu()), "cache write launch");
}

cf_status commfuse_step_tables(const cf_tables_desc *d, const cf_tables *t, void *hip_stream)
{
    if (d == nullptr || t == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "descriptor or tables is NULL");
    if (d->page_size < 16 || d->page_size > 1024 || (d->page_size & (d->page_size - 1)))
        return CF_FAIL(CF_ERR_INVALID_ARG, "page_size = %d must be a power of two in [16, 1024]", d->page_size);
    if (d->n_seqs < 0 || d->max_pages < 0 || (d->clear_back != 0 && d->clear_back != 1) || d->n_pages < 0 || d->n_pages > INT32_MAX || d->max_tokens < 0 || d->max_tokens > INT32_MAX - 1024)
        return CF_FAIL(CF_ERR_INVALID_ARG, "n_seqs = %d, max_pages = %d, clear_back = %d, n_pages = %lld, max_tokens = %lld", d->n_seqs, d->max_pages, d->clear_back,
                       (long long)d->n_pages, (long long)d->max_tokens);
    if (d->n_seqs > cf::MAX_TABLE_SEQS)
        return CF_FAIL(CF_ERR_UNSUPPORTED, "n_seqs = %d: the kernel keeps the sums of up to %d sequences", d->n_seqs, cf::MAX_TABLE_SEQS);
    const bool seqs = d->n_seqs > 0, table = seqs && d->max_pages > 0;
    if (t->free_count == nullptr || t->free_left == nullptr || t->q_start == nullptr || (seqs && (t->held == nullptr || t->new_tokens == nullptr || t->kv_len == nullptr)) ||
        (table && t->page_table == nullptr) || (d->n_pages > 0 && t->free_pages == nullptr) || (d->max_tokens > 0 && (t->slots == nullptr || t->positions == nullptr)))
        return CF_FAIL(CF_ERR_NULL_PTR, "tables must not be NULL but for back_from and back_to");
    if ((t->back_from == nullptr) != (t->back_to == nullptr))
        return CF_FAIL(CF_ERR_NULL_PTR, "back_from and back_to go together");
    for (const void *x : {static_cast<const void *>(t->held), static_cast<const void *>(t->new_tokens), static_cast<const void *>(t->back_from),
                          static_cast<const void *>(t->back_to), static_cast<const void *>(t->page_table), static_cast<const void *>(t->free_pages),
                          static_cast<const void *>(t->free_count), static_cast<const void *>(t->free_left), static_cast<const void *>(t->q_start),
                          static_cast<const void *>(t->kv_len), static_cast<const void *>(t->positions)})
        if (!aligned(x, 4))
            return CF_FAIL(CF_ERR_MISALIGNED, "tables must be 4-byte aligned, slots 8-byte");
    if (!aligned(t->slots, 8))
        return CF_FAIL(CF_ERR_MISALIGNED, "tables must be 4-byte aligned, slots 8-byte");
    if (seqs && (t->kv_len == t->held || t->kv_len == t->new_tokens || t->q_start == t->held || t->q_start == t->new_tokens))
        return CF_FAIL(CF_ERR_INVALID_ARG, "q_start and kv_len may not alias held or new_tokens");
    cf::TableParams p;
    p.n_seqs = d->n_seqs;
    p.page_shift = __builtin_ctz((unsigned)d->page_size);
    p.max_pages = d->max_pages;
    p.n_pages = (int)d->n_pages;
    p.max_tokens = (int)d->max_tokens;
    p.clear_back = d->clear_back != 0;
    p.held = t->held;
    p.new_tokens = t->new_tokens;
    p.back_from = t->back_from;
    p.back_to = t->back_to;
    p.free_count = t->free_count;
    p.page_table = t->page_table;
    p.free_pages = t->free_pages;
    p.free_left = t->free_left;
    p.q_start = t->q_start;
    p.kv_len = t->kv_len;
    p.positions = t->positions;
    p.slots = t->slots;
    return launched(cf::launch_step_tables(p, static_cast<hipStream_t>(hip_stream)), "tables launch");
}

namespace {

// Packed prompts, with a window or without.
cf_status attn_prompt(const cf_prompt_desc *desc, bool with_window, const cf_window *window, const void *Q, const void *K, const void *V, const int32_t *seq_start,
                      void *out, float *lse, void *hip_stream)
{
    cf::CausalParams p;
    bool nothing;
    if (cf_status st = resolve_prompt(desc, &p, &nothing))
        return st;
    if (with_window)
        if (cf_status st = resolve_window(window, p.tokens, &p))
            return st;
    if (nothing)
        return CF_OK;
    if (Q == nullptr || K == nullptr || V == nullptr || seq_start == nullptr || out == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "Q, K, V, seq_start and out must not be NULL");
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(seq_start, 4))
        return CF_FAIL(CF_ERR_MISALIGNED, "tensor pointers must be 16-byte aligned, lse and seq_start 4-byte");
    if (out == Q || out == K || out == V)
        return CF_FAIL(CF_ERR_INVALID_ARG, "out may not alias an operand");
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    p.Q = Q;
    p.K = K;
    p.V = V;
    p.starts = seq_start;
    p.out = out;
    p.lse = lse;
    use_workspace(p, s);
    return launched(cf::launch_attn_prompt(p, s, cf::num_cu()), "attention launch");
}

cf_status attn_prompt_grad(const cf_prompt_desc *desc, bool with_window, const cf_window *window, const void *Q, const void *K, const void *V, const void *out,
                           const float *lse, const void *dout, const int32_t *seq_start, float *delta, void *dQ, void *dK, void *dV, void *hip_stream)
{
    cf::GradParams p = {};
    bool nothing;
    if (cf_status st = resolve_prompt(desc, &p.c, &nothing))
        return st;
    if (with_window)
        if (cf_status st = resolve_window(window, p.c.tokens, &p.c))
            return st;
    if (nothing)
        return CF_OK;
    const void *const in[] = {Q, K, V, out, lse, dout, seq_start};
    const void *const result[] = {dQ, dK, dV, delta};
    for (const void *x : in)
        if (x == nullptr)
            return CF_FAIL(CF_ERR_NULL_PTR, "Q, K, V, out, lse, dout and seq_start must not be NULL");
    for (const void *x : result)
        if (x == nullptr)
            return CF_FAIL(CF_ERR_NULL_PTR, "delta, dQ, dK and dV must not be NULL");
    for (const void *x : {Q, K, V, out, dout, static_cast<const void *>(dQ), static_cast<const void *>(dK), static_cast<const void *>(dV)})
        if (!aligned(x, 16))
            return CF_FAIL(CF_ERR_MISALIGNED, "tensor pointers must be 16-byte aligned");
    if (!aligned(lse, 4) || !aligned(delta, 4) || !aligned(seq_start, 4))
        return CF_FAIL(CF_ERR_MISALIGNED, "lse, delta and seq_start must be 4-byte aligned");
    for (int i = 0; i < 4; ++i) {
        for (const void *x : in)
            if (result[i] == x)
                return CF_FAIL(CF_ERR_INVALID_ARG, "delta, dQ, dK and dV may not alias an operand");
        for (int j = 0; j < i; ++j)
            if (result[i] == result[j])
                return CF_FAIL(CF_ERR_INVALID_ARG, "delta, dQ, dK and dV may not alias each other");
    }
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    p.c.Q = Q;
    p.c.K = K;
    p.c.V = V;
    p.c.out = const_cast<void *>(out);                           // (read only, as lse)
    p.c.lse = const_cast<float *>(lse);
    p.c.starts = seq_start;
    p.dout = dout;
    p.delta = delta;
    p.dq = dQ;
    p.dk = dK;
    p.dv = dV;
    use_workspace(p.c, s);
    return launched(cf::launch_attn_prompt_grad(p, s, cf::num_cu()), "attention gradient launch");
}

size_t attn_prompt_workspace_bytes(const cf_prompt_desc *desc, bool with_window, const cf_window *window)
{
    cf::CausalParams p;
    bool nothing;
    if (resolve_prompt(desc, &p, &nothing) != CF_OK || nothing || (with_window && resolve_window(window, p.tokens, &p) != CF_OK))
        return 0;
    const size_t parts = cf::attn_prompt_part_bytes(p, cf::num_cu());
    return parts > 0 ? cf::WORKSPACE_HEAD_BYTES + parts : 0;
}

cf_status attn_paged(const cf_cache_desc *cache_desc, const cf_cache *cache, const cf_paged_desc *desc, bool with_window, const cf_window *window, const void *Q,
                     const int32_t *q_start, const int32_t *kv_len, const int32_t *page_table, void *out, float *lse, void *hip_stream)
{
    cf::CausalParams p;
    bool nothing;
    if (cf_status st = resolve_paged(cache_desc, cache, desc, &p, &nothing))
        return st;
    if (with_window)
        if (cf_status st = resolve_window(window, p.max_kv, &p))
            return st;
    if (nothing)
        return CF_OK;
    if (Q == nullptr || q_start == nullptr || kv_len == nullptr || (page_table == nullptr && desc->max_pages > 0) || out == nullptr)
        return CF_FAIL(CF_ERR_NULL_PTR, "Q, q_start, kv_len, page_table and out must not be NULL");
    if (!aligned(Q, 16) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(q_start, 4) || !aligned(kv_len, 4) || !aligned(page_table, 4))
        return CF_FAIL(CF_ERR_MISALIGNED, "tensor pointers must be 16-byte aligned, lse and the tables 4-byte");
    if (out == Q || out == p.pool.k || out == p.pool.v)
        return CF_FAIL(CF_ERR_INVALID_ARG, "out may not alias an operand");
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    p.Q = Q;
    p.starts = q_start;
    p.kv_len = kv_len;
    p.table = page_table;
    p.out = out;
    p.lse = lse;
    use_workspace(p, s);
    return launched(cf::attn_few_takes(p) ? cf::launch_attn_few(p, s, cf::num_cu()) : cf::launch_attn_paged_blocks(p, s, cf::num_cu()), "attention launch");
}

size_t attn_paged_workspace_bytes(const cf_cache_desc *cache_desc, const cf_paged_desc *desc, bool with_window, const cf_window *window)
{
    cf_cache any = {};
    any.k = any.v = any.k_exp = any.v_exp = reinterpret_cast<uint8_t *>(256);      // (of the pool's geometry, addresses are not looked at)
    cf::CausalParams p;
    bool nothing;
    if (resolve_paged(cache_desc, &any, desc, &p, &nothing) != CF_OK || nothing || (with_window && resolve_window(window, p.max_kv, &p) != CF_OK))
        return 0;
    const size_t parts = cf::attn_few_takes(p) ? cf::attn_few_part_bytes(p, cf::num_cu()) : cf::attn_paged_blocks_part_bytes(p, cf::num_cu());
    return parts > 0 ? cf::WORKSPACE_HEAD_BYTES + parts : 0;
}

}  // namespace

cf_status commfuse_attn_prompt(const cf_prompt_desc *desc, const void *Q, const void *K, const void *V, const int32_t *seq_start, void *out, float *lse, void *hip_stream)
{
    return attn_prompt(desc, false, nullptr, Q, K, V, seq_start, out, lse, hip_stream);
}

cf_status commfuse_attn_prompt_window(const cf_prompt_desc *desc, const cf_window *window, const void *Q, const void *K, const void *V, const int32_t *seq_start,
                                      void *out, float *lse, void *hip_stream)
{
    return attn_prompt(desc, true, window, Q, K, V, seq_start, out, lse, hip_stream);
}

cf_status commfuse_attn_prompt_grad(const cf_prompt_desc *desc, const void *Q, const void *K, const void *V, const void *out, const float *lse, const void *dout,
                                    const int32_t *seq_start, float *delta, void *dQ, void *dK, void *dV, void *hip_stream)
{
    return attn_prompt_grad(desc, false, nullptr, Q, K, V, out, lse, dout, seq_start, delta, dQ, dK, dV, hip_stream);
}

cf_status commfuse_attn_prompt_window_grad(const cf_prompt_desc *desc, const cf_window *window, const void *Q, const void *K, const void *V, const void *out,
                                           const float *lse, const void *dout, const int32_t *seq_start, float *delta, void *dQ, void *dK, void *dV, void *hip_stream)
{
    return attn_prompt_grad(desc, true, window, Q, K, V, out, lse, dout, seq_start, delta, dQ, dK, dV, hip_stream);
}

size_t commfuse_attn_prompt_workspace_bytes(const cf_prompt_desc *desc) { return attn_prompt_workspace_bytes(desc, false, nullptr); }

size_t commfuse_attn_prompt_window_workspace_bytes(const cf_prompt_desc *desc, const cf_window *window) { return attn_prompt_workspace_bytes(desc, true, window); }

cf_status commfuse_attn_paged(const cf_cache_desc *cache_desc, const cf_cache *cache, const cf_paged_desc *desc, const void *Q, const int32_t *q_start,
                              const int32_t *kv_len, const int32_t *page_table, void *out, float *lse, void *hip_stream)
{
    return attn_paged(cache_desc, cache, desc, false, nullptr, Q, q_start, kv_len, page_table, out, lse, hip_stream);
}

cf_status commfuse_attn_paged_window(const cf_cache_desc *cache_desc, const cf_cache *cache, const cf_paged_desc *desc, const cf_window *window, const void *Q,
                                     const int32_t *q_start, const int32_t *kv_len, const int32_t *page_table, void *out, float *lse, void *hip_stream)
{
    return attn_paged(cache_desc, cache, desc, true, window, Q, q_start, kv_len, page_table, out, lse, hip_stream);
}

size_t commfuse_attn_paged_workspace_bytes(const cf_cache_desc *cache_desc, const cf_paged_desc *desc)
{
    return attn_paged_workspace_bytes(cache_desc, desc, false, nullptr);
}

size_t commfuse_attn_paged_window_workspace_bytes(const cf_cache_desc *cache_desc, const cf_paged_desc *desc, const cf_window *window)
{
    return attn_paged_workspace_bytes(cache_desc, desc, true, window);
}

}  // extern "C"
