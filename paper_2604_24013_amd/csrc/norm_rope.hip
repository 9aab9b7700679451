// Every head of Q and K divided by its root mean square, times a weight, and rotated by positions on several axes; the gradient of that; the
// same on the way into the paged cache.
//   r = (mean x^2 + eps)^-1/2,  n = r x,  y = R (n (offset + w))
//   g = R^T dy,  dw = sum over tokens and heads of g n,  h = g (offset + w),  dx = r (h - n mean(h n))
//
// Bound by HBM: forward every feature is read and written once, backward x and dy are read and dx is written.  A thread owns a unit of one
// head (W rotated pairs, or 2 W features that are copied), the lanes of a head are neighbours, a power of two of them, and add up its
// squares by moves inside the wave.  Nothing is kept for the gradient: r costs less to compute again than to read, since x is read in any
// case.  Weights, angles and the weights' gradients of a unit stay in its thread's registers over the heads and tokens that it takes.
// The gradients of the weights are sums over all tokens: every workgroup leaves one for each of its columns in the caller's scratch
// memory, and a second launch adds those up in order.  No atomics: the same call gives the same bits.
#include "rope_units.h"

namespace cf {
namespace {

// Cosine and sine of the W pairs from `j` on, of which each has an axis of its own: two bits of `axis`.
template <int W>
__device__ __forceinline__ void angles_of_axes(const AxesRotation &R, int j, const int32_t *positions, unsigned token, float sign, float (&c)[W], float (&s)[W])
{
    int32_t p[4];
#pragma unroll
    for (int a = 0; a < 4; ++a)
        p[a] = a < R.n_axes ? positions[a * R.position_axis + token] : 0;
    const unsigned which = R.axis_bits[j >> 4] >> 2 * (j & 15);      // (W divides 16: a unit's pairs lie in one word)
    const float factor = R.magnitude;
#pragma unroll
    for (int e = 0; e < W; ++e) {
        const unsigned a = which >> 2 * e & 3;
        const int32_t position = a & 2 ? (a & 1 ? p[3] : p[2]) : (a & 1 ? p[1] : p[0]);
        float ce[1], se[1];
        angles<1>(R.turn, j + e, position, factor, sign * factor, ce, se);
        c[e] = ce[0];
        s[e] = se[0];
    }
}

// Sum over the `lanes` neighbouring lanes (a power of two) of a head; every one of them gets it.
__device__ __forceinline__ float sum_of_lanes(float x, unsigned lanes)
{
    auto moved = [](float y, auto control) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, y), decltype(control)::value, 0xf, 0xf, true));
    };
    if (lanes > 1)
        x += moved(x, std::integral_constant<int, 0xB1>{});          // from the other lane of a pair
    if (lanes > 2)
        x += moved(x, std::integral_constant<int, 0x4E>{});          // ... pair of four
    if (lanes > 4)
        x += moved(x, std::integral_constant<int, 0x141>{});         // ... four of eight (mirrored)
    if (lanes > 8)
        x += moved(x, std::integral_constant<int, 0x140>{});         // ... eight of sixteen (mirrored)
    if (lanes > 16)
        x += __shfl_xor(x, 16);
    if (lanes > 32)
        x += __shfl_xor(x, 32);
    return x;
}

// One over the root mean square of a head's features, of which a lane holds N.  Squares of more than 2^128 together: scaled down first.
template <int N>
__device__ __forceinline__ float inverse_root(const float (&x)[N], unsigned lanes, int head_dim, float eps)
{
    float ss = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e)
        ss = __builtin_fmaf(x[e], x[e], ss);
    ss = sum_of_lanes(ss, lanes);
    const float inv_dim = 1.0f / head_dim;
    float r = 1.0f / sqrtf(__builtin_fmaf(ss, inv_dim, eps));
    if (ss == INFINITY) {                                            // (the same in all lanes of a head)
        float small = 0.0f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float y = x[e] * 0x1p-70f;
            small = __builtin_fmaf(y, y, small);
        }
        r = 0x1p-70f / sqrtf(sum_of_lanes(small, lanes) * inv_dim);
    }
    return r;
}

// The weights of a thread's units, as factors: (offset + w), or 1 without weights.
template <int W, int PER>
__device__ __forceinline__ void load_factors(const NormParams &N, const void *w, const Unit (&at)[PER], const bool (&mine)[PER], float (&f)[PER][2 * W])
{
#pragma unroll
    for (int k = 0; k < PER; ++k)
#pragma unroll
        for (int e = 0; e < 2 * W; ++e) {
            const int i = e < W ? at[k].a + e : at[k].b + e - W;
            f[k][e] = !mine[k] ? 0.0f : w == nullptr ? 1.0f : N.offset + (N.weight_bf16 ? (float)static_cast<const __bf16 *>(w)[i] : static_cast<const float *>(w)[i]);
        }
}

// What every kernel here has of its thread: the lane of a head, and its units (PER, `lanes` apart; those behind the head's last are not there).
template <int W, int PER>
struct HeadLane {
    unsigned lanes, u;
    Unit at[PER];
    bool mine[PER];
    __device__ __forceinline__ HeadLane(unsigned lanes_, int head_dim, int rot_dim, bool interleaved) : lanes(lanes_), u(threadIdx.x & (lanes_ - 1))
    {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            mine[k] = (u + k * lanes) * 2 * W < (unsigned)head_dim;
            at[k] = unit_at<W>(mine[k] ? u + k * lanes : 0, rot_dim, interleaved);
        }
    }
};

template <typename T, int W, int PER>
__device__ __forceinline__ void load_units(const T *row, const HeadLane<W, PER> &L, float (&v)[PER][2 * W])
{
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        if (L.mine[k])
            load_unit<T, W>(row, L.at[k], v[k]);
        else
#pragma unroll
            for (int e = 0; e < 2 * W; ++e)
                v[k][e] = 0.0f;
    }
}
template <typename T, int W, int PER>
__device__ __forceinline__ void store_units(T *row, const HeadLane<W, PER> &L, const float (&v)[PER][2 * W])
{
#pragma unroll
    for (int k = 0; k < PER; ++k)
        if (L.mine[k])
            store_unit<T, W>(row, L.at[k], v[k]);
}
template <int W, int PER>
__device__ __forceinline__ void find_angles(const AxesRotation &R, const HeadLane<W, PER> &L, const int32_t *positions, unsigned token, float sign, float (&c)[PER][W],
                                            float (&s)[PER][W])
{
#pragma unroll
    for (int k = 0; k < PER; ++k)
        if (L.mine[k] && L.at[k].rotated)
            angles_of_axes<W>(R, L.at[k].pair, positions, token, sign, c[k], s[k]);
}
template <int W, int PER>
__device__ __forceinline__ void turn_units(const HeadLane<W, PER> &L, float (&v)[PER][2 * W], const float (&c)[PER][W], const float (&s)[PER][W], bool interleaved)
{
#pragma unroll
    for (int k = 0; k < PER; ++k)
        if (L.mine[k] && L.at[k].rotated)
            turn_unit<W>(v[k], c[k], s[k], interleaved);
}
// x becomes (offset + w) x / root(mean x^2 + eps)
template <int W, int PER>
__device__ __forceinline__ void norm_units(const NormParams &N, unsigned lanes, int head_dim, float (&v)[PER][2 * W], const float (&f)[PER][2 * W])
{
    float (&flat)[PER * 2 * W] = reinterpret_cast<float (&)[PER * 2 * W]>(v);
    const float r = inverse_root(flat, lanes, head_dim, N.eps);
#pragma unroll
    for (int k = 0; k < PER; ++k)
#pragma unroll
        for (int e = 0; e < 2 * W; ++e)
            v[k][e] = v[k][e] * r * f[k][e];
}

template <typename T, int W, int PER>
__global__ __launch_bounds__(THREADS) void norm_rope_kernel(HeadParams P)
{
    const HeadLane<W, PER> L(P.lanes, P.head_dim, P.rot.rot_dim, P.rot.interleaved);
    const unsigned per_block = THREADS / L.lanes, rows = P.heads + P.kv_heads;
    float fq[PER][2 * W], fk[PER][2 * W];
    if (P.norm.on) {
        load_factors<W, PER>(P.norm, P.norm.wq, L.at, L.mine, fq);
        load_factors<W, PER>(P.norm, P.norm.wk, L.at, L.mine, fk);
    }
    for (unsigned item = blockIdx.x * per_block + threadIdx.x / L.lanes; item < P.tokens * P.groups; item += gridDim.x * per_block) {
        const unsigned token = item / P.groups, group = item - token * P.groups;
        float c[PER][W], s[PER][W];
        find_angles<W, PER>(P.rot, L, P.positions, token, 1.0f, c, s);
        for (unsigned row = group; row < rows; row += P.groups) {
            const bool is_k = row >= P.heads;
            const unsigned h = is_k ? row - P.heads : row;
            const T *x = is_k ? static_cast<const T *>(P.k) + (int64_t)token * P.k_token + h * P.k_head : static_cast<const T *>(P.q) + (int64_t)token * P.q_token + h * P.q_head;
            T *out = is_k ? static_cast<T *>(P.k_out) + (int64_t)token * P.ok_token + h * P.ok_head : static_cast<T *>(P.q_out) + (int64_t)token * P.oq_token + h * P.oq_head;
            float v[PER][2 * W];
            load_units<T, W, PER>(x, L, v);
            if (P.norm.on) {
                if (is_k)
                    norm_units<W, PER>(P.norm, L.lanes, P.head_dim, v, fk);
                else
                    norm_units<W, PER>(P.norm, L.lanes, P.head_dim, v, fq);
            }
            turn_units<W, PER>(L, v, c, s, P.rot.interleaved);
            store_units<T, W, PER>(out, L, v);
        }
    }
}

// dQ, dK; and of every workgroup the sums for dwq and dwk, [2][head_dim] floats.
template <typename T, int W, int PER>
__global__ __launch_bounds__(THREADS) void norm_rope_grad_kernel(HeadParams P, const void *dq_out, const void *dk_out, void *dq, void *dk, float *sums)
{
    const HeadLane<W, PER> L(P.lanes, P.head_dim, P.rot.rot_dim, P.rot.interleaved);
    const unsigned per_block = THREADS / L.lanes, rows = P.heads + P.kv_heads, slot = threadIdx.x / L.lanes;
    const float inv_dim = 1.0f / P.head_dim;
    float fq[PER][2 * W], fk[PER][2 * W], aq[PER][2 * W] = {}, ak[PER][2 * W] = {};
    if (P.norm.on) {
        load_factors<W, PER>(P.norm, P.norm.wq, L.at, L.mine, fq);
        load_factors<W, PER>(P.norm, P.norm.wk, L.at, L.mine, fk);
    }
    for (unsigned item = blockIdx.x * per_block + slot; item < P.tokens * P.groups; item += gridDim.x * per_block) {
        const unsigned token = item / P.groups, group = item - token * P.groups;
        float c[PER][W], s[PER][W];
        find_angles<W, PER>(P.rot, L, P.positions, token, -1.0f, c, s);
        for (unsigned row = group; row < rows; row += P.groups) {
            const bool is_k = row >= P.heads;
            const unsigned h = is_k ? row - P.heads : row;
            const int64_t in = is_k ? (int64_t)token * P.k_token + h * P.k_head : (int64_t)token * P.q_token + h * P.q_head;
            const int64_t from = is_k ? (int64_t)token * P.ok_token + h * P.ok_head : (int64_t)token * P.oq_token + h * P.oq_head;
            float g[PER][2 * W], n[PER][2 * W];
            load_units<T, W, PER>(static_cast<const T *>(is_k ? dk_out : dq_out) + from, L, g);
            if (P.norm.on)
                load_units<T, W, PER>(static_cast<const T *>(is_k ? P.k : P.q) + in, L, n);
            turn_units<W, PER>(L, g, c, s, P.rot.interleaved);
            if (P.norm.on) {
                auto norm_grad = [&](const float (&f)[PER][2 * W], float (&a)[PER][2 * W]) __attribute__((always_inline)) {
                    const float r = inverse_root(reinterpret_cast<float (&)[PER * 2 * W]>(n), L.lanes, P.head_dim, P.norm.eps);
                    float hn = 0.0f;
#pragma unroll
                    for (int k = 0; k < PER; ++k)
#pragma unroll
                        for (int e = 0; e < 2 * W; ++e) {
                            n[k][e] *= r;
                            a[k][e] = __builtin_fmaf(g[k][e], n[k][e], a[k][e]);
                            g[k][e] *= f[k][e];
                            hn = __builtin_fmaf(g[k][e], n[k][e], hn);
                        }
                    hn = sum_of_lanes(hn, L.lanes) * inv_dim;
#pragma unroll
                    for (int k = 0; k < PER; ++k)
#pragma unroll
                        for (int e = 0; e < 2 * W; ++e)
                            g[k][e] = r * __builtin_fmaf(-n[k][e], hn, g[k][e]);
                };
                if (is_k)
                    norm_grad(fk, ak);
                else
                    norm_grad(fq, aq);
            }
            store_units<T, W, PER>(static_cast<T *>(is_k ? dk : dq) + in, L, g);
        }
    }
    if (sums == nullptr)
        return;
    // [slots of the workgroup][2][head_dim] in LDS, then a column a thread
    __shared__ float parts[THREADS * 4 * W * PER];                         // (a slot's lanes hold 2 W PER features each)
    const unsigned columns = 2 * P.head_dim;
#pragma unroll
    for (int k = 0; k < PER; ++k)
        if (L.mine[k])
#pragma unroll
            for (int e = 0; e < 2 * W; ++e) {
                const int i = e < W ? L.at[k].a + e : L.at[k].b + e - W;
                parts[slot * columns + i] = aq[k][e];
                parts[slot * columns + P.head_dim + i] = ak[k][e];
            }
    __syncthreads();
    for (unsigned i = threadIdx.x; i < columns; i += THREADS) {
        float total = 0.0f;
        for (unsigned j = 0; j < per_block; ++j)
            total += parts[j * columns + i];
        sums[(size_t)blockIdx.x * columns + i] = total;
    }
}

// dwq and dwk: sixteen columns a workgroup, each added up by sixteen threads and those by the first.
constexpr unsigned SUM_COLUMNS = 16;
__global__ __launch_bounds__(THREADS) void norm_weights_kernel(const float *sums, unsigned count, unsigned head_dim, float *dwq, float *dwk)
{
    __shared__ float parts[THREADS];
    const unsigned columns = 2 * head_dim, i = blockIdx.x * SUM_COLUMNS + threadIdx.x % SUM_COLUMNS, first = threadIdx.x / SUM_COLUMNS;
    float total = 0.0f;
    if (i < columns)
        for (unsigned j = first; j < count; j += THREADS / SUM_COLUMNS)
            total += sums[(size_t)j * columns + i];
    parts[threadIdx.x] = total;
    __syncthreads();
    if (first == 0 && i < columns) {
        for (unsigned j = 1; j < THREADS / SUM_COLUMNS; ++j)
            total += parts[j * SUM_COLUMNS + threadIdx.x];
        float *to = i < head_dim ? dwq : dwk;
        if (to != nullptr)
            to[i < head_dim ? i : i - head_dim] = total;
    }
}

// The cache's writer with normed heads: `lanes` neighbouring lanes share a row, its squares and, in e4m3, its largest magnitude.
template <bool E4M3>
__global__ __launch_bounds__(THREADS) void cache_write_norm_kernel(CachePool C, CacheRows R, AxesRotation A, NormParams N)
{
    constexpr int W = 8;
    unsigned lanes = 1;
    while (lanes * 16 < (unsigned)C.head_dim)
        lanes *= 2;
    const HeadLane<W, 1> L(lanes, C.head_dim, A.rot_dim, A.interleaved);
    const unsigned per_block = THREADS / lanes, total = R.tokens * R.groups;
    const unsigned heads = R.q != nullptr ? R.heads : 0, rows = heads + 2 * C.kv_heads;
    float fq[1][2 * W], fk[1][2 * W];
    if (N.on) {
        load_factors<W, 1>(N, heads > 0 ? N.wq : nullptr, L.at, L.mine, fq);
        load_factors<W, 1>(N, N.wk, L.at, L.mine, fk);
    }
    for (unsigned item = blockIdx.x * per_block + threadIdx.x / lanes; item < total; item += gridDim.x * per_block) {
        const unsigned token = item / R.groups, group = item - token * R.groups;
        float c[1][W], s[1][W];
        if (group < heads + C.kv_heads)
            find_angles<W, 1>(A, L, R.positions, token, 1.0f, c, s);
        const int64_t slot = R.slots[token];
        const bool stored = slot >= 0 && (slot >> C.page_shift) < C.n_pages;
        const int64_t page = stored ? slot >> C.page_shift : 0;
        const int in_page = (int)(slot & ((1 << C.page_shift) - 1));
        for (unsigned row = group; row < rows; row += R.groups) {    // (the lanes of a row together)
            const bool is_q = row < heads, is_v = row >= heads + C.kv_heads;
            const unsigned h = is_q ? row : is_v ? row - heads - C.kv_heads : row - heads;
            float v[1][2 * W];
            load_units<__bf16, W, 1>(is_q ? static_cast<const __bf16 *>(R.q) + (int64_t)token * R.q_token + h * R.q_head
                                     : is_v ? static_cast<const __bf16 *>(R.v) + (int64_t)token * R.v_token + h * R.v_head
                                            : static_cast<const __bf16 *>(R.k) + (int64_t)token * R.k_token + h * R.k_head, L, v);
            if (!is_v) {
                if (N.on) {
                    if (is_q)
                        norm_units<W, 1>(N, lanes, C.head_dim, v, fq);
                    else
                        norm_units<W, 1>(N, lanes, C.head_dim, v, fk);
                }
                turn_units<W, 1>(L, v, c, s, A.interleaved);
            }
            const int64_t place = page * C.page_stride + h * C.head_stride + in_page * C.token_stride;
            if (is_q) {
                store_units<__bf16, W, 1>(static_cast<__bf16 *>(R.q_out) + (int64_t)token * R.o_token + h * R.o_head, L, v);
                continue;
            }
            if constexpr (!E4M3) {
                if (stored)
                    store_units<__bf16, W, 1>(static_cast<__bf16 *>(is_v ? C.v : C.k) + place, L, v);
            } else {
                float top = 0.0f;
#pragma unroll
                for (int i = 0; i < 2 * W; ++i)
                    top = fmaxf(top, __builtin_isfinite(v[0][i]) ? fabsf(v[0][i]) : 0.0f);
                for (unsigned d = 1; d < lanes; d *= 2)
                    top = fmaxf(top, __shfl_xor(top, (int)d));
                const int e = exponent_of(top);
                if (stored && L.mine[0]) {
                    unsigned char *dst = static_cast<unsigned char *>(is_v ? C.v : C.k) + place;
                    store_codes(dst, L.at[0], codes(v[0], e));
                    if (L.u == 0)
                        (is_v ? C.v_exp : C.k_exp)[((page * C.kv_heads + h) << C.page_shift) + in_page] = (uint8_t)(e + 127);
                }
            }
        }
    }
}

unsigned lanes_of(int units)                                         // of a head: a power of two, at most a wave
{
    unsigned lanes = 1;
    while ((int)lanes < units && lanes < 64)
        lanes *= 2;
    return lanes;
}

// Whole 16-byte accesses where a unit's two parts start on them.
bool wide_units(const HeadParams &p, bool bf16)
{
    const int w = bf16 ? 8 : 4;
    return p.head_dim % (2 * w) == 0 && p.rot.rot_dim % (2 * w) == 0;
}

// Workgroups of the gradient at the most, each of which leaves sums.
constexpr unsigned GRAD_BLOCKS = 1024;

}  // namespace

hipError_t launch_norm_rope(const HeadParams &p_in, bool bf16, hipStream_t s, int num_cu)
{
    HeadParams p = p_in;
    const bool wide = wide_units(p, bf16);
    p.lanes = lanes_of(p.head_dim / (!wide ? 2 : bf16 ? 16 : 8));
    p.groups = groups_of(p.tokens, p.lanes, p.heads + p.kv_heads, num_cu);
    const dim3 grid(blocks_of((uint64_t)p.tokens * p.groups, THREADS / p.lanes));
    if (bf16 && wide)
        hipLaunchKernelGGL((norm_rope_kernel<__bf16, 8, 1>), grid, dim3(THREADS), 0, s, p);
    else if (bf16)
        hipLaunchKernelGGL((norm_rope_kernel<__bf16, 1, 2>), grid, dim3(THREADS), 0, s, p);
    else if (wide)
        hipLaunchKernelGGL((norm_rope_kernel<float, 4, 1>), grid, dim3(THREADS), 0, s, p);
    else
        hipLaunchKernelGGL((norm_rope_kernel<float, 1, 2>), grid, dim3(THREADS), 0, s, p);
    return hipGetLastError();
}

size_t norm_rope_scratch_bytes(int head_dim) { return (size_t)GRAD_BLOCKS * 2 * head_dim * sizeof(float); }

hipError_t launch_norm_rope_grad(const HeadParams &p_in, const void *dq_out, const void *dk_out, void *dq, void *dk, float *dwq, float *dwk, float *scratch,
                                 bool bf16, hipStream_t s, int num_cu)
{
    HeadParams p = p_in;
    const bool wide = wide_units(p, bf16);
    p.lanes = lanes_of(p.head_dim / (!wide ? 2 : bf16 ? 16 : 8));
    const bool nothing = p.tokens == 0 || p.heads + p.kv_heads == 0; // (the sums over nothing are zeros)
    p.groups = nothing ? 1 : groups_of(p.tokens, p.lanes, p.heads + p.kv_heads, num_cu);
    unsigned blocks = nothing ? 0 : blocks_of((uint64_t)p.tokens * p.groups, THREADS / p.lanes);
    float *sums = dwq != nullptr || dwk != nullptr ? scratch : nullptr;
    if (sums != nullptr && blocks > GRAD_BLOCKS)
        blocks = GRAD_BLOCKS;
    const dim3 grid(blocks);
    if (nothing)
        ;
    else if (bf16 && wide)
        hipLaunchKernelGGL((norm_rope_grad_kernel<__bf16, 8, 1>), grid, dim3(THREADS), 0, s, p, dq_out, dk_out, dq, dk, sums);
    else if (bf16)
        hipLaunchKernelGGL((norm_rope_grad_kernel<__bf16, 1, 2>), grid, dim3(THREADS), 0, s, p, dq_out, dk_out, dq, dk, sums);
    else if (wide)
        hipLaunchKernelGGL((norm_rope_grad_kernel<float, 4, 1>), grid, dim3(THREADS), 0, s, p, dq_out, dk_out, dq, dk, sums);
    else
        hipLaunchKernelGGL((norm_rope_grad_kernel<float, 1, 2>), grid, dim3(THREADS), 0, s, p, dq_out, dk_out, dq, dk, sums);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || sums == nullptr)
        return e;
    hipLaunchKernelGGL(norm_weights_kernel, dim3((2 * p.head_dim + SUM_COLUMNS - 1) / SUM_COLUMNS), dim3(THREADS), 0, s, sums, blocks, (unsigned)p.head_dim, dwq, dwk);
    return hipGetLastError();
}

hipError_t launch_cache_write_norm(const CachePool &c, const CacheRows &r_in, const AxesRotation &a, const NormParams &n, hipStream_t s, int num_cu)
{
    CacheRows r = r_in;
    const unsigned lanes = lanes_of(c.head_dim / 16);
    r.groups = groups_of(r.tokens, lanes, (r.q != nullptr ? r.heads : 0) + 2 * c.kv_heads, num_cu);
    const dim3 grid(blocks_of((uint64_t)r.tokens * r.groups, THREADS / lanes));
    if (c.e4m3)
        hipLaunchKernelGGL((cache_write_norm_kernel<true>), grid, dim3(THREADS), 0, s, c, r, a, n);
    else
        hipLaunchKernelGGL((cache_write_norm_kernel<false>), grid, dim3(THREADS), 0, s, c, r, a, n);
    return hipGetLastError();
}

}  // namespace cf
