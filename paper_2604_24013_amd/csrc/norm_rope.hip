// Every head of Q and K divided by its root mean square, times a weight, and rotated by positions on several axes; the gradient of that; the
// same on the way into the paged cache.
//   r = (mean x^2 + eps)^-1/2,  n = r x,  y = R (n (offset + w))
//   g = R^T dy,  dw = sum over tokens and heads of g n,  h = g (offset + w),  dx = r (h - n mean(h n))
//
// Bound by HBM: forward every feature is read and written once, backward x and dy are read and dx is written.  A thread owns a unit of one
// head (W rotated pairs, or 2 W features that are copied), the lanes of a head are neighbours, a power of two of them, and add up its
// squares by moves inside the wave.  Nothing is kept for the gradient: r costs less to compute again than to read, since x is read in any
// case.
// A workgroup takes some tokens, and its waves share out jobs of one head of as many tokens as fill a wave, each with two jobs on their way from memory:
// nine heads of sixteen tokens are nine jobs a wave.  Cosines and sines of its tokens are computed once by all threads together and come from
// LDS: for every wave anew they took more than half of the vector instructions (64-bit products and two series a pair).  So do the weights.
// The gradients of the weights are sums over all tokens: every workgroup leaves one row of them in the caller's scratch memory, and a second
// launch adds those up in order.  No atomics: the same call gives the same bits.
// Measured (us, traced): 8192 tokens of 8 + 1 bf16 heads of 128 features, all rotated: 12.3, 3.1 TB/s (rotation alone 9.4; a strided copy of the heads by torch
// 11.3, this 14.2 with nothing in the last-level cache); the gradient 19.0, 3.0 TB/s, and 4.0 for the sums (the sum of two such tensors
// into a third by torch 10.9: a workgroup's waves have four or five jobs each, with little between start and end that hides either).  4099 tokens of 5 + 2 fp32 heads, half of each
// rotated: 9.5, 14.6, 4.0.  Into the cache in e4m3, 8 + 1 + 1 heads: 14.2.  Waves wait for memory for 60 % of their cycles, with four a SIMD.
#include "rope_units.h"

namespace cf {
namespace {

constexpr unsigned WAVES = THREADS / 64;
constexpr int MAX_DIM = 256;             // features of a head

// Cosines and sines of the tokens of a workgroup, [tokens][pairs] of each, found by all its threads.  (64 lanes hold the heads of a job, so that there are 64 W PER
// pairs of its tokens at the most.)  Two buffers: the next tokens' are written while the last ones' may still be read.
constexpr int MAX_SUBS = 4;              // jobs of a head
template <int W, int PER>
struct AngleTable {
    static constexpr int SIZE = MAX_SUBS * 64 * W * PER;
    float c[2][SIZE] __attribute__((aligned(16))), s[2][SIZE] __attribute__((aligned(16)));
    __device__ __forceinline__ void fill(int buf, const AxesRotation &R, const int32_t *positions, unsigned first, unsigned per_block, unsigned tokens, float sign)
    {
        const unsigned pairs = (unsigned)R.rot_dim / 2;
        for (unsigned i = threadIdx.x; i < per_block * pairs; i += THREADS) {
            const unsigned t = i / pairs, j = i - t * pairs, axis = R.axis_bits[j >> 4] >> 2 * (j & 15) & 3;
            const unsigned token = first + t < tokens ? first + t : tokens - 1;
            cos_sin(phase_of(R.turn[j], positions[axis * R.position_axis + token]), R.magnitude, sign * R.magnitude, &c[buf][i], &s[buf][i]);
        }
    }
};

template <int CONTROL>
__device__ __forceinline__ float moved(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CONTROL, 0xf, 0xf, true)); }

// Sum over the `lanes` neighbouring lanes (a power of two) of a head; every one of them gets it.
__device__ __forceinline__ float sum_of_lanes(float x, unsigned lanes)
{
    if (lanes > 1)
        x += moved<0xB1>(x);                                         // from the other lane of a pair
    if (lanes > 2)
        x += moved<0x4E>(x);                                         // ... pair of four
    if (lanes > 4)
        x += moved<0x141>(x);                                        // ... four of eight (mirrored)
    if (lanes > 8)
        x += moved<0x140>(x);                                        // ... eight of sixteen (mirrored)
    if (lanes > 16)
        x += __shfl_xor(x, 16);
    if (lanes > 32)
        x += __shfl_xor(x, 32);
    return x;
}

// What a thread has of a head: the lane, and its units (PER, `lanes` apart; those behind the head's last are not there).
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
    __device__ __forceinline__ int feature(int k, int e) const { return e < W ? at[k].a + e : at[k].b + e - W; }
};

// One over the root mean square of a head, of which a lane's units hold PER times N features.  Squares of more than 2^128 together: scaled down first.
template <int W, int PER>
__device__ __forceinline__ float inverse_root(const HeadLane<W, PER> &L, const float (&x)[PER][2 * W], float inv_dim, float eps)
{
    float all = 0.0f, most = 0.0f;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < 2 * W; ++e)
            ss = __builtin_fmaf(x[k][e], x[k][e], ss);
        all += L.mine[k] ? ss : 0.0f;
    }
    const float ss = sum_of_lanes(all, L.lanes);
    float r = __builtin_amdgcn_rsqf(__builtin_fmaf(ss, inv_dim, eps));
    if (__builtin_amdgcn_ballot_w64(ss == INFINITY) != 0) {
#pragma unroll
        for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int e = 0; e < 2 * W; ++e) {
                const float y = x[k][e] * 0x1p-70f;
                most = L.mine[k] ? __builtin_fmaf(y, y, most) : most;
            }
        r = ss == INFINITY ? 0x1p-70f * __builtin_amdgcn_rsqf(sum_of_lanes(most, L.lanes) * inv_dim) : r;
    }
    return r;
}

// A thread's part of a head as it comes from memory.
template <typename T, int W, int PER>
struct Raw {
    typedef T V __attribute__((ext_vector_type(W)));
    V a[PER], b[PER];
    __device__ __forceinline__ void load(const T *row, const HeadLane<W, PER> &L)
    {
#pragma unroll
        for (int k = 0; k < PER; ++k) {                              // (a unit that is not there: the head's first)
            a[k] = *reinterpret_cast<const V *>(row + L.at[k].a);
            b[k] = *reinterpret_cast<const V *>(row + L.at[k].b);
        }
    }
    __device__ __forceinline__ void get(float (&v)[PER][2 * W]) const
    {
#pragma unroll
        for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int e = 0; e < W; ++e) {
                v[k][e] = (float)a[k][e];
                v[k][W + e] = (float)b[k][e];
            }
    }
};

template <typename T, int W, int PER>
__device__ __forceinline__ void store_units(T *row, const HeadLane<W, PER> &L, const float (&v)[PER][2 * W])
{
#pragma unroll
    for (int k = 0; k < PER; ++k)
        if (L.mine[k])
            store_unit<T, W>(row, L.at[k], v[k]);
}

// The weights of Q and of K as factors (offset + w), or 1 without weights: in LDS, from where a head takes sixteen at a time (in registers, of both, they
// would cost a wave's neighbours their place).
template <int W, int PER>
struct FactorTable {
    float f[2][MAX_DIM] __attribute__((aligned(16)));
    __device__ __forceinline__ void fill(const NormParams &N, int head_dim)
    {
        for (int i = threadIdx.x; i < 2 * head_dim; i += THREADS) {
            const int k = i >= head_dim, at = k ? i - head_dim : i;
            const void *w = k ? N.wk : N.wq;
            f[k][at] = w == nullptr ? 1.0f : N.offset + (N.weight_bf16 ? (float)static_cast<const __bf16 *>(w)[at] : static_cast<const float *>(w)[at]);
        }
    }
    __device__ __forceinline__ void read(int of, const HeadLane<W, PER> &L, float (&x)[PER][2 * W]) const
    {
#pragma unroll
        for (int k = 0; k < PER; ++k)
            load_unit<float, W>(f[of], L.at[k], x[k]);
    }
};

// A thread's cosines and sines of token `t` of the workgroup's.
template <int W, int PER>
__device__ __forceinline__ void read_angles(const AngleTable<W, PER> &T, int buf, const HeadLane<W, PER> &L, unsigned t, unsigned pairs, float (&c)[PER][W], float (&s)[PER][W])
{
#pragma unroll
    for (int k = 0; k < PER; ++k)
        if (L.mine[k] && L.at[k].rotated) {
            load<float, W>(&T.c[buf][t * pairs + L.at[k].pair], c[k]);
            load<float, W>(&T.s[buf][t * pairs + L.at[k].pair], s[k]);
        }
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
__device__ __forceinline__ void norm_units(const HeadLane<W, PER> &L, float inv_dim, float eps, float (&v)[PER][2 * W], const FactorTable<W, PER> &factors, int of)
{
    float f[PER][2 * W];
    factors.read(of, L, f);
    const float r = inverse_root(L, v, inv_dim, eps);
#pragma unroll
    for (int k = 0; k < PER; ++k)
#pragma unroll
        for (int e = 0; e < 2 * W; ++e)
            v[k][e] = v[k][e] * r * f[k][e];
}

// use(i, what load(i) asked for) for i = first, first + step, .. below count with two of them on their way; `before` behind the first two loads.
template <typename F1, typename F2, typename F3>
__device__ __forceinline__ void over_jobs(unsigned first, unsigned count, unsigned step, F1 &&load, F2 &&before, F3 &&use)
{
    const unsigned last = count - 1;
    auto next = load(first < count ? first : last), then = load(first + step < count ? first + step : last);
    before();
#pragma unroll 1
    for (unsigned i = first; i < count; i += step) {
        const auto now = next;
        next = then;
        if (i + 2 * step < count)
            then = load(i + 2 * step);
        use(i, now);
    }
}

// Which jobs a wave takes: first, first + step, .. of the (head, part of the workgroup's tokens) pairs; heads are Q's, then K's (and V's).
struct Jobs {
    unsigned first, step, per_job, in_job, sub_shift;
    unsigned block, rounds, per_block;
    __device__ __forceinline__ Jobs(unsigned groups, unsigned lanes, unsigned subs_shift)
    {
        const unsigned wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        first = blockIdx.x % groups * WAVES + wave;
        step = groups * WAVES;
        block = blockIdx.x / groups;
        rounds = gridDim.x / groups;
        per_job = 64 / lanes;
        in_job = (threadIdx.x & 63) / lanes;
        sub_shift = subs_shift;
        per_block = per_job << subs_shift;
    }
    __device__ __forceinline__ unsigned head(unsigned job) const { return job >> sub_shift; }
    __device__ __forceinline__ unsigned from(unsigned job) const { return (job & ((1u << sub_shift) - 1)) * per_job; }     // the first token, in the workgroup's
};

// (INTER, the layout of pairs, is known when the kernels are built: with a branch on it the units came to lie in scratch memory.)
template <typename T, int W, int PER, bool INTER>
__global__ __launch_bounds__(THREADS) void norm_rope_kernel(HeadParams P)
{
    __shared__ AngleTable<W, PER> table;
    __shared__ FactorTable<W, PER> factors;
    const HeadLane<W, PER> L(P.lanes, P.head_dim, P.rot.rot_dim, INTER);
    const Jobs J(P.groups, P.lanes, P.subs_shift);
    const unsigned heads = P.heads + P.kv_heads, pairs = P.rot.rot_dim / 2;
    const float inv_dim = 1.0f / P.head_dim;
    // (addresses: of a job in scalar registers, and the lane's token behind the first)
    const int64_t q_in = J.in_job * P.q_token, k_in = J.in_job * P.k_token, q_to = J.in_job * P.oq_token, k_to = J.in_job * P.ok_token;
    int buf = 0;
    bool filled = false;                                             // (the weights, once)
    for (unsigned t0 = J.block * J.per_block; t0 < P.tokens; t0 += J.rounds * J.per_block, buf ^= 1) {
        over_jobs(
            J.first, heads << J.sub_shift, J.step,
            [&](unsigned job) __attribute__((always_inline)) {
                Raw<T, W, PER> raw;
                const unsigned i = J.head(job), t = t0 + J.from(job);
                if (t + J.in_job < P.tokens) {
                    if (i < P.heads)
                        raw.load(static_cast<const T *>(P.q) + (t * P.q_token + i * P.q_head) + q_in, L);
                    else
                        raw.load(static_cast<const T *>(P.k) + (t * P.k_token + (i - P.heads) * P.k_head) + k_in, L);
                }
                return raw;
            },
            [&]() __attribute__((always_inline)) {
                if (P.norm.on && !filled)
                    factors.fill(P.norm, P.head_dim);
                if (pairs > 0)
                    table.fill(buf, P.rot, P.positions, t0, J.per_block, P.tokens, 1.0f);
                if (pairs > 0 || !filled)
                    __syncthreads();
                filled = true;
            },
            [&](unsigned job, const Raw<T, W, PER> &raw) __attribute__((always_inline)) {
                const unsigned i = J.head(job), t = t0 + J.from(job);
                if (t + J.in_job >= P.tokens)
                    return;
                const bool is_k = i >= P.heads;                      // (uniform)
                float v[PER][2 * W], c[PER][W], s[PER][W];
                raw.get(v);
                if (P.norm.on)
                    norm_units<W, PER>(L, inv_dim, P.norm.eps, v, factors, is_k);
                read_angles<W, PER>(table, buf, L, J.from(job) + J.in_job, pairs, c, s);
                turn_units<W, PER>(L, v, c, s, INTER);
                if (is_k)
                    store_units<T, W, PER>(static_cast<T *>(P.k_out) + (t * P.ok_token + (i - P.heads) * P.ok_head) + k_to, L, v);
                else
                    store_units<T, W, PER>(static_cast<T *>(P.q_out) + (t * P.oq_token + i * P.oq_head) + q_to, L, v);
            });
    }
}

// dQ, dK; and of every workgroup a row of sums for the weights of both, [2][head_dim] floats.
template <typename T, int W, int PER, bool INTER>
__global__ __launch_bounds__(THREADS, 4) void norm_rope_grad_kernel(HeadParams P, const void *dq_out, const void *dk_out, void *dq, void *dk, float *sums)
{
    __shared__ AngleTable<W, PER> table;
    __shared__ FactorTable<W, PER> factors;
    const HeadLane<W, PER> L(P.lanes, P.head_dim, P.rot.rot_dim, INTER);
    const Jobs J(P.groups, P.lanes, P.subs_shift);
    const unsigned heads = P.heads + P.kv_heads, pairs = P.rot.rot_dim / 2;
    const float inv_dim = 1.0f / P.head_dim;
    const int64_t q_in = J.in_job * P.q_token, k_in = J.in_job * P.k_token, q_from = J.in_job * P.oq_token, k_from = J.in_job * P.ok_token;
    // The sums of the tensor that the wave is at; what its tokens have of a tensor goes to LDS when it turns to the other one (in registers, both took
    // the place of every second wave).
    __shared__ float parts[2][WAVES][MAX_DIM];
    const unsigned wave = threadIdx.x >> 6;
    float sum[PER][2 * W] = {};
    bool of_k = false;
    for (int i = threadIdx.x & 63; i < P.head_dim; i += 64)
        parts[0][wave][i] = parts[1][wave][i] = 0.0f;
    auto put_away = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int e = 0; e < 2 * W; ++e) {
                float y = sum[k][e];
                for (unsigned d = P.lanes; d < 64; d *= 2)
                    y += __shfl_xor(y, (int)d);
                if (L.mine[k] && J.in_job == 0)
                    parts[of_k][wave][L.feature(k, e)] += y;
                sum[k][e] = 0.0f;
            }
    };
    struct Both {
        Raw<T, W, PER> g, x;
    };
    int buf = 0;
    bool filled = false;
    for (unsigned t0 = J.block * J.per_block; t0 < P.tokens; t0 += J.rounds * J.per_block, buf ^= 1) {
        auto at_q = [&](unsigned t, unsigned i) __attribute__((always_inline)) { return (t * P.q_token + i * P.q_head) + q_in; };
        auto at_k = [&](unsigned t, unsigned i) __attribute__((always_inline)) { return (t * P.k_token + (i - P.heads) * P.k_head) + k_in; };
        over_jobs(
            J.first, heads << J.sub_shift, J.step,
            [&](unsigned job) __attribute__((always_inline)) {
                Both raw;
                const unsigned i = J.head(job), t = t0 + J.from(job);
                if (t + J.in_job < P.tokens) {
                    if (i < P.heads) {
                        raw.g.load(static_cast<const T *>(dq_out) + (t * P.oq_token + i * P.oq_head) + q_from, L);
                        if (P.norm.on)
                            raw.x.load(static_cast<const T *>(P.q) + at_q(t, i), L);
                    } else {
                        raw.g.load(static_cast<const T *>(dk_out) + (t * P.ok_token + (i - P.heads) * P.ok_head) + k_from, L);
                        if (P.norm.on)
                            raw.x.load(static_cast<const T *>(P.k) + at_k(t, i), L);
                    }
                }
                return raw;
            },
            [&]() __attribute__((always_inline)) {
                if (P.norm.on && !filled)
                    factors.fill(P.norm, P.head_dim);
                if (pairs > 0)
                    table.fill(buf, P.rot, P.positions, t0, J.per_block, P.tokens, -1.0f);
                if (pairs > 0 || !filled)
                    __syncthreads();
                filled = true;
            },
            [&](unsigned job, const Both &raw) __attribute__((always_inline)) {
                const unsigned i = J.head(job), t = t0 + J.from(job);
                const bool is_k = i >= P.heads;                      // (uniform)
                if (is_k != of_k) {
                    if (P.norm.on)
                        put_away();
                    of_k = is_k;
                }
                if (t + J.in_job >= P.tokens)
                    return;
                float g[PER][2 * W], n[PER][2 * W], c[PER][W], s[PER][W];
                raw.g.get(g);
                read_angles<W, PER>(table, buf, L, J.from(job) + J.in_job, pairs, c, s);
                turn_units<W, PER>(L, g, c, s, INTER);
                if (P.norm.on) {
                    raw.x.get(n);
                    const float r = inverse_root(L, n, inv_dim, P.norm.eps);
                    float hn = 0.0f;
                    float f[PER][2 * W];
                    factors.read(is_k, L, f);
#pragma unroll
                    for (int k = 0; k < PER; ++k) {
                        float part = 0.0f;
#pragma unroll
                        for (int e = 0; e < 2 * W; ++e) {
                            n[k][e] *= r;
                            sum[k][e] = __builtin_fmaf(g[k][e], n[k][e], sum[k][e]);
                            g[k][e] *= f[k][e];
                            part = __builtin_fmaf(g[k][e], n[k][e], part);
                        }
                        hn += L.mine[k] ? part : 0.0f;
                    }
                    hn = sum_of_lanes(hn, P.lanes) * inv_dim;
#pragma unroll
                    for (int k = 0; k < PER; ++k)
#pragma unroll
                        for (int e = 0; e < 2 * W; ++e)
                            g[k][e] = r * __builtin_fmaf(-n[k][e], hn, g[k][e]);
                }
                if (is_k)
                    store_units<T, W, PER>(static_cast<T *>(dk) + at_k(t, i), L, g);
                else
                    store_units<T, W, PER>(static_cast<T *>(dq) + at_q(t, i), L, g);
            });
    }
    if (sums == nullptr)
        return;
    put_away();
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * P.head_dim; i += THREADS) {
        const int k = i >= P.head_dim, at = k ? i - P.head_dim : i;
        float total = 0.0f;
#pragma unroll
        for (unsigned w = 0; w < WAVES; ++w)
            total += parts[k][w][at];
        sums[(size_t)blockIdx.x * 2 * P.head_dim + i] = total;
    }
}

// dwq and dwk from `count` rows of sums: sixteen columns a workgroup, sixty-four threads for each of them, which have eight loads on their way (one by
// one by sixteen threads: 20 us).
constexpr unsigned SUM_THREADS = 1024, SUM_COLUMNS = 16, SUM_ROWS = SUM_THREADS / SUM_COLUMNS;
__global__ __launch_bounds__(SUM_THREADS) void norm_weights_kernel(const float *sums, unsigned count, unsigned head_dim, float *dwq, float *dwk)
{
    __shared__ float parts[SUM_ROWS][SUM_COLUMNS + 1];
    const unsigned column = threadIdx.x % SUM_COLUMNS, i = blockIdx.x * SUM_COLUMNS + column, row = threadIdx.x / SUM_COLUMNS, columns = 2 * head_dim;
    float total = 0.0f;
    if (i < columns)
        for (unsigned j0 = row; j0 < count; j0 += 8 * SUM_ROWS) {
            float x[8];
#pragma unroll
            for (unsigned u = 0; u < 8; ++u) {
                const unsigned j = j0 + u * SUM_ROWS;
                x[u] = sums[(size_t)(j < count ? j : j0) * columns + i];
            }
#pragma unroll
            for (unsigned u = 0; u < 8; ++u)
                total += j0 + u * SUM_ROWS < count ? x[u] : 0.0f;
        }
    parts[row][column] = total;
    __syncthreads();
    if (threadIdx.x < SUM_COLUMNS * 16) {                            // sixteen threads a column
        const unsigned mine = threadIdx.x / 16, part = threadIdx.x % 16, to = blockIdx.x * SUM_COLUMNS + mine;
        float all = 0.0f;
#pragma unroll
        for (unsigned j = 0; j < SUM_ROWS / 16; ++j)
            all += parts[part * (SUM_ROWS / 16) + j][mine];
        all = sum_of_lanes(all, 16);
        float *dw = to < head_dim ? dwq : dwk;
        if (part == 0 && to < columns && dw != nullptr)
            dw[to < head_dim ? to : to - head_dim] = all;
    }
}

// The cache's writer with normed heads: of every token the heads of Q, K and V; the lanes of a row share its squares and, in e4m3, its largest
// magnitude.
template <bool E4M3, bool INTER>
__global__ __launch_bounds__(THREADS) void cache_write_norm_kernel(CachePool C, CacheRows R, AxesRotation A, NormParams N, unsigned lanes, unsigned subs_shift)
{
    constexpr int W = 8;
    __shared__ AngleTable<W, 1> table;
    __shared__ FactorTable<W, 1> factors;
    __shared__ int64_t slots[2][MAX_SUBS * 64];
    const HeadLane<W, 1> L(lanes, C.head_dim, A.rot_dim, INTER);
    const Jobs J(R.groups, lanes, subs_shift);
    const unsigned q_heads = R.q != nullptr ? R.heads : 0, v_from = q_heads + C.kv_heads, heads = v_from + C.kv_heads, pairs = A.rot_dim / 2;
    const float inv_dim = 1.0f / C.head_dim;
    const int64_t q_in = J.in_job * R.q_token, k_in = J.in_job * R.k_token, v_in = J.in_job * R.v_token, q_to = J.in_job * R.o_token;
    int buf = 0;
    bool filled = false;
    for (unsigned t0 = J.block * J.per_block; t0 < R.tokens; t0 += J.rounds * J.per_block, buf ^= 1) {
        over_jobs(
            J.first, heads << J.sub_shift, J.step,
            [&](unsigned job) __attribute__((always_inline)) {
                Raw<__bf16, W, 1> raw;
                const unsigned i = J.head(job), t = t0 + J.from(job);
                if (t + J.in_job < R.tokens) {
                    if (i < q_heads)
                        raw.load(static_cast<const __bf16 *>(R.q) + (t * R.q_token + i * R.q_head) + q_in, L);
                    else if (i < v_from)
                        raw.load(static_cast<const __bf16 *>(R.k) + (t * R.k_token + (i - q_heads) * R.k_head) + k_in, L);
                    else
                        raw.load(static_cast<const __bf16 *>(R.v) + (t * R.v_token + (i - v_from) * R.v_head) + v_in, L);
                }
                return raw;
            },
            [&]() __attribute__((always_inline)) {
                if (N.on && !filled)
                    factors.fill(N, C.head_dim);
                for (unsigned i = threadIdx.x; i < J.per_block; i += THREADS)
                    slots[buf][i] = t0 + i < R.tokens ? R.slots[t0 + i] : -1;
                if (pairs > 0)
                    table.fill(buf, A, R.positions, t0, J.per_block, R.tokens, 1.0f);
                __syncthreads();
                filled = true;
            },
            [&](unsigned job, const Raw<__bf16, W, 1> &raw) __attribute__((always_inline)) {
                const unsigned i = J.head(job), t = t0 + J.from(job);
                if (t + J.in_job >= R.tokens)
                    return;
                const bool is_q = i < q_heads, is_v = i >= v_from;   // (uniform)
                float v[1][2 * W];
                raw.get(v);
                if (!is_v) {
                    float c[1][W], s[1][W];
                    if (N.on)
                        norm_units<W, 1>(L, inv_dim, N.eps, v, factors, !is_q);
                    read_angles<W, 1>(table, buf, L, J.from(job) + J.in_job, pairs, c, s);
                    turn_units<W, 1>(L, v, c, s, INTER);
                }
                const unsigned h = is_v ? i - v_from : i - q_heads;
                const int64_t to = slots[buf][J.from(job) + J.in_job];
                const bool stored = to >= 0 && (to >> C.page_shift) < C.n_pages;
                const int64_t page = stored ? to >> C.page_shift : 0;
                const int in_page = (int)(to & ((1 << C.page_shift) - 1));
                const int64_t place = page * C.page_stride + h * C.head_stride + in_page * C.token_stride;
                if (is_q) {
                    store_units<__bf16, W, 1>(static_cast<__bf16 *>(R.q_out) + (t * R.o_token + i * R.o_head) + q_to, L, v);
                } else if constexpr (!E4M3) {
                    if (stored)
                        store_units<__bf16, W, 1>(static_cast<__bf16 *>(is_v ? C.v : C.k) + place, L, v);
                } else {
                    float top = 0.0f;
#pragma unroll
                    for (int e = 0; e < 2 * W; ++e)
                        top = fmaxf(top, __builtin_isfinite(v[0][e]) ? fabsf(v[0][e]) : 0.0f);
                    top = L.mine[0] ? top : 0.0f;
                    for (unsigned d = 1; d < lanes; d *= 2)
                        top = fmaxf(top, __shfl_xor(top, (int)d));
                    const int e = exponent_of(top);
                    if (stored && L.mine[0]) {
                        store_codes(static_cast<unsigned char *>(is_v ? C.v : C.k) + place, L.at[0], codes(v[0], e));
                        if (L.u == 0)
                            (is_v ? C.v_exp : C.k_exp)[((page * C.kv_heads + h) << C.page_shift) + in_page] = (uint8_t)(e + 127);
                    }
                }
            });
    }
}

unsigned lanes_of(int units)                                         // of a head: a power of two, at most a wave
{
    unsigned lanes = 1;
    while ((int)lanes < units && lanes < 64)
        lanes *= 2;
    return lanes;
}


// Whole accesses where a unit's two parts start on them.
bool wide_units(const HeadParams &p, int w)
{
    return p.head_dim % (2 * w) == 0 && p.rot.rot_dim % (2 * w) == 0;
}

// f(type, W, PER, layout) of the kernel that takes p, whose units of bf16 are of W pairs where that gives whole accesses
template <int W_BF16, typename F>
void for_kind(const HeadParams &p, bool bf16, F &&f)
{
    auto by_layout = [&](auto t, auto w, auto per) {
        if (p.rot.interleaved)
            f(t, w, per, std::true_type{});
        else
            f(t, w, per, std::false_type{});
    };
    using one = std::integral_constant<int, 1>;
    using two = std::integral_constant<int, 2>;
    if (bf16 && wide_units(p, W_BF16))
        by_layout((__bf16)0.0f, std::integral_constant<int, W_BF16>{}, one{});
    else if (bf16)
        by_layout((__bf16)0.0f, one{}, two{});
    else if (wide_units(p, 4))
        by_layout(0.0f, std::integral_constant<int, 4>{}, one{});
    else
        by_layout(0.0f, one{}, two{});
}

// Jobs of a head and workgroup (1 << subs_shift), and workgroups that share out the heads of its tokens: as few jobs of a head, up to MAX_SUBS, as make four
// workgroups or less for every compute unit, which it holds at once; where tokens alone do not make those, heads are shared out, with a job for every wave at the least.
struct Shape {
    unsigned subs_shift, groups;
    uint64_t blocks;                     // of tokens
};
Shape shape_of(uint64_t tokens, unsigned lanes, unsigned heads, int num_cu)
{
    const uint64_t per_job = 64 / lanes, jobs = (tokens + per_job - 1) / per_job;
    Shape s;
    s.subs_shift = 0;
    while (1 << s.subs_shift < MAX_SUBS && (jobs + (1u << s.subs_shift) - 1) >> s.subs_shift > 4 * (uint64_t)num_cu)
        ++s.subs_shift;
    s.blocks = (jobs + (1u << s.subs_shift) - 1) >> s.subs_shift;
    const uint64_t want = (4 * (uint64_t)num_cu + s.blocks - 1) / s.blocks, most = ((uint64_t)heads + WAVES - 1) / WAVES;
    s.groups = s.subs_shift > 0 ? 1 : (unsigned)(want < most ? want : most);
    return s;
}

// Workgroups of the gradient at the most, each of which leaves a row of sums.
constexpr unsigned GRAD_BLOCKS = 1024;

// The launch's shape: workgroups of at most `most` / groups rounds of tokens (more tokens: one after the other).
unsigned choose_heads(HeadParams &p, int width, unsigned most, int num_cu)
{
    p.lanes = lanes_of(p.head_dim / (wide_units(p, width) ? 2 * width : 2));
    const Shape s = shape_of(p.tokens, p.lanes, p.heads + p.kv_heads, num_cu);
    p.groups = s.groups;
    p.subs_shift = s.subs_shift;
    const uint64_t rounds = most / p.groups > 1 ? most / p.groups : 1;
    return (unsigned)(s.blocks < rounds ? s.blocks : rounds) * p.groups;
}

}  // namespace

hipError_t launch_norm_rope(const HeadParams &p_in, bool bf16, hipStream_t s, int num_cu)
{
    HeadParams p = p_in;
    const dim3 grid(choose_heads(p, bf16 ? 8 : 4, 1u << 20, num_cu));
    for_kind<8>(p, bf16, [&](auto t, auto w, auto per, auto inter) {
        hipLaunchKernelGGL((norm_rope_kernel<decltype(t), decltype(w)::value, decltype(per)::value, decltype(inter)::value>), grid, dim3(THREADS), 0, s, p);
    });
    return hipGetLastError();
}

// (a group takes WAVES heads at the least)
static size_t grad_rows(unsigned heads) { return heads / WAVES + 1 > GRAD_BLOCKS ? heads / WAVES + 1 : GRAD_BLOCKS; }
size_t norm_rope_scratch_bytes(int head_dim, unsigned heads) { return grad_rows(heads) * 2 * head_dim * sizeof(float); }

hipError_t launch_norm_rope_grad(const HeadParams &p_in, const void *dq_out, const void *dk_out, void *dq, void *dk, float *dwq, float *dwk, float *scratch,
                                 bool bf16, hipStream_t s, int num_cu)
{
    HeadParams p = p_in;
    float *sums = dwq != nullptr || dwk != nullptr ? scratch : nullptr;
    unsigned blocks = 0;
    if (p.tokens > 0 && p.heads + p.kv_heads > 0) {                  // (else the sums over nothing are zeros)
        blocks = choose_heads(p, 4, sums != nullptr ? GRAD_BLOCKS : 1u << 20, num_cu);
        const dim3 grid(blocks);
        for_kind<4>(p, bf16, [&](auto t, auto w, auto per, auto inter) {
            hipLaunchKernelGGL((norm_rope_grad_kernel<decltype(t), decltype(w)::value, decltype(per)::value, decltype(inter)::value>), grid, dim3(THREADS), 0, s, p, dq_out,
                               dk_out, dq, dk, sums);
        });
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    if (sums == nullptr)
        return hipSuccess;
    hipLaunchKernelGGL(norm_weights_kernel, dim3((2 * p.head_dim + SUM_COLUMNS - 1) / SUM_COLUMNS), dim3(SUM_THREADS), 0, s, sums, blocks, (unsigned)p.head_dim, dwq, dwk);
    return hipGetLastError();
}

hipError_t launch_cache_write_norm(const CachePool &c, const CacheRows &r_in, const AxesRotation &a, const NormParams &n, hipStream_t s, int num_cu)
{
    CacheRows r = r_in;
    const unsigned lanes = lanes_of(c.head_dim / 16), heads = (r.q != nullptr ? r.heads : 0) + 2 * c.kv_heads;
    const Shape shape = shape_of(r.tokens, lanes, heads, num_cu);
    r.groups = shape.groups;
    const uint64_t rounds = (1u << 20) / r.groups > 1 ? (1u << 20) / r.groups : 1;
    const dim3 grid((unsigned)(shape.blocks < rounds ? shape.blocks : rounds) * r.groups);
    auto launch = [&](auto e4m3, auto inter) { hipLaunchKernelGGL((cache_write_norm_kernel<decltype(e4m3)::value, decltype(inter)::value>), grid, dim3(THREADS), 0, s, c, r, a, n, lanes, shape.subs_shift); };
    using yes = std::true_type;
    using no = std::false_type;
    if (c.e4m3)
        a.interleaved ? launch(yes{}, yes{}) : launch(yes{}, no{});
    else
        a.interleaved ? launch(no{}, yes{}) : launch(no{}, no{});
    return hipGetLastError();
}

}  // namespace cf
