// Rotary positions, and the paged cache's writing and reading back.
//
// All three are bound by HBM: every feature is read and written once, with 16-byte accesses.  A thread owns a unit of one
// head: W rotated pairs (half layout: W features at j and W at j + rot_dim / 2; interleaved: 2 W in a row) or 2 W features
// that are copied, so that no value moves between lanes.  Its angles depend on the token and the unit alone: a thread goes
// over several heads of its token with them where there are threads enough to fill the chip.
// Measured: 9 heads of 8192 tokens in bf16 8.6 us, 4.4 TB/s (a copy reaches 4.7); 8 + 2 heads of 8192 tokens into an e4m3 cache and
// back, two launches, 15.5 us, 3.0 TB/s; smaller calls take what the host needs for a launch.
//
// Angle: the frequency of a pair is kept in turns per position as a 0.64-bit binary fraction, so that position * turn in
// 64-bit integers IS the angle modulo one turn, exact at any position.
#include "decoder_internal.h"

namespace cf {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));

constexpr int THREADS = 256;

// N consecutive features, in 32 bits; bf16 by eights and fp32 by fours from 16-byte lines, else one by one
template <typename T, int N>
__device__ __forceinline__ void load(const T *p, float (&x)[N])
{
    if constexpr (sizeof(T) == 2 && N % 8 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 8) {
            const bf16x8_t t = *reinterpret_cast<const bf16x8_t *>(p + i);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[i + e] = (float)t[e];
        }
    } else if constexpr (sizeof(T) == 4 && N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const f32x4_t t = *reinterpret_cast<const f32x4_t *>(p + i);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[i + e] = t[e];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            x[i] = (float)p[i];
    }
}

template <typename T, int N>
__device__ __forceinline__ void store(T *p, const float (&x)[N])
{
    if constexpr (sizeof(T) == 2 && N % 8 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 8) {
            bf16x8_t t;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                t[e] = (__bf16)x[i + e];
            *reinterpret_cast<bf16x8_t *>(p + i) = t;
        }
    } else if constexpr (sizeof(T) == 4 && N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4)
            *reinterpret_cast<f32x4_t *>(p + i) = f32x4_t{x[i], x[i + 1], x[i + 2], x[i + 3]};
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            p[i] = (T)x[i];
    }
}

// Cosine and sine of a position's angles with the W pairs from `j` on.  The phase's two upper bits and the next one say which quarter turn is
// nearest, the bits below how far it is from there, exactly: at most an eighth of a turn, where Taylor's series of both to the tenth
// power are good to 2^-28.  (An angle rounded to 32 bits as a whole is off by up to 2^-23.3; so it is by 2^-24 of at most pi / 4.)
template <int W>
__device__ __forceinline__ void angles(const uint64_t *turn, int j, int32_t position, float cos_factor, float sin_factor, float (&c)[W], float (&s)[W])
{
#pragma unroll
    for (int e = 0; e < W; ++e) {
        const uint64_t phase = (uint64_t)(int64_t)position * turn[j + e];
        const unsigned quarter = (unsigned)(phase >> 62) + ((unsigned)(phase >> 61) & 1u);
        const float x = (float)(int32_t)(unsigned)(phase >> 30) * (6.283185307179586f * 0x1p-34f), x2 = x * x;
        const float sine = __builtin_fmaf(x * x2, __builtin_fmaf(x2, __builtin_fmaf(x2, __builtin_fmaf(x2, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), x);
        const float cosine = __builtin_fmaf(x2, __builtin_fmaf(x2, __builtin_fmaf(x2, __builtin_fmaf(x2, __builtin_fmaf(x2, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
        const float cs = quarter & 1 ? sine : cosine, sn = quarter & 1 ? cosine : sine;
        c[e] = (quarter + 1 & 2 ? -cs : cs) * cos_factor;
        s[e] = (quarter & 2 ? -sn : sn) * sin_factor;
    }
}

// Where the 2 W features of unit u lie: the first W (or all) at `a`, the others at `b`.
struct Unit {
    int a, b, pair;
    bool rotated, apart;
};
template <int W>
__device__ __forceinline__ Unit unit_at(int u, int rot_dim, bool interleaved)
{
    Unit t;
    t.rotated = u * 2 * W < rot_dim;
    t.apart = t.rotated && !interleaved;
    t.pair = u * W;
    t.a = t.apart ? u * W : u * 2 * W;
    t.b = t.apart ? t.a + rot_dim / 2 : t.a + W;
    return t;
}

template <typename T, int W>
__device__ __forceinline__ void load_unit(const T *row, const Unit &at, float (&v)[2 * W])
{
    float a[W], b[W];
    load<T, W>(row + at.a, a);
    load<T, W>(row + at.b, b);
#pragma unroll
    for (int e = 0; e < W; ++e) {
        v[e] = a[e];
        v[W + e] = b[e];
    }
}

template <typename T, int W>
__device__ __forceinline__ void store_unit(T *row, const Unit &at, const float (&v)[2 * W])
{
    float a[W], b[W];
#pragma unroll
    for (int e = 0; e < W; ++e) {
        a[e] = v[e];
        b[e] = v[W + e];
    }
    store<T, W>(row + at.a, a);
    store<T, W>(row + at.b, b);
}

// The rotated unit: x holds features a .. a + W - 1, then b .. b + W - 1.  (Which product is rounded is written down: left to the compiler,
// a row that the cache's writer rotates and one rotated by itself came out a bit apart now and then.)
template <int W>
__device__ __forceinline__ void turn_unit(float (&x)[2 * W], const float (&c)[W], const float (&s)[W], bool interleaved)
{
    if (interleaved) {
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const float p = x[2 * e], q = x[2 * e + 1];
            x[2 * e] = __builtin_fmaf(p, c[e], -(q * s[e]));
            x[2 * e + 1] = __builtin_fmaf(q, c[e], p * s[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const float p = x[e], q = x[W + e];
            x[e] = __builtin_fmaf(p, c[e], -(q * s[e]));
            x[W + e] = __builtin_fmaf(q, c[e], p * s[e]);
        }
    }
}

template <typename T, int W>
__global__ __launch_bounds__(THREADS) void rope_kernel(RopeParams P)
{
    const unsigned units = P.head_dim / (2 * W), per_block = THREADS / units;
    const unsigned local = threadIdx.x / units, u = threadIdx.x - local * units;
    if (local >= per_block)
        return;
    const Unit at = unit_at<W>(u, P.rot_dim, P.interleaved);
    for (unsigned item = blockIdx.x * per_block + local; item < P.tokens * P.groups; item += gridDim.x * per_block) {
        const unsigned token = item / P.groups, group = item - token * P.groups;
        float c[W], s[W];
        if (at.rotated)
            angles<W>(P.turn, at.pair, P.positions[token], P.cos_factor, P.sin_factor, c, s);
        const T *x = static_cast<const T *>(P.x) + (int64_t)token * P.x_token;
        T *out = static_cast<T *>(P.out) + (int64_t)token * P.o_token;
        for (unsigned h = group; h < P.heads; h += P.groups) {
            float v[2 * W];
            load_unit<T, W>(x + h * P.x_head, at, v);
            if (at.rotated)
                turn_unit<W>(v, c, s, P.interleaved);
            store_unit<T, W>(out + h * P.o_head, at, v);
        }
    }
}

// Sixteen values as e4m3 codes of x * 2^-e (rounded to nearest even; |x * 2^-e| <= 448 by the choice of e, and with e = 120
// no code above 240: the next, 256, would stand for 2^128).
__device__ __forceinline__ u32x4_t codes(const float (&x)[16], int e)
{
    const float most = e < 120 ? 448.0f : 240.0f;
    u32x4_t r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float t[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float y = fminf(fmaxf(ldexpf(x[4 * i + k], -e), -most), most);
            t[k] = __builtin_isfinite(x[4 * i + k]) ? y : __builtin_nanf("");
        }
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], w, true);
        r[i] = (unsigned)w;
    }
    return r;
}

// One row of one head: `lanes` (a power of two) neighbouring lanes share its amax.
template <bool E4M3>
__global__ __launch_bounds__(THREADS) void cache_write_kernel(CachePool C, CacheRows R)
{
    constexpr int W = 8;
    const unsigned units = C.head_dim / 16;
    unsigned lanes = 1;
    while (lanes < units)
        lanes *= 2;
    const unsigned per_block = THREADS / lanes, total = R.tokens * R.groups;
    const unsigned u = threadIdx.x & (lanes - 1);
    const Unit at = unit_at<W>(u, R.rot_dim, R.interleaved);
    const unsigned heads = R.q != nullptr ? R.heads : 0, rows = heads + 2 * C.kv_heads;
    for (unsigned base = blockIdx.x * per_block; base < total; base += gridDim.x * per_block) {
        const unsigned item = base + threadIdx.x / lanes;
        const bool there = item < total && u < units;
        const unsigned token = there ? item / R.groups : 0, group = there ? item - token * R.groups : 0;
        float c[W], s[W];
        if (there && at.rotated && group < heads + C.kv_heads)
            angles<W>(R.turn, at.pair, R.positions[token], R.magnitude, R.magnitude, c, s);
        const int64_t slot = there ? R.slots[token] : -1;
        const bool stored = slot >= 0 && (slot >> C.page_shift) < C.n_pages;
        const int64_t page = stored ? slot >> C.page_shift : 0;
        const int in_page = (int)(slot & ((1 << C.page_shift) - 1));
        for (unsigned first = 0; first < rows; first += R.groups) {  // (uniform: every lane takes part in the exchanges)
            const unsigned row = first + group;
            const bool mine = there && row < rows;
            const bool is_q = row < heads, is_v = row >= heads + C.kv_heads;
            const unsigned h = is_q ? row : is_v ? row - heads - C.kv_heads : row - heads;
            float v[2 * W] = {};
            if (mine) {
                load_unit<__bf16, W>(is_q ? static_cast<const __bf16 *>(R.q) + (int64_t)token * R.q_token + h * R.q_head
                                     : is_v ? static_cast<const __bf16 *>(R.v) + (int64_t)token * R.v_token + h * R.v_head
                                            : static_cast<const __bf16 *>(R.k) + (int64_t)token * R.k_token + h * R.k_head, at, v);
                if (at.rotated && !is_v)
                    turn_unit<W>(v, c, s, R.interleaved);
            }
            const int64_t place = page * C.page_stride + h * C.head_stride + in_page * C.token_stride;
            if (!E4M3 || is_q) {
                if (mine && is_q)
                    store_unit<__bf16, W>(static_cast<__bf16 *>(R.q_out) + (int64_t)token * R.o_token + h * R.o_head, at, v);
                else if (mine && stored)
                    store_unit<__bf16, W>(static_cast<__bf16 *>(is_v ? C.v : C.k) + place, at, v);
            }
            if constexpr (E4M3) {
                float top = 0.0f;
#pragma unroll
                for (int i = 0; i < 2 * W; ++i)
                    top = fmaxf(top, __builtin_isfinite(v[i]) ? fabsf(v[i]) : 0.0f);
                for (unsigned d = 1; d < lanes; d *= 2)
                    top = fmaxf(top, __shfl_xor(top, (int)d));
                const int bits = __builtin_bit_cast(int, top);
                int e = (bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000 ? 1 : 0);     // 448 = 1.75 * 2^8
                e = bits == 0 ? 0 : e < -126 ? -126 : e;
                if (mine && !is_q && stored) {
                    unsigned char *dst = static_cast<unsigned char *>(is_v ? C.v : C.k) + place;
                    const u32x4_t w = codes(v, e);
                    if (at.apart) {
                        *reinterpret_cast<u32x2_t *>(dst + at.a) = u32x2_t{w[0], w[1]};
                        *reinterpret_cast<u32x2_t *>(dst + at.b) = u32x2_t{w[2], w[3]};
                    } else {
                        *reinterpret_cast<u32x4_t *>(dst + at.a) = w;
                    }
                    if (u == 0)
                        (is_v ? C.v_exp : C.k_exp)[((page * C.kv_heads + h) << C.page_shift) + in_page] = (uint8_t)(e + 127);
                }
            }
        }
    }
}

// Sixteen features a thread (e4m3) or eight (bf16): a row of K or V of one token and head.
template <bool E4M3>
__global__ __launch_bounds__(THREADS) void cache_read_kernel(CachePool C, CacheRows R, __bf16 *K, __bf16 *V)
{
    constexpr unsigned N = E4M3 ? 16 : 8;
    const unsigned units = C.head_dim / N, per_block = THREADS / units;
    const unsigned local = threadIdx.x / units, u = threadIdx.x - local * units;
    const unsigned rows = 2 * C.kv_heads;
    if (local >= per_block)
        return;
    for (unsigned item = blockIdx.x * per_block + local; item < R.tokens * rows; item += gridDim.x * per_block) {
        const unsigned token = item / rows, row = item - token * rows;
        const bool is_v = row >= (unsigned)C.kv_heads;
        const unsigned h = is_v ? row - C.kv_heads : row;
        const int64_t slot = R.slots[token], page = slot >> C.page_shift;
        if (slot < 0 || page >= C.n_pages)
            continue;
        const int in_page = (int)(slot & ((1 << C.page_shift) - 1));
        const int64_t at = page * C.page_stride + h * C.head_stride + in_page * C.token_stride + u * N;
        __bf16 *dst = (is_v ? V + (int64_t)token * R.v_token + h * R.v_head : K + (int64_t)token * R.k_token + h * R.k_head) + u * N;
        if constexpr (E4M3) {
            const u32x4_t w = *reinterpret_cast<const u32x4_t *>(static_cast<const unsigned char *>(is_v ? C.v : C.k) + at);
            const int e = (int)(is_v ? C.v_exp : C.k_exp)[((page * C.kv_heads + h) << C.page_shift) + in_page] - 127;
            float x[16];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
                x[4 * i] = ldexpf(lo[0], e);
                x[4 * i + 1] = ldexpf(lo[1], e);
                x[4 * i + 2] = ldexpf(hi[0], e);
                x[4 * i + 3] = ldexpf(hi[1], e);
            }
            store<__bf16, 16>(dst, x);
        } else {
            *reinterpret_cast<u32x4_t *>(dst) = *reinterpret_cast<const u32x4_t *>(static_cast<const __bf16 *>(is_v ? C.v : C.k) + at);
        }
    }
}

// Groups that a token's heads are shared out to: as few as fill the chip with four waves per SIMD.
unsigned groups_of(unsigned tokens, unsigned lanes, unsigned rows, int num_cu)
{
    const uint64_t threads = (uint64_t)num_cu * 1024, per_group = (uint64_t)tokens * lanes;
    const uint64_t g = (threads + per_group - 1) / per_group;
    return g < rows ? (unsigned)g : rows;
}

// (HIP counts threads in 32 bits: larger launches go over their items in rounds)
unsigned blocks_of(uint64_t items, unsigned per_block)
{
    const uint64_t b = (items + per_block - 1) / per_block;
    return b < (1u << 20) ? (unsigned)b : 1u << 20;
}

template <typename T, int W>
hipError_t launch(const RopeParams &p, hipStream_t s)
{
    const unsigned per_block = THREADS / (p.head_dim / (2 * W));
    hipLaunchKernelGGL((rope_kernel<T, W>), dim3(blocks_of((uint64_t)p.tokens * p.groups, per_block)), dim3(THREADS), 0, s, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeParams &p_in, bool bf16, hipStream_t s, int num_cu)
{
    RopeParams p = p_in;
    // whole 16-byte accesses where the unit's two parts start on them
    const int w = bf16 ? 8 : 4;
    const bool wide = p.head_dim % (2 * w) == 0 && p.rot_dim % (2 * w) == 0;
    p.groups = groups_of(p.tokens, p.head_dim / (wide ? 2 * w : 2), p.heads, num_cu);
    if (bf16)
        return wide ? launch<__bf16, 8>(p, s) : launch<__bf16, 1>(p, s);
    return wide ? launch<float, 4>(p, s) : launch<float, 1>(p, s);
}

hipError_t launch_cache_write(const CachePool &c, const CacheRows &r_in, hipStream_t s, int num_cu)
{
    CacheRows r = r_in;
    const unsigned units = c.head_dim / 16;
    unsigned lanes = 1;
    while (lanes < units)
        lanes *= 2;
    r.groups = groups_of(r.tokens, lanes, (r.q != nullptr ? r.heads : 0) + 2 * c.kv_heads, num_cu);
    const unsigned per_block = THREADS / lanes;
    const dim3 grid(blocks_of((uint64_t)r.tokens * r.groups, per_block));
    if (c.e4m3)
        hipLaunchKernelGGL((cache_write_kernel<true>), grid, dim3(THREADS), 0, s, c, r);
    else
        hipLaunchKernelGGL((cache_write_kernel<false>), grid, dim3(THREADS), 0, s, c, r);
    return hipGetLastError();
}

hipError_t launch_cache_read(const CachePool &c, const CacheRows &r, void *K, void *V, hipStream_t s)
{
    const unsigned per_block = THREADS / (c.head_dim / (c.e4m3 ? 16 : 8));
    const dim3 grid(blocks_of((uint64_t)r.tokens * 2 * c.kv_heads, per_block));
    __bf16 *k = static_cast<__bf16 *>(K), *v = static_cast<__bf16 *>(V);
    if (c.e4m3)
        hipLaunchKernelGGL((cache_read_kernel<true>), grid, dim3(THREADS), 0, s, c, r, k, v);
    else
        hipLaunchKernelGGL((cache_read_kernel<false>), grid, dim3(THREADS), 0, s, c, r, k, v);
    return hipGetLastError();
}

}  // namespace cf
