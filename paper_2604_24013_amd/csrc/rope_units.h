// Device helpers of the kernels that rotate heads: units of features that a thread loads, turns and stores, cosines and sines of exact
// angles, e4m3 codes.
#pragma once
#include "decoder_internal.h"

#include <cmath>
#include <type_traits>

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

// Position times turn, modulo one turn, in units of 2^-64.  (By two products of 32 bits: the sign of a position takes the turn's lower half off the upper.)
__device__ __forceinline__ uint64_t phase_of(uint64_t turn, int32_t position)
{
    const unsigned lo = (unsigned)turn, hi = (unsigned)(turn >> 32), u = (unsigned)position;
    const uint64_t low = (uint64_t)u * lo;
    return low + ((uint64_t)(u * hi - (position < 0 ? lo : 0u)) << 32);
}

// Cosine and sine of a phase.  Its two upper bits and the next one say which quarter turn is
// nearest, the bits below how far it is from there, exactly: at most an eighth of a turn, where Taylor's series of both to the tenth
// power are good to 2^-28.  (An angle rounded to 32 bits as a whole is off by up to 2^-23.3; so it is by 2^-24 of at most pi / 4.)
__device__ __forceinline__ void cos_sin(uint64_t phase, float cos_factor, float sin_factor, float *c, float *s)
{
    const unsigned quarter = (unsigned)(phase >> 62) + ((unsigned)(phase >> 61) & 1u);
    const float x = (float)(int32_t)(unsigned)(phase >> 30) * (6.283185307179586f * 0x1p-34f), x2 = x * x;
    const float sine = __builtin_fmaf(x * x2, __builtin_fmaf(x2, __builtin_fmaf(x2, __builtin_fmaf(x2, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), x);
    const float cosine = __builtin_fmaf(x2, __builtin_fmaf(x2, __builtin_fmaf(x2, __builtin_fmaf(x2, __builtin_fmaf(x2, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
    const float cs = quarter & 1 ? sine : cosine, sn = quarter & 1 ? cosine : sine;
    *c = (quarter + 1 & 2 ? -cs : cs) * cos_factor;
    *s = (quarter & 2 ? -sn : sn) * sin_factor;
}
template <int W>
__device__ __forceinline__ void angles(const uint64_t *turn, int j, int32_t position, float cos_factor, float sin_factor, float (&c)[W], float (&s)[W])
{
#pragma unroll
    for (int e = 0; e < W; ++e)
        cos_sin(phase_of(turn[j + e], position), cos_factor, sin_factor, &c[e], &s[e]);
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

// The smallest e with top <= 448 * 2^e (448 = 1.75 * 2^8), in [-126, 120]; 0 for a row of zeros.
__device__ __forceinline__ int exponent_of(float top)
{
    const int bits = __builtin_bit_cast(int, top);
    const int e = (bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000 ? 1 : 0);
    return bits == 0 ? 0 : e < -126 ? -126 : e;
}

__device__ __forceinline__ void store_codes(unsigned char *row, const Unit &at, const u32x4_t &w)
{
    if (at.apart) {
        *reinterpret_cast<u32x2_t *>(row + at.a) = u32x2_t{w[0], w[1]};
        *reinterpret_cast<u32x2_t *>(row + at.b) = u32x2_t{w[2], w[3]};
    } else {
        *reinterpret_cast<u32x4_t *>(row + at.a) = w;
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

}  // namespace
}  // namespace cf
