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
#include "rope_units.h"

namespace cf {
namespace {

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
                const int e = exponent_of(top);
                if (mine && !is_q && stored) {
                    unsigned char *dst = static_cast<unsigned char *>(is_v ? C.v : C.k) + place;
                    store_codes(dst, at, codes(v, e));
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
