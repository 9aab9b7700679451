// Gradient of causal attention over packed prompts for gfx950: dQ, dK, dV from bf16 operands, fp32 accumulation.
//   P = exp(scale q k - lse),  delta = sum dout out,  dP = dout v,  dS = P (dP - delta)
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dout
// Two launches, each with every sum in one place (no atomics, the same bits every time): one workgroup of the first owns rows and
// walks over keys (and leaves delta for the second), one of the second owns keys and walks over the rows that see them, all
// query heads of the key head.  Both multiply the scores anew: seven products where five would do with sums spread over memory.
// As in the forward kernel a lane owns one row (or key) and 16 of every 32 keys (rows) of a product's result, which is, rounded to
// bf16, the "B" operand of the next product as it stands: nothing moves between lanes.  Tiles lie in LDS once and are read both by rows
// and transposed: 16-byte chunks XOR-ed with (row & 15), which the transposing read can follow lane by lane.
// Rows behind a walk are read from its last row, or as zero, and masked.  A result that is not finite is computed once more over what is
// visible only, so that what the mask hides has no influence.
#include "attn_tiles.h"

namespace cf {
namespace {

constexpr int DS = DH / 16;              // 16-wide feature slices
constexpr int DT = DH / 32;              // 32-wide feature tiles

// Wave-wide 16-byte-per-lane (or 4-byte) load from per-lane addresses straight into LDS (lane L lands at lds_addr + 16 L or 4 L).
__device__ __forceinline__ void gather_load_16(const void *at, unsigned lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\t"
                 "global_load_lds_dwordx4 %1, off"
                 :
                 : "s"(lds_addr), "v"(at)
                 : "memory");
}
__device__ __forceinline__ void gather_load_4(const void *at, unsigned lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\t"
                 "global_load_lds_dword %1, off"
                 :
                 : "s"(lds_addr), "v"(at)
                 : "memory");
}

// Addresses inside a tile of rows of 256 bytes whose 16-byte chunks are XOR-ed with (row & 15).
struct TileRead {
    int row[DS];                         // "A" operand: lane (row = lane & 31, half = lane >> 5), chunk 2 ks + half
    int lo, hi;                          // its transposed: rows 4 half + .. and 8 more of a slice of 16; feature tile t at (lo ^ t << 6)
    __device__ __forceinline__ TileRead()
    {
        const int lane = threadIdx.x & 63, lq = lane & 31, lh = lane >> 5, blk = lane >> 4, i16 = lane & 15;
#pragma unroll
        for (int ks = 0; ks < DS; ++ks)
            row[ks] = lq * ROWB + (((2 * ks + lh) ^ (lq & 15)) << 4);
        const int r = 4 * (blk >> 1) + (i16 >> 2), c = 2 * (blk & 1) + ((i16 & 3) >> 1);
        lo = r * ROWB + ((c ^ r) << 4) + (i16 & 1) * 8;
        hi = (r + 8) * ROWB + ((c ^ (r + 8)) << 4) + (i16 & 1) * 8;
    }
    __device__ __forceinline__ bf16x8_t rows(const unsigned char *tile, int ks) const { return *reinterpret_cast<const bf16x8_t *>(tile + row[ks]); }
    __device__ __forceinline__ bf16x8_t transposed(const unsigned char *slice, int t) const
    {
        const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)(slice + (lo ^ (t << 6))));
        const s16x4_t c = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)(slice + (hi ^ (t << 6))));
        return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(a, c, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// Split sums: N registers of every thread parked in the workspace, added up in split order by the workgroup that arrives last; false:
// not this one.
template <int N, int NT>
__device__ __forceinline__ bool join_splits(float (&x)[N], const CausalParams &P, int group, int split, int splits, unsigned *arrived)
{
    constexpr int COHERENT = 1 | 16;
    const int tid = threadIdx.x;
    const size_t part = (size_t)N * NT;
    auto rsrc = [&](int sp) {
        return __builtin_amdgcn_make_buffer_rsrc(P.parts + ((size_t)group * P.max_splits + sp) * part, 0, (int)(part * 4), 0x00020000);
    };
    {
        __amdgpu_buffer_rsrc_t rs = rsrc(split);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float v = x[i];
            asm volatile("" : "+v"(v));      // (through a plain VGPR, as in the forward kernel)
            __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), rs, (i * NT + tid) * 4, 0, COHERENT);
        }
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (tid == 0)
        *arrived = __hip_atomic_fetch_add(&P.counters[group], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (*arrived != (unsigned)(splits - 1))
        return false;
    if (tid == 0)
        __hip_atomic_store(&P.counters[group], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
    for (int i = 0; i < N; ++i)
        x[i] = 0.0f;
    for (int sp = 0; sp < splits; ++sp) {
        __amdgpu_buffer_rsrc_t rs = rsrc(sp);
        constexpr int AT = 64;
#pragma unroll
        for (int i0 = 0; i0 < N; i0 += AT) {
            float v[AT];
#pragma unroll
            for (int i = 0; i < AT; ++i)
                v[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rs, ((i0 + i) * NT + tid) * 4, 0, COHERENT));
#pragma unroll
            for (int i = 0; i < AT; ++i)
                x[i0 + i] += v[i];
        }
    }
    return true;
}

__device__ __forceinline__ float wave_sum(float x)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
        x += __shfl_xor(x, d);
    return x;
}
__device__ __forceinline__ f32x2_t pair_at(const void *row)          // features 2 lane, 2 lane + 1
{
    const bf16x2_t v = static_cast<const bf16x2_t *>(row)[threadIdx.x & 63];
    return f32x2_t{(float)v[0], (float)v[1]};
}
__device__ __forceinline__ void put_pair(void *row, float a, float b)
{
    bf16x2_t v;
    v[0] = (__bf16)a;
    v[1] = (__bf16)b;
    static_cast<bf16x2_t *>(row)[threadIdx.x & 63] = v;
}

// dQ of one row, key by key.
__device__ __forceinline__ void careful_dq(const GradParams &P, int t, int head, int first, float delta)
{
    const CausalParams &C = P.c;
    const int kvh = head / C.group;
    const __bf16 *K = static_cast<const __bf16 *>(C.K) + kvh * C.k_head, *V = static_cast<const __bf16 *>(C.V) + kvh * C.v_head;
    const f32x2_t q = pair_at(static_cast<const __bf16 *>(C.Q) + (int64_t)t * C.q_token + head * C.q_head);
    const f32x2_t g = pair_at(static_cast<const __bf16 *>(P.dout) + (int64_t)t * C.o_token + head * C.o_head);
    const float lse = C.lse[(int64_t)head * C.lse_stride + t];
    float a = 0.0f, b = 0.0f;
    for (int key = first; key <= t; ++key) {
        const f32x2_t k = pair_at(K + (int64_t)key * C.k_token), v = pair_at(V + (int64_t)key * C.v_token);
        const float s = wave_sum(q[0] * k[0] + q[1] * k[1]), dp = wave_sum(g[0] * v[0] + g[1] * v[1]);
        const float ds = exp2f((s * C.scale - lse) * LOG2E) * (dp - delta);
        a += ds * k[0];
        b += ds * k[1];
    }
    put_pair(static_cast<__bf16 *>(P.dq) + (int64_t)t * C.q_token + head * C.q_head, a * C.scale, b * C.scale);
}

// dK and dV of one key, row by row.
__device__ __forceinline__ void careful_key(const GradParams &P, int key, int kvh, int end)
{
    const CausalParams &C = P.c;
    const f32x2_t k = pair_at(static_cast<const __bf16 *>(C.K) + (int64_t)key * C.k_token + kvh * C.k_head);
    const f32x2_t v = pair_at(static_cast<const __bf16 *>(C.V) + (int64_t)key * C.v_token + kvh * C.v_head);
    float ka = 0.0f, kb = 0.0f, va = 0.0f, vb = 0.0f;
    for (int head = kvh * C.group; head < (kvh + 1) * C.group; ++head)
        for (int t = key; t < end; ++t) {
            const f32x2_t q = pair_at(static_cast<const __bf16 *>(C.Q) + (int64_t)t * C.q_token + head * C.q_head);
            const f32x2_t g = pair_at(static_cast<const __bf16 *>(P.dout) + (int64_t)t * C.o_token + head * C.o_head);
            const float s = wave_sum(q[0] * k[0] + q[1] * k[1]), dp = wave_sum(g[0] * v[0] + g[1] * v[1]);
            const int64_t at = (int64_t)head * C.lse_stride + t;
            const float p = exp2f((s * C.scale - C.lse[at]) * LOG2E), ds = p * (dp - P.delta[at]);
            ka += ds * q[0];
            kb += ds * q[1];
            va += p * g[0];
            vb += p * g[1];
        }
    put_pair(static_cast<__bf16 *>(P.dk) + (int64_t)key * C.k_token + kvh * C.k_head, ka * C.scale, kb * C.scale);
    put_pair(static_cast<__bf16 *>(P.dv) + (int64_t)key * C.v_token + kvh * C.v_head, va, vb);
}

// A lane's row of a result X^T (feature tiles by registers), times `factor`, as bf16.  True if a value is not finite.
__device__ __forceinline__ bool store_row(const float *x, float factor, __bf16 *row, bool there)
{
    const int lh = (threadIdx.x & 63) >> 5;
    float odd = 0.0f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            bf16x4_t h;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float y = x[d * 16 + 4 * g + e] * factor;
                odd = __builtin_fmaf(y, 0.0f, odd);
                h[e] = (__bf16)y;
            }
            if (there)
                *reinterpret_cast<u32x2_t *>(row + d * 32 + 8 * g + 4 * lh) = __builtin_bit_cast(u32x2_t, h);
        }
    return there && odd != 0.0f;
}

// The sequence of token t, between two that enclose it: how many of starts[1 ..] are <= t.
__device__ __forceinline__ int sequence_between(const int32_t *starts, int a, int b, int t)
{
    while (a < b) {
        const int mid = (a + b) >> 1;
        if (starts[mid + 1] <= t)
            a = mid + 1;
        else
            b = mid;
    }
    return a;
}

template <int NW>
__global__ __launch_bounds__(64 * NW, 2) void attn_dq_kernel(GradParams P)
{
    const CausalParams &C = P.c;
    constexpr int NT = 64 * NW, BQ = NW * 32;
    constexpr int LOADS = TILE_BYTES / 1024 / NW;                    // wave-loads per wave of a K or V tile: four rows each
    __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * TILE_BYTES];    // K, K, V, V

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lq = lane & 31, lh = lane >> 5;
    const int G = C.group;

    // Rows and walk as in the forward kernel
    const int kvh = blockIdx.x % C.kv_heads;
    int rest = blockIdx.x / C.kv_heads;
    const int groups = gridDim.x / (unsigned)(C.kv_heads * C.max_splits);
    const int split = rest / groups;
    rest -= split * groups;
    const int64_t r0 = (int64_t)(groups - 1 - rest) * BQ;
    const int64_t r1 = r0 + BQ < (int64_t)C.tokens * G ? r0 + BQ : (int64_t)C.tokens * G;
    const int t_base = (int)(r0 / G), t_last = (int)((r1 - 1) / G), row0 = (int)(r0 - (int64_t)t_base * G);
    const int seq_a = sequence_of(C.starts, C.n_seqs, t_base);
    if (seq_a == C.n_seqs)
        return;
    const int seq_b = sequence_of(C.starts, C.n_seqs, t_last);
    const int begin = C.starts[seq_a], stop = C.starts[C.n_seqs];
    const int lo = begin < 0 ? 0 : begin, hi = t_last + 1 < stop ? t_last + 1 : stop;
    if (lo >= hi)
        return;
    const int tiles = (hi - lo + BKV - 1) / BKV;
    const int splits = C.chunk > 0 && tiles > C.chunk ? (tiles + C.chunk - 1) / C.chunk : 1;
    if (split >= splits)
        return;
    const int kt0 = (int)(((int64_t)tiles * split) / splits), nkt = (int)(((int64_t)tiles * (split + 1)) / splits);

    const int r = row0 + wave * 32 + lq;
    const int rt = r / G, head = kvh * G + r - rt * G;
    bool there = t_base + rt <= t_last;
    const int t = t_base + (there ? rt : 0);
    const int a = sequence_between(C.starts, seq_a, seq_b, t);
    int first = a < C.n_seqs ? C.starts[a] : t + 1;
    there = there && first <= t;
    first = there ? (first < 0 ? 0 : first) : t;
    int wt0 = kt0, wt1 = kt0, all_from, all_to;
    {
        int f_min = there ? first : 0x7FFFFFFF, f_max = there ? first : 0, l_min = there ? t : 0x7FFFFFFF, l_max = there ? t : -1;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            f_min = min(f_min, __shfl_xor(f_min, d));
            f_max = max(f_max, __shfl_xor(f_max, d));
            l_min = min(l_min, __shfl_xor(l_min, d));
            l_max = max(l_max, __shfl_xor(l_max, d));
        }
        f_min = uniform(f_min);
        l_max = uniform(l_max);
        all_from = uniform(f_max) - lo;
        all_to = uniform(l_min) - lo;
        if (l_max >= f_min) {
            wt0 = max(kt0, (f_min - lo) / BKV);
            wt1 = min(nkt, (l_max - lo) / BKV + 1);
        }
    }

    // Tile loads, straight into LDS
    const unsigned lds_base = lds_address(smem);
    const int ld_row = wave * 4 + (lane >> 4);
    const unsigned swizzled = ((lane & 15) ^ (ld_row & 15)) << 4;
    const unsigned k_off = (unsigned)((lane >> 4) * (int)(C.k_token * 2)) + swizzled, v_off = (unsigned)((lane >> 4) * (int)(C.v_token * 2)) + swizzled;
    const unsigned char *kb = static_cast<const unsigned char *>(C.K) + kvh * C.k_head * 2, *vb = static_cast<const unsigned char *>(C.V) + kvh * C.v_head * 2;
    auto issue = [&](int kt, const unsigned char *base, int64_t row_bytes, unsigned off, unsigned lds) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int key = lo + kt * BKV + wave * 4 + j * NW * 4, left = hi - key < 4 ? hi - key : 4;
            direct_load_16(make_rsrc(base + (int64_t)key * row_bytes, left > 0 ? (unsigned)(left * (int)row_bytes) : 0u), off,
                           lds + wave * 1024 + j * NW * 1024);
        }
    };
    issue(kt0, kb, C.k_token * 2, k_off, lds_base);
    issue(kt0, vb, C.v_token * 2, v_off, lds_base + 2 * TILE_BYTES);

    bf16x8_t qf[DS], gf[DS];
    float delta = 0.0f;
    {
        const __bf16 *q = static_cast<const __bf16 *>(C.Q) + (int64_t)t * C.q_token + head * C.q_head + lh * 8;
        const __bf16 *g = static_cast<const __bf16 *>(P.dout) + (int64_t)t * C.o_token + head * C.o_head + lh * 8;
        const __bf16 *o = static_cast<const __bf16 *>(C.out) + (int64_t)t * C.o_token + head * C.o_head + lh * 8;
#pragma unroll
        for (int ks = 0; ks < DS; ++ks) {
            qf[ks] = *reinterpret_cast<const bf16x8_t *>(q + ks * 16);
            gf[ks] = *reinterpret_cast<const bf16x8_t *>(g + ks * 16);
            const bf16x8_t of = *reinterpret_cast<const bf16x8_t *>(o + ks * 16);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                delta = __builtin_fmaf((float)gf[ks][e], (float)of[e], delta);
        }
        delta = sum_of_halves(delta);
    }
    if (split == 0 && there && lh == 0)
        P.delta[(int64_t)head * C.lse_stride + t] = delta;
    const float sl2 = C.scale * LOG2E, lse2 = C.lse[(int64_t)head * C.lse_stride + t] * LOG2E;

    const TileRead at;
    f32x16_t acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            acc[d][e] = 0.0f;

    wait_vmcnt<0>();
    __syncthreads();
    for (int kt = kt0; kt < nkt; ++kt) {
        const int b = (kt - kt0) & 1;
        if (kt + 1 < nkt) {
            issue(kt + 1, kb, C.k_token * 2, k_off, lds_base + (1 - b) * TILE_BYTES);
            issue(kt + 1, vb, C.v_token * 2, v_off, lds_base + (3 - b) * TILE_BYTES);
        }
        if (kt >= wt0 && kt < wt1) {
            const bool border = kt * BKV < all_from || (kt + 1) * BKV - 1 > all_to;
#pragma unroll
            for (int j = 0; j < 2; ++j) {                            // 32 keys at a time
                const unsigned char *kt_at = smem + b * TILE_BYTES + j * 32 * ROWB, *vt_at = smem + (2 + b) * TILE_BYTES + j * 32 * ROWB;
                f32x16_t s, dp;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    s[e] = dp[e] = 0.0f;
#pragma unroll
                for (int ks = 0; ks < DS; ++ks) {
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.rows(kt_at, ks), qf[ks], s, 0, 0, 0);
                    dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.rows(vt_at, ks), gf[ks], dp, 0, 0, 0);
                }
                if (border) {
                    const unsigned key0 = (unsigned)(lo + kt * BKV + j * 32 + 4 * lh - first), span = (unsigned)(t - first);
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (key0 + (unsigned)(8 * (e >> 2) + (e & 3)) > span)
                            s[e] = -INFINITY;
                }
                bf16x8_t df[2];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], sl2, -lse2));
                    df[e >> 3][e & 7] = (__bf16)(p * (dp[e] - delta));
                }
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int d = 0; d < DT; ++d)
                        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.transposed(kt_at + c * 16 * ROWB, d), df[c], acc[d], 0, 0, 0);
            }
        }
        if (kt + 1 < nkt) {
            wait_vmcnt<0>();
            __syncthreads();
        }
    }

    float x[DT * 16];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            x[d * 16 + e] = acc[d][e];
    if (splits > 1) {
        __syncthreads();
        if (!join_splits<DT * 16, NT>(x, C, rest * C.kv_heads + kvh, split, splits, reinterpret_cast<unsigned *>(smem)))
            return;
    }
    const bool odd = store_row(x, C.scale, static_cast<__bf16 *>(P.dq) + (int64_t)t * C.q_token + head * C.q_head, there);
    unsigned long long again = __builtin_amdgcn_ballot_w64(odd);
    again = (again | again >> 32) & 0xFFFFFFFFull;
    if (again != 0) {
        __builtin_amdgcn_s_waitcnt(0);                               // the row's first result is written before its second
        for (; again != 0; again &= again - 1) {
            const int l = __builtin_ctzll(again);
            careful_dq(P, __shfl(t, l), __shfl(head, l), __shfl(first, l), __shfl(delta, l));
        }
    }
}

constexpr int GRAD_KEYS = 128;           // keys of a workgroup of the second launch: four waves of 32

__global__ __launch_bounds__(256, 1) void attn_dkv_kernel(GradParams P)
{
    const CausalParams &C = P.c;
    constexpr int NT = 256, ROWS = 64;                               // rows per tile
    __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * TILE_BYTES];    // Q, Q, dout, dout
    __shared__ __attribute__((aligned(16))) float stat[2][2][ROWS];  // buffer; lse, delta
    __shared__ unsigned arrived;

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lq = lane & 31, lh = lane >> 5;
    const int G = C.group;

    const int kvh = blockIdx.x % C.kv_heads;
    int rest = blockIdx.x / C.kv_heads;
    const int groups = gridDim.x / (unsigned)(C.kv_heads * C.max_splits);
    const int split = rest / groups;
    rest -= split * groups;
    const int k0 = rest * GRAD_KEYS;                                 // (the first keys are seen by most rows)
    const int stop = C.starts[C.n_seqs] < C.tokens ? C.starts[C.n_seqs] : C.tokens;
    const int k1 = k0 + GRAD_KEYS < stop ? k0 + GRAD_KEYS : stop;
    const int begin = C.starts[0] > k0 ? C.starts[0] : k0;
    if (begin >= k1)
        return;
    const int seq_a = sequence_of(C.starts, C.n_seqs, begin), seq_b = sequence_of(C.starts, C.n_seqs, k1 - 1);
    if (seq_b >= C.n_seqs)
        return;
    const int end_b = C.starts[seq_b + 1] < C.tokens ? C.starts[seq_b + 1] : C.tokens;
    if (end_b <= begin)
        return;
    // The walk over rows [lo, hi) = (token, head of the group), tokens [begin, end_b)
    const int lo = begin * G, hi = end_b * G;
    const int tiles = (int)(((int64_t)hi - lo + ROWS - 1) / ROWS);
    const int splits = C.chunk > 0 && tiles > C.chunk ? (tiles + C.chunk - 1) / C.chunk : 1;
    if (split >= splits)
        return;
    const int rt0 = (int)(((int64_t)tiles * split) / splits), nrt = (int)(((int64_t)tiles * (split + 1)) / splits);

    // The lane's key, seen by rows [from, to)
    const int key = k0 + wave * 32 + lq;
    bool there = key >= begin && key < k1;
    const int kk = there ? key : begin;
    const int a = sequence_between(C.starts, seq_a, seq_b, kk);
    int end = a < C.n_seqs ? C.starts[a + 1] : 0;
    end = end < end_b ? end : end_b;
    there = there && end > kk;
    const int from = kk * G, to = there ? end * G : from;
    int wr0 = rt0, wr1 = rt0, all_from, all_to;
    {
        int f_min = there ? from : 0x7FFFFFFF, f_max = there ? from : 0, l_min = there ? to : 0x7FFFFFFF, l_max = there ? to : 0;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            f_min = min(f_min, __shfl_xor(f_min, d));
            f_max = max(f_max, __shfl_xor(f_max, d));
            l_min = min(l_min, __shfl_xor(l_min, d));
            l_max = max(l_max, __shfl_xor(l_max, d));
        }
        f_min = uniform(f_min);
        l_max = uniform(l_max);
        all_from = uniform(f_max) - lo;
        all_to = uniform(l_min) - lo;
        if (l_max > f_min) {
            wr0 = max(rt0, (f_min - lo) / ROWS);
            wr1 = min(nrt, (l_max - lo + ROWS - 1) / ROWS);
        }
    }

    bf16x8_t kf[DS], vf[DS];
    {
        const __bf16 *k = static_cast<const __bf16 *>(C.K) + (int64_t)kk * C.k_token + kvh * C.k_head + lh * 8;
        const __bf16 *v = static_cast<const __bf16 *>(C.V) + (int64_t)kk * C.v_token + kvh * C.v_head + lh * 8;
#pragma unroll
        for (int ks = 0; ks < DS; ++ks) {
            kf[ks] = *reinterpret_cast<const bf16x8_t *>(k + ks * 16);
            vf[ks] = *reinterpret_cast<const bf16x8_t *>(v + ks * 16);
        }
    }

    // Row loads: wave w takes rows 16 w + 4 j + (lane >> 4) of a tile, j = 0 .. 3, by four wave-loads of Q and of dout; wave 0 the 64
    // lse, wave 1 the deltas.  Rows are (token, head) pairs that advance by 64 a tile.
    const unsigned lds_base = lds_address(smem), stat_base = lds_address(stat);
    const int step_t = ROWS / G, step_g = ROWS - step_t * G;
    struct Row {
        int t, g;
    };
    auto row_at = [&](int row) __attribute__((always_inline)) {      // row of the walk, from lo on
        Row x;
        const int64_t at = (int64_t)lo + row;
        x.t = (int)(at / G);
        x.g = (int)(at - (int64_t)x.t * G);
        return x;
    };
    auto advance = [&](Row &x) __attribute__((always_inline)) {
        x.g += step_g;
        x.t += step_t;
        if (x.g >= G) {
            x.g -= G;
            x.t += 1;
        }
    };
    Row rows[4], srow = row_at(rt0 * ROWS + lane);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        rows[j] = row_at(rt0 * ROWS + wave * 16 + j * 4 + (lane >> 4));
    const __bf16 *qb = static_cast<const __bf16 *>(C.Q) + (int64_t)kvh * G * C.q_head, *gb = static_cast<const __bf16 *>(P.dout) + (int64_t)kvh * G * C.o_head;
    const float *lb = C.lse + (int64_t)kvh * G * C.lse_stride, *db = P.delta + (int64_t)kvh * G * C.lse_stride;
    auto issue = [&](int b) __attribute__((always_inline)) {         // the next tile: rows behind the walk are its last row
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool in = rows[j].t < end_b;
            const int64_t tt = in ? rows[j].t : end_b - 1, g = in ? rows[j].g : G - 1;
            const int chunk = ((lane & 15) ^ ((j * 4 + (lane >> 4)) & 15)) * 8;
            gather_load_16(qb + tt * C.q_token + g * C.q_head + chunk, lds_base + b * TILE_BYTES + wave * 4096 + j * 1024);
            gather_load_16(gb + tt * C.o_token + g * C.o_head + chunk, lds_base + (2 + b) * TILE_BYTES + wave * 4096 + j * 1024);
            advance(rows[j]);
        }
        if (wave < 2) {
            const bool in = srow.t < end_b;
            const int64_t i = (in ? srow.g : G - 1) * C.lse_stride + (in ? srow.t : end_b - 1);
            gather_load_4((wave == 0 ? lb : db) + i, stat_base + (b * 2 + wave) * ROWS * 4);
            advance(srow);
        }
    };

    const TileRead at;
    const float sl2 = C.scale * LOG2E;
    f32x16_t dk[DT], dv[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            dk[d][e] = dv[d][e] = 0.0f;

    issue(0);
    wait_vmcnt<0>();
    __syncthreads();
    for (int rt = rt0; rt < nrt; ++rt) {
        const int b = (rt - rt0) & 1;
        if (rt + 1 < nrt)
            issue(1 - b);
        if (rt >= wr0 && rt < wr1) {
            const bool border = rt * ROWS < all_from || (rt + 1) * ROWS > all_to;
#pragma unroll
            for (int j = 0; j < 2; ++j) {                            // 32 rows at a time
                const unsigned char *q_at = smem + b * TILE_BYTES + j * 32 * ROWB, *g_at = smem + (2 + b) * TILE_BYTES + j * 32 * ROWB;
                f32x16_t s, dp;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    s[e] = dp[e] = 0.0f;
#pragma unroll
                for (int ks = 0; ks < DS; ++ks) {
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.rows(q_at, ks), kf[ks], s, 0, 0, 0);
                    dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.rows(g_at, ks), vf[ks], dp, 0, 0, 0);
                }
                if (border) {
                    const unsigned row0 = (unsigned)(lo + rt * ROWS + j * 32 + 4 * lh - from), span = (unsigned)(to - from);
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (row0 + (unsigned)(8 * (e >> 2) + (e & 3)) >= span)
                            s[e] = -INFINITY;
                }
                bf16x8_t pf[2], df[2];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4_t lse = *reinterpret_cast<const f32x4_t *>(&stat[b][0][j * 32 + 8 * q + 4 * lh]);
                    const f32x4_t del = *reinterpret_cast<const f32x4_t *>(&stat[b][1][j * 32 + 8 * q + 4 * lh]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int e = 4 * q + c;
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], sl2, -lse[c] * LOG2E));
                        pf[e >> 3][e & 7] = (__bf16)p;
                        df[e >> 3][e & 7] = (__bf16)(p * (dp[e] - del[c]));
                    }
                }
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        dv[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.transposed(g_at + c * 16 * ROWB, d), pf[c], dv[d], 0, 0, 0);
                        dk[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.transposed(q_at + c * 16 * ROWB, d), df[c], dk[d], 0, 0, 0);
                    }
            }
        }
        if (rt + 1 < nrt) {
            wait_vmcnt<0>();
            __syncthreads();
        }
    }

    float x[2 * DT * 16];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            x[d * 16 + e] = dk[d][e];
            x[DT * 16 + d * 16 + e] = dv[d][e];
        }
    if (splits > 1 && !join_splits<2 * DT * 16, NT>(x, C, rest * C.kv_heads + kvh, split, splits, &arrived))
        return;
    const bool odd_k = store_row(x, C.scale, static_cast<__bf16 *>(P.dk) + (int64_t)kk * C.k_token + kvh * C.k_head, there);
    const bool odd_v = store_row(x + DT * 16, 1.0f, static_cast<__bf16 *>(P.dv) + (int64_t)kk * C.v_token + kvh * C.v_head, there);
    unsigned long long again = __builtin_amdgcn_ballot_w64(odd_k || odd_v);
    again = (again | again >> 32) & 0xFFFFFFFFull;
    if (again != 0) {
        __builtin_amdgcn_s_waitcnt(0);                               // the key's first result is written before its second
        for (; again != 0; again &= again - 1) {
            const int l = __builtin_ctzll(again);
            careful_key(P, __shfl(kk, l), kvh, __shfl(end, l));
        }
    }
}

}  // namespace

hipError_t launch_attn_prompt_grad(const GradParams &p_in, hipStream_t s, int num_cu)
{
    const Tuning tn = tuning();
    auto split = [&](CausalParams &c, int64_t groups, int tiles, size_t part) {
        c.chunk = tn.causal_chunk;
        c.max_splits = c.chunk > 0 ? (tiles + c.chunk - 1) / c.chunk : 1;
        if (c.max_splits < 2 || c.parts == nullptr || groups > c.max_counters || (size_t)groups * c.max_splits * part > c.part_bytes) {
            c.chunk = 0;
            c.max_splits = 1;
        }
    };
    GradParams p = p_in;
    const int64_t rows = (int64_t)p.c.tokens * p.c.group;
    const int waves = tn.causal_waves == 8 ? 8 : 4;
    const int64_t blocks = (rows + waves * 32 - 1) / (waves * 32);
    split(p.c, blocks * p.c.kv_heads, (p.c.tokens + BKV - 1) / BKV, (size_t)64 * 64 * waves * 4);
    const dim3 grid((unsigned)(blocks * p.c.kv_heads * p.c.max_splits));
    if (waves == 8)
        hipLaunchKernelGGL((attn_dq_kernel<8>), grid, dim3(512), 0, s, p);
    else
        hipLaunchKernelGGL((attn_dq_kernel<4>), grid, dim3(256), 0, s, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    const int64_t key_blocks = (p.c.tokens + GRAD_KEYS - 1) / GRAD_KEYS;
    split(p.c, key_blocks * p.c.kv_heads, (int)((rows + 63) / 64), (size_t)128 * 256 * 4);
    hipLaunchKernelGGL(attn_dkv_kernel, dim3((unsigned)(key_blocks * p.c.kv_heads * p.c.max_splits)), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace cf
