// Gradient of causal attention over packed prompts for gfx950: dQ, dK, dV from bf16 operands, fp32 accumulation.
//   P = exp(scale q k - lse),  delta = sum dout out,  dP = dout v,  dS = P (dP - delta)
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dout
// Two launches, each with every sum in one place (no atomics, the same bits every time): one workgroup of the first owns rows and
// walks over keys (and leaves delta for the second), one of the second owns keys and walks over the rows that see them, all
// query heads of the key head.  Both multiply the scores anew: seven products where five would do with sums spread over memory.  Walks are
// cut into splits as in the forward kernel; a third launch adds up what they parked.
// Bound: the matrix pipe, and beside it LDS: every product's "A" fragment, 1 KiB, comes from LDS for one MFMA of 32 cycles, so that four waves
// ask for all of its 128 bytes a cycle.  dK and dV hold 128 sums, 64 scores and 64 registers of K and V a lane: one wave a SIMD, which
// has to fill the pipe alone, so both kernels run as pipelines of 32-row units with one MFMA a segment.
// Measured (us, traced; dQ, dK and dV, sums): 4096 tokens, 8 heads of one key head 69 to 73, 92 to 96, 12 to 14 -- 51 and 69 GFLOP at 730 and 750
// TFLOP/s; 2048 + 1365 + 683 tokens, 4 heads of their own 26, 36, 11, of which 11 a launch are start, search, first loads and parking.
// As in the forward kernel a lane owns one row (or key) and 16 of every 32 keys (rows) of a product's result, which is, rounded to
// bf16, the "B" operand of the next product as it stands: nothing moves between lanes.  Tiles lie in LDS once and are read both by rows
// and transposed: 16-byte chunks XOR-ed with a permutation of (row & 15), which the transposing read can follow lane by lane.
// Precision: P and dS are rounded to bf16 for their products, and delta is made of the bf16 `out`.  From 64 bits dQ is 0.0026 off (2048 + 1365 + 683 tokens, 4
// heads; up to 0.0033 in packs of ten tokens a sequence, where the rounding of `out` weighs most), dK 0.0025, dV 0.0023; rounding exact
// results once gives 0.0017, with dS alone rounded before its products 0.0024.  dS as the sum of two bf16 numbers, a product more each for dQ and dK,
// gives 0.0019 and 0.0018 and takes 97 us instead of 90 with the forward call (4096 tokens, 8 heads of one key head 239 instead of 207): not worth it.
// Rows behind a walk are read as zero, and masked.  Results that are not finite are computed once more where what the mask
// hides can have been the reason, so that it has no influence.
#include "attn_tiles.h"

namespace cf {
namespace {

constexpr int LEAST_TILES = 4;           // of a split: 1 us each for dQ, 1.9 for dK and dV (2000 tokens and less: 42 to 52 us, with eight 49 to 55)
constexpr int DS = DH / 16;              // 16-wide feature slices
constexpr int DT = DH / 32;              // 32-wide feature tiles

// Wave-wide 16-byte-per-lane load from per-lane addresses straight into LDS (lane L lands at lds_addr + 16 L).
__device__ __forceinline__ void gather_load_16(const void *at, unsigned lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\t"
                 "global_load_lds_dwordx4 %1, off"
                 :
                 : "s"(lds_addr), "v"(at)
                 : "memory");
}
__device__ __forceinline__ void gather_load_4(const void *at, unsigned lds_addr)      // (... at lds_addr + 4 L)
{
    asm volatile("s_mov_b32 m0, %0\n\t"
                 "global_load_lds_dword %1, off"
                 :
                 : "s"(lds_addr), "v"(at)
                 : "memory");
}

// Tiles of rows of 256 bytes: chunk c of 16 bytes of a row lies at position c ^ spread(row & 15).  Sixteen rows' chunk c (a read by
// rows) lie on sixteen positions, and so do chunks 4 t .. 4 t + 3 of four rows (a transposing read): all 64 banks either way.  (With
// row & 15 itself the four rows of a transposing read share four positions.)
__device__ __forceinline__ int spread(int row) { return (row & 3) << 2 | (row >> 2 & 3); }

// Addresses in such a tile, in registers, so that a read costs no arithmetic: what is added to them is a constant.  `move` takes them to
// another tile (16 additions instead of one a read).
struct RowRead {                         // "A" operand: lane (row = lane & 31, half = lane >> 5), chunk 2 ks + half
    int at[DS];
    __device__ __forceinline__ RowRead()
    {
        const int lane = threadIdx.x & 63, lq = lane & 31, lh = lane >> 5;
#pragma unroll
        for (int ks = 0; ks < DS; ++ks)
            at[ks] = lq * ROWB + (((2 * ks + lh) ^ spread(lq)) << 4);
    }
    __device__ __forceinline__ void move(int bytes)
    {
#pragma unroll
        for (int ks = 0; ks < DS; ++ks) {
            at[ks] += bytes;
            asm volatile("" : "+v"(at[ks]));
        }
    }
    __device__ __forceinline__ bf16x8_t read(const unsigned char *lds, int off, int ks) const { return *reinterpret_cast<const bf16x8_t *>(lds + at[ks] + off); }
};
struct TransposedRead {                  // its transposed: rows 4 half + .. and 8 more of a slice of 16, feature tile t
    int lo[DT], hi[DT];
    __device__ __forceinline__ TransposedRead()
    {
        const int lane = threadIdx.x & 63, blk = lane >> 4, i16 = lane & 15;
        const int r = 4 * (blk >> 1) + (i16 >> 2), c = 2 * (blk & 1) + ((i16 & 3) >> 1);
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            lo[t] = r * ROWB + (((4 * t + c) ^ spread(r)) << 4) + (i16 & 1) * 8;
            hi[t] = (r + 8) * ROWB + (((4 * t + c) ^ spread(r + 8)) << 4) + (i16 & 1) * 8;
        }
    }
    __device__ __forceinline__ void move(int bytes)
    {
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            lo[t] += bytes;
            hi[t] += bytes;
            asm volatile("" : "+v"(lo[t]), "+v"(hi[t]));
        }
    }
    __device__ __forceinline__ bf16x8_t read(const unsigned char *lds, int off, int t) const
    {
        const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)(lds + lo[t] + off));
        const s16x4_t c = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)(lds + hi[t] + off));
        return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(a, c, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// The exponentials of a unit, spread over the MFMAs that run meanwhile.  A wave issues in order and has the SIMD for itself, so that between
// two MFMAs (32 cycles each) there is room for a handful of vector instructions, none of which should wait for the one before: element
// e begins in segment 4 e / 3, and its three steps -- argument, exponential, products -- lie in three segments.
template <int SEGMENT, typename F1, typename F2, typename F3>
__device__ __forceinline__ void stages(F1 &&argument, F2 &&exponential, F3 &&product)
{
    constexpr auto begins = [](int segment) { return segment >= 0 && segment <= 20 && segment % 4 != 3 ? segment - segment / 4 : -1; };
    constexpr int e3 = begins(SEGMENT - 2), e2 = begins(SEGMENT - 1), e1 = begins(SEGMENT);
    if constexpr (e3 >= 0)
        product(std::integral_constant<int, e3>{});
    if constexpr (e2 >= 0)
        exponential(std::integral_constant<int, e2>{});
    if constexpr (e1 >= 0)
        argument(std::integral_constant<int, e1>{});
}

// A split's sums, `regs` registers of every thread of the workgroup, sixteen (a feature tile) after sixteen; a launch of its own adds them up in
// split order, eight or four workgroups a block, one a feature tile.  (The last workgroup to arrive adding up all by itself: 4096 tokens, 8
// heads of one key head, up to 16 splits of 128 KiB: 575 us instead of 92 and 12 for dK and dV.)  That launch reads what was parked, 45 MiB
// there, at 4 TB/s.
template <int NT>
__device__ __forceinline__ float *part_of(const CausalParams &P, int regs, const Item &it, int split, int tile)
{
    return parked_at(P, it, split, (size_t)regs * NT) + ((size_t)tile * 16 * NT + threadIdx.x * 4);
}
template <int NT>
__device__ __forceinline__ void park(const f32x16_t &x, float *at)
{
#pragma unroll
    for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4_t *>(at + q * 4 * NT) = f32x4_t{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
}
template <int NT>
__device__ __forceinline__ f32x16_t sum_of_parts(const CausalParams &P, int regs, const Item &it, int tile)
{
    const int splits = it.splits;
    f32x16_t x = {};
    int sp = 0;
    auto add = [&](auto n_tag) __attribute__((always_inline)) {      // n splits in flight
        constexpr int N = decltype(n_tag)::value;
        f32x4_t v[N][4];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float *at = part_of<NT>(P, regs, it, sp + k, tile);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                v[k][q] = *reinterpret_cast<const f32x4_t *>(at + q * 4 * NT);
        }
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                x[e] += v[k][e >> 2][e & 3];
        sp += N;
    };
#pragma unroll 1
    while (sp + 8 <= splits)
        add(std::integral_constant<int, 8>{});
    if (sp + 4 <= splits)
        add(std::integral_constant<int, 4>{});
    if (sp + 2 <= splits)
        add(std::integral_constant<int, 2>{});
    if (sp < splits)
        add(std::integral_constant<int, 1>{});
    return x;
}

// A lane's row of a feature tile of a result X^T, times `factor`, as bf16.  True if a value is not finite.
__device__ __forceinline__ bool store_tile(const f32x16_t &x, float factor, __bf16 *row, int tile, bool there)
{
    const int lh = (threadIdx.x & 63) >> 5;
    float odd = 0.0f;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        bf16x4_t h;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float y = x[4 * g + e] * factor;
            odd = __builtin_fmaf(y, 0.0f, odd);
            h[e] = (__bf16)y;
        }
        if (there)
            *reinterpret_cast<u32x2_t *>(row + tile * 32 + 8 * g + 4 * lh) = __builtin_bit_cast(u32x2_t, h);
    }
    return there && odd != 0.0f;
}

// Rows (or keys) of the wave with a value that is not finite, in both lanes that share one.
__device__ __forceinline__ bool odd_row(bool odd)
{
    const unsigned long long rows = __builtin_amdgcn_ballot_w64(odd);
    return (rows | rows >> 32) >> (threadIdx.x & 31) & 1;
}

// One of the three results for 32 columns (rows of Q, or keys) by one wave, from memory: as in `rows_again`.  A lane's column (lane & 31) has rows
// b1, b2 and sees indices [lo, hi): keys, or with KEYS rows (token, head of the group); stored where `wanted`: all features, or (TILES = 1, a quarter of
// the registers) those of tile `tile`.
// dQ: sum over keys of dS k; dK: over rows of dS q; dV (`values`): over rows of P dout.  6144 tokens, 4 heads of one key head: 0.19 ms, with an
// infinite element of dout in their middle 1.8.
template <bool KEYS, int TILES>
__device__ __forceinline__ void grad_again(const GradParams &P, int kvh, const __bf16 *b1, const __bf16 *b2, int lo, int hi, float lse, float delta, bool values,
                                           bool wanted, __bf16 *out, int tile)
{
    const CausalParams &C = P.c;
    const int lane = threadIdx.x & 63, lq = lane & 31, lh = lane >> 5;
    const int from = least_of(wanted ? lo : 0x7FFFFFFF), to = most_of(wanted ? hi : 0);
    f32x16_t acc[TILES];
#pragma unroll
    for (int d = 0; d < TILES; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            acc[d][e] = 0.0f;
#pragma unroll 1
    for (int at0 = from & ~31; at0 < to; at0 += 32) {
        const int mine = at0 + lq < from ? from : at0 + lq < to ? at0 + lq : to - 1;
        const __bf16 *a1, *a2;
        float lse_of = 0.0f, delta_of = 0.0f;
        if constexpr (KEYS) {
            const int t = mine / C.group, head = kvh * C.group + mine - t * C.group;
            a1 = static_cast<const __bf16 *>(C.Q) + (int64_t)t * C.q_token + head * C.q_head;
            a2 = static_cast<const __bf16 *>(P.dout) + (int64_t)t * C.o_token + head * C.o_head;
            lse_of = C.lse[(int64_t)head * C.lse_stride + t];
            delta_of = P.delta[(int64_t)head * C.lse_stride + t];
        } else {
            a1 = static_cast<const __bf16 *>(C.K) + (int64_t)mine * C.k_token + kvh * C.k_head;
            a2 = static_cast<const __bf16 *>(C.V) + (int64_t)mine * C.v_token + kvh * C.v_head;
        }
        u32x2_t four[TILES == DT ? 16 : 1];                          // of the indices that a lane's sixteen slots stand for
        __bf16 one[TILES == DT ? 1 : 16];
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            const __bf16 *row = of_slot(values ? a2 : a1, 8 * (x >> 2) + (x & 3));
            if constexpr (TILES == DT)
                four[x] = reinterpret_cast<const u32x2_t *>(row)[lq];
            else
                one[x] = row[tile * 32 + lq];
        }
        __builtin_amdgcn_sched_barrier(0);
        f32x16_t s = {}, dp = {};
        asm volatile("" : "+v"(b1), "+v"(b2));                       // (read in every unit: 64 registers)
#pragma unroll
        for (int ks = 0; ks < DS; ++ks) {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(reinterpret_cast<const bf16x8_t *>(a1)[2 * ks + lh], reinterpret_cast<const bf16x8_t *>(b1)[2 * ks + lh], s, 0, 0, 0);
            dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(reinterpret_cast<const bf16x8_t *>(a2)[2 * ks + lh], reinterpret_cast<const bf16x8_t *>(b2)[2 * ks + lh], dp, 0, 0, 0);
            if (TILES == 1 || ks % 4 == 1)
                __builtin_amdgcn_sched_barrier(0);                   // (fewer registers)
        }
        __builtin_amdgcn_sched_barrier(0);
        unsigned seen = 0;
        bf16x8_t w[2];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int slot = 8 * (i >> 2) + (i & 3), at = at0 + slot + 4 * lh;
            const bool sees = at >= lo && at < hi;
            seen |= (unsigned)sees << i;
            const float l = KEYS ? __builtin_bit_cast(float, of_slot(__builtin_bit_cast(int, lse_of), slot)) : lse;
            const float d = KEYS ? __builtin_bit_cast(float, of_slot(__builtin_bit_cast(int, delta_of), slot)) : delta;
            const float p = __builtin_amdgcn_exp2f((s[i] * C.scale - l) * LOG2E);
            w[i >> 3][i & 7] = (__bf16)(sees ? values ? p : p * (dp[i] - d) : 0.0f);
            if (i % 4 == 3)
                __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
            bf16x8_t v[TILES];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if constexpr (TILES == DT) {
                    put_pair(v, i, four[2 * i], four[2 * i + 1]);
                    four[2 * i] = four[8 + 2 * i];
                    four[2 * i + 1] = four[8 + 2 * i + 1];
                } else {
                    v[0][2 * i] = one[2 * i];
                    v[0][2 * i + 1] = one[2 * i + 1];
                    one[2 * i] = one[8 + 2 * i];
                    one[2 * i + 1] = one[8 + 2 * i + 1];
                }
            add_seen(acc, v, w[0], seen);
            seen >>= 8;
            w[0] = w[1];
        }
        if ((at0 & 0xE0) == 0) {                                     // now and then: does anything that follows matter?
            bool done = true;
#pragma unroll
            for (int d = 0; d < TILES; ++d)
                done = done && none_finite(acc[d]);
            if (__builtin_amdgcn_ballot_w64(wanted && !done) == 0)
                break;
        }
    }
    if constexpr (TILES == DT) {
        if (wanted)
            store_fours(acc, values ? 1.0f : C.scale, out);
    } else {
        store_tile(acc[0], values ? 1.0f : C.scale, out, tile, wanted);
    }
}

// A workgroup's rows and walk, as in the forward kernel.
constexpr int DQ_WAVES = 4, DQ_ROWS = DQ_WAVES * 32;
struct RowBlock {
    const Sequences seqs;
    int blocks;                          // of one key head
    Item it;
    int t_base, t_last, row0, seq_a, seq_b, lo, hi, tiles;
    __device__ __forceinline__ void rows_of(const CausalParams &C, int block, int *base, int *row, int *last) const
    {
        const int64_t r0 = (int64_t)(blocks - 1 - block) * DQ_ROWS, all = (int64_t)C.tokens * C.group, r1 = r0 + DQ_ROWS < all ? r0 + DQ_ROWS : all;   // long blocks first
        *base = (int)((unsigned)r0 / (unsigned)C.group);
        *row = (int)(r0 - (int64_t)*base * C.group);
        *last = (int)((unsigned)(r1 - 1) / (unsigned)C.group);
    }
    __device__ __forceinline__ int tiles_of(const CausalParams &C, int block) const
    {
        int base, row, last, start, end;
        rows_of(C, block, &base, &row, &last);
        seqs.around(base, &start, &end);
        const int stop = seqs.end_of(C.n_seqs - 1), from = start < 0 ? 0 : start, to = last + 1 < stop ? last + 1 : stop;
        return from < to ? (to - from + BKV - 1) / BKV : 0;
    }
    __device__ __forceinline__ RowBlock(const CausalParams &C) : seqs(C.starts, C.n_seqs), blocks((int)(((int64_t)C.tokens * C.group + DQ_ROWS - 1) / DQ_ROWS)) {}
    __device__ __forceinline__ int bound(const CausalParams &C) const { return C.items > 0 ? (seqs.longest() + DQ_ROWS / C.group + 2 * BKV) / BKV : 0; }
    // the rows and the walk of it.block; false: nothing to do
    __device__ __forceinline__ bool look(const CausalParams &C)
    {
        rows_of(C, it.block, &t_base, &row0, &t_last);
        seq_a = seqs.at(t_base);
        if (seq_a == C.n_seqs)
            return false;
        seq_b = seqs.at(t_last);
        const int begin = seqs.start_of(seq_a), stop = seqs.end_of(C.n_seqs - 1);
        lo = begin < 0 ? 0 : begin;
        hi = t_last + 1 < stop ? t_last + 1 : stop;
        tiles = (hi - lo + BKV - 1) / BKV;
        return lo < hi;
    }
};
struct DqRow {                           // a lane's row: token t sees keys first .. t
    int t, head, first;
    bool there;
    __device__ __forceinline__ DqRow(const CausalParams &C, const RowBlock &B, int kvh)
    {
        const int r = B.row0 + (threadIdx.x >> 6) * 32 + (threadIdx.x & 31), rt = r / C.group;
        head = kvh * C.group + r - rt * C.group;
        there = B.t_base + rt <= B.t_last;
        t = B.t_base + (there ? rt : 0);
        int end;
        const int a = B.seqs.between(B.seq_a, B.seq_b, t, &first, &end);
        first = a < C.n_seqs ? first : t + 1;
        there = there && first <= t;
        first = there ? (first < 0 ? 0 : first) : t;                 // (a row of no sequence: any visible key will do, it is not stored)
    }
};

// Rows whose dQ is not finite once more, where keys that they do not see can have been the reason: by products with 0 (K, V not finite) or by a
// dP that is infinite.  (A row whose lse or delta is not finite has no other result.)
template <int TILES>
__device__ __forceinline__ void dq_again(const GradParams &P, const RowBlock &B, const DqRow &row, int kvh, bool odd, int tile)
{
    const CausalParams &C = P.c;
    odd = odd_row(odd);
    if (__builtin_amdgcn_ballot_w64(odd) == 0)
        return;
    __builtin_amdgcn_s_waitcnt(0);                                   // the first results, and delta, are written
    int t = row.t, head = row.head;
    asm volatile("" : "+v"(t), "+v"(head));                          // (addresses anew: kept, they would take registers from the walk)
    const __bf16 *g = static_cast<const __bf16 *>(P.dout) + (int64_t)t * C.o_token + head * C.o_head;
    const float lse = C.lse[(int64_t)head * C.lse_stride + t], delta = P.delta[(int64_t)head * C.lse_stride + t];
    odd = odd && __builtin_isfinite(lse) && __builtin_isfinite(delta);
    Keys<PACKED> K, V;
    K.base = reinterpret_cast<const unsigned char *>(static_cast<const __bf16 *>(C.K) + kvh * C.k_head);
    K.row_bytes = C.k_token * 2;
    V.base = reinterpret_cast<const unsigned char *>(static_cast<const __bf16 *>(C.V) + kvh * C.v_head);
    V.row_bytes = C.v_token * 2;
    int f_min = 0, f_max = 0, l_min = 0, l_max = 0;
    edges(row.there, row.first, row.t, &f_min, &f_max, &l_min, &l_max);
    const int front = B.lo + max(0, (f_min - B.lo) / BKV) * BKV, behind = min(B.hi, B.lo + ((l_max - B.lo) / BKV + 1) * BKV);
    const int seen_by_all = min(f_max, B.hi), unseen = max(l_min + 1, B.lo);   // front .. seen_by_all, unseen .. behind: keys that some rows do not see
    if (__builtin_amdgcn_ballot_w64(odd) == 0 || (__builtin_amdgcn_ballot_w64(odd && large_row(g)) == 0 && !any_large(K, front, seen_by_all) &&
                                                  !any_large(V, front, seen_by_all) && !any_large(K, unseen, behind) && !any_large(V, unseen, behind)))
        return;
    grad_again<false, TILES>(P, kvh, static_cast<const __bf16 *>(C.Q) + (int64_t)t * C.q_token + head * C.q_head, g, row.first, t + 1, lse, delta, false, odd,
                      static_cast<__bf16 *>(P.dq) + (int64_t)t * C.q_token + head * C.q_head, tile);
}

__global__ __launch_bounds__(64 * DQ_WAVES, 2) void attn_dq_kernel(GradParams P)
{
    const CausalParams &C = P.c;
    constexpr int NW = DQ_WAVES, NT = 64 * NW;
    constexpr int UNIT_BYTES = TILE_BYTES;                           // 32 rows of K, then of V
    __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * UNIT_BYTES];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lh = lane >> 5;

    RowBlock block(C);
    if (!my_item<NT, true>(C, block.blocks, LEAST_TILES, 1, block.bound(C), [&](int i) { return block.tiles_of(C, i); }, &block.it) || !block.look(C))
        return;
    const int kvh = block.it.kvh, split = block.it.split, splits = block.it.splits;
    const int lo = block.lo, hi = block.hi;
    int kt0, nkt;
    block.it.share(block.tiles, &kt0, &nkt);
    const DqRow row(C, block, kvh);
    const int t = row.t, head = row.head, first = row.first;
    const bool there = row.there;
    int wt0 = kt0, wt1 = kt0, all_from = 0, all_to = 0;
    {
        int f_min, f_max, l_min, l_max;
        if (edges(there, first, t, &f_min, &f_max, &l_min, &l_max) && l_max >= f_min) {
            all_from = f_max - lo;
            all_to = l_min - lo;
            wt0 = max(kt0, (f_min - lo) / BKV);
            wt1 = min(nkt, (l_max - lo) / BKV + 1);
        }
    }

    // Loads of a unit, 32 keys, straight into LDS: K and V into one of four places.  Wave-load j covers rows 4 wave + 16 j + 0 .. 3; rows
    // behind the walk read as zero.
    const unsigned lds_base = lds_address(smem);
    const int ld_row = wave * 4 + (lane >> 4), k_row = (int)C.k_token * 2, v_row = (int)C.v_token * 2;
    const unsigned swizzled = ((lane & 15) ^ spread(ld_row)) << 4;
    const unsigned k_off = (unsigned)(ld_row * k_row) + swizzled, v_off = (unsigned)(ld_row * v_row) + swizzled;
    const unsigned char *kb = static_cast<const unsigned char *>(C.K) + kvh * C.k_head * 2, *vb = static_cast<const unsigned char *>(C.V) + kvh * C.v_head * 2;
    auto issue = [&](int unit) __attribute__((always_inline)) {
        const int key = lo + unit * 32, left = hi - key < 32 ? hi - key : 32;
        const unsigned rows = left > 0 ? (unsigned)left : 0u, lds = lds_base + (unit & 3) * UNIT_BYTES + wave * 1024;
        const i32x4_t k = make_rsrc(kb + (int64_t)key * k_row, rows * (unsigned)k_row), v = make_rsrc(vb + (int64_t)key * v_row, rows * (unsigned)v_row);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            direct_load_16(k, k_off + (unsigned)(j * 16 * k_row), lds + j * 4096);
            direct_load_16(v, v_off + (unsigned)(j * 16 * v_row), lds + UNIT_BYTES / 2 + j * 4096);
        }
    };
    constexpr int LOADS = 4;             // of a wave and unit
    const int u0 = 2 * kt0, u1 = 2 * nkt;
    issue(u0);
    issue(u0 + 1);
    issue(u0 + 2);

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

    RowRead row_read;
    TransposedRead col_read;
    f32x16_t acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            acc[d][e] = 0.0f;
    constexpr f32x16_t zero = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    auto products = [&](f32x16_t &s, f32x16_t &dp) __attribute__((always_inline)) {
        s = dp = zero;
#pragma unroll
        for (int ks = 0; ks < DS; ++ks) {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_read.read(smem, 0, ks), qf[ks], s, 0, 0, 0);
            dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_read.read(smem, UNIT_BYTES / 2, ks), gf[ks], dp, 0, 0, 0);
        }
    };
    // A pipeline of one unit's depth: under the exponentials of unit u the products of unit u + 1 with Q and dout (segments 0 .. 15), then
    // those of unit u with K (16 .. 23), one MFMA a segment, its fragment requested three segments ahead.  row_read is at unit u + 1,
    // col_read at unit u.
    auto unit = [&](int u, f32x16_t &s, f32x16_t &dp, f32x16_t &sn, f32x16_t &dpn) __attribute__((always_inline)) {
        constexpr int AHEAD = 3;
        if (u * 32 < all_from || (u + 1) * 32 - 1 > all_to) {        // border, uniform
            float ninf = -INFINITY;
            asm volatile("" : "+v"(ninf));
            const unsigned key0 = (unsigned)(lo + u * 32 + 4 * lh - first), span = (unsigned)(t - first);
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (key0 + (unsigned)(8 * (e >> 2) + (e & 3)) > span)
                    s[e] = ninf;
        }
        bf16x8_t frag[AHEAD + 1], df[2];
        auto fetch = [&](auto s_tag) __attribute__((always_inline)) {
            constexpr int i = decltype(s_tag)::value;
            if constexpr (i < 16)
                frag[i % (AHEAD + 1)] = row_read.read(smem, (i & 1) * (UNIT_BYTES / 2), i >> 1);
            else if constexpr (i < 24)
                frag[i % (AHEAD + 1)] = col_read.read(smem, ((i - 16) >> 2) * 16 * ROWB, (i - 16) & 3);
        };
        auto argument = [&](auto e_tag) __attribute__((always_inline)) {
            constexpr int e = decltype(e_tag)::value;
            s[e] = __builtin_fmaf(s[e], sl2, -lse2);
        };
        auto exponential = [&](auto e_tag) __attribute__((always_inline)) {
            constexpr int e = decltype(e_tag)::value;
            s[e] = __builtin_amdgcn_exp2f(s[e]);
            dp[e] -= delta;
        };
        auto product = [&](auto e_tag) __attribute__((always_inline)) {
            constexpr int e = decltype(e_tag)::value;
            dp[e] *= s[e];
            if constexpr (e & 1) {                                   // rounded in pairs
                df[e >> 3][(e & 7) - 1] = (__bf16)dp[e - 1];
                df[e >> 3][e & 7] = (__bf16)dp[e];
            }
        };
        auto segment = [&](auto s_tag) __attribute__((always_inline)) {
            constexpr int i = decltype(s_tag)::value;
            fetch(std::integral_constant<int, i + AHEAD>{});
            if constexpr (i < 16) {
                if constexpr (i & 1)
                    dpn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i % (AHEAD + 1)], gf[i >> 1], i < 2 ? zero : dpn, 0, 0, 0);
                else
                    sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i % (AHEAD + 1)], qf[i >> 1], i < 2 ? zero : sn, 0, 0, 0);
            } else {
                constexpr int c = (i - 16) >> 2, d = (i - 16) & 3;
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i % (AHEAD + 1)], df[c], acc[d], 0, 0, 0);
            }
            if constexpr (i < 16) {                                  // element i in three segments; what is left in front of the second half of dQ
                argument(std::integral_constant<int, i>{});
                if constexpr (i >= 1)
                    exponential(std::integral_constant<int, i - 1>{});
                if constexpr (i >= 2)
                    product(std::integral_constant<int, i - 2>{});
            } else if constexpr (i == 16) {
                exponential(std::integral_constant<int, 15>{});
                product(std::integral_constant<int, 14>{});
            } else if constexpr (i == 17) {
                product(std::integral_constant<int, 15>{});
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        each<0, 1>(fetch, std::make_integer_sequence<int, AHEAD>{});
        __builtin_amdgcn_sched_barrier(0);
        each<0, 1>(segment, std::make_integer_sequence<int, 24>{});
    };

    wait_vmcnt<LOADS>();
    __syncthreads();
    int u = u0;
    auto to_next = [&](int at) { return (at & 3) == 3 ? -3 * UNIT_BYTES : UNIT_BYTES; };
    auto turn = [&]() __attribute__((always_inline)) {               // unit u + 2 has landed, and every wave is done with unit u
        wait_vmcnt<LOADS>();
        __syncthreads();
        ++u;
    };
    if (wt0 < wt1) {
        while (u < 2 * wt0) {                                        // units of other waves only
            issue(u + 3);
            turn();
        }
        f32x16_t sa, da, sb, db;
        row_read.move((u & 3) * UNIT_BYTES);
        col_read.move((u & 3) * UNIT_BYTES);
        products(sa, da);
        row_read.move(to_next(u));
        while (u < 2 * wt1) {                                        // (behind the last unit the products of one more, unused)
            issue(u + 3);
            unit(u, sa, da, sb, db);
            col_read.move(to_next(u));
            row_read.move(to_next(u + 1));
            turn();
            issue(u + 3);
            unit(u, sb, db, sa, da);
            col_read.move(to_next(u));
            row_read.move(to_next(u + 1));
            turn();
        }
    }
    while (u < u1) {
        issue(u + 3);
        turn();
    }
    wait_vmcnt<0>();                                                 // (nothing lands behind the kernel's end)

    if (splits > 1) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
            park<NT>(acc[d], part_of<NT>(C, DT * 16, block.it, split, d));
        return;
    }
    __bf16 *out = static_cast<__bf16 *>(P.dq) + (int64_t)t * C.q_token + head * C.q_head;
    bool odd = false;
#pragma unroll
    for (int d = 0; d < DT; ++d)
        odd = store_tile(acc[d], C.scale, out, d, there) || odd;
    dq_again<DT>(P, block, row, kvh, odd, 0);
}

// Workgroup `at` of the sums over the splits of dQ: one feature tile of one block.
__device__ __forceinline__ void join_dq(const GradParams &P, int at, int *looked_at)
{
    const CausalParams &C = P.c;
    const int tile = at % DT, group = at / DT, kvh = group % C.kv_heads;
    RowBlock block(C);
    block.it.kvh = kvh;
    block.it.block = group / C.kv_heads;
    Splits<256, true>(C, block.blocks, LEAST_TILES, 1, block.bound(C), [&](int i) { return block.tiles_of(C, i); }, looked_at).of_block(block.it.block, &block.it);
    if (block.it.splits < 2 || !block.look(C))
        return;
    const DqRow row(C, block, kvh);
    const f32x16_t x = sum_of_parts<64 * DQ_WAVES>(C, DT * 16, block.it, tile);
    const bool odd = store_tile(x, C.scale, static_cast<__bf16 *>(P.dq) + (int64_t)row.t * C.q_token + row.head * C.q_head, tile, row.there);
    dq_again<1>(P, block, row, kvh, odd, tile);
}

constexpr int GRAD_KEYS = 128;           // keys of a workgroup of the second launch: four waves of 32
constexpr int GRAD_ROWS = 64;            // rows per tile
// Its keys [begin, k1), and the walk over rows [lo, hi) = (token, head of the group), tokens [begin, end_b)
struct KeyBlock {
    const Sequences seqs;
    int blocks;                          // of one key head
    Item it;
    int k0, k1, begin, seq_a, seq_b, end_b, lo, hi, tiles;
    __device__ __forceinline__ int stop(const CausalParams &C) const
    {
        const int last = seqs.end_of(C.n_seqs - 1);
        return last < C.tokens ? last : C.tokens;
    }
    __device__ __forceinline__ int tiles_of(const CausalParams &C, int block) const
    {
        const int a = block * GRAD_KEYS, s = seqs.start_of(0), b = a + GRAD_KEYS < stop(C) ? a + GRAD_KEYS : stop(C), from = s > a ? s : a;
        int start, end;
        seqs.around(b - 1, &start, &end);
        end = end < C.tokens ? end : C.tokens;
        return from < b && end > from ? (int)(((int64_t)(end - from) * C.group + GRAD_ROWS - 1) / GRAD_ROWS) : 0;
    }
    __device__ __forceinline__ KeyBlock(const CausalParams &C) : seqs(C.starts, C.n_seqs), blocks((C.tokens + GRAD_KEYS - 1) / GRAD_KEYS) {}
    __device__ __forceinline__ int bound(const CausalParams &C) const
    {
        return C.items > 0 ? (int)min((int64_t)0x7FFFFFFF, ((int64_t)(seqs.longest() + GRAD_KEYS + 1) * C.group + GRAD_ROWS) / GRAD_ROWS) : 0;
    }
    // the keys and the walk of it.block; false: nothing to do
    __device__ __forceinline__ bool look(const CausalParams &C)
    {
        k0 = it.block * GRAD_KEYS;           // (the first keys are seen by most rows)
        k1 = k0 + GRAD_KEYS < stop(C) ? k0 + GRAD_KEYS : stop(C);
        begin = seqs.start_of(0) > k0 ? seqs.start_of(0) : k0;
        if (begin >= k1)
            return false;
        seq_a = seqs.at(begin);
        seq_b = seqs.at(k1 - 1);
        if (seq_b >= C.n_seqs)
            return false;
        end_b = seqs.end_of(seq_b) < C.tokens ? seqs.end_of(seq_b) : C.tokens;
        if (end_b <= begin)
            return false;
        lo = begin * C.group;
        hi = end_b * C.group;
        tiles = (int)(((int64_t)hi - lo + GRAD_ROWS - 1) / GRAD_ROWS);
        return true;
    }
};
struct GradKey {                         // a lane's key, seen by tokens key .. end - 1 of its sequence
    int key, end;
    bool there;
    __device__ __forceinline__ GradKey(const CausalParams &C, const KeyBlock &B)
    {
        const int k = B.k0 + (threadIdx.x >> 6) * 32 + (threadIdx.x & 31);
        there = k >= B.begin && k < B.k1;
        key = there ? k : B.begin;
        int start;
        const int a = B.seqs.between(B.seq_a, B.seq_b, key, &start, &end);
        end = a < C.n_seqs ? end : 0;
        end = end < B.end_b ? end : B.end_b;
        there = there && end > key;
    }
};

// Keys whose dK or dV is not finite once more, where rows that do not see them can have been the reason: by products with 0 (Q, dout not finite), an
// infinite dP, or an lse or delta that is not finite.
template <int TILES>
__device__ __forceinline__ void dkv_again(const GradParams &P, const KeyBlock &B, const GradKey &mine, int kvh, bool odd_k, bool odd_v, int tile)
{
    const CausalParams &C = P.c;
    odd_k = odd_row(odd_k);
    odd_v = odd_row(odd_v);
    if (__builtin_amdgcn_ballot_w64(odd_k || odd_v) == 0)
        return;
    __builtin_amdgcn_s_waitcnt(0);                                   // the first results are written
    const int G = C.group, lo = B.lo, hi = B.hi, first = mine.key * G, end = mine.there ? mine.end * G : first;
    const __bf16 *k = static_cast<const __bf16 *>(C.K) + (int64_t)mine.key * C.k_token + kvh * C.k_head;
    const __bf16 *v = static_cast<const __bf16 *>(C.V) + (int64_t)mine.key * C.v_token + kvh * C.v_head;
    auto any_odd = [&](int from, int to) {                           // of the rows [from, to)
        for (; from < to; from += 64) {
            const int r = from + (int)(threadIdx.x & 63);
            bool odd = false;
            if (r < to) {
                const int t = r / G, head = kvh * G + r - t * G;
                odd = large_row(static_cast<const __bf16 *>(C.Q) + (int64_t)t * C.q_token + head * C.q_head) ||
                      large_row(static_cast<const __bf16 *>(P.dout) + (int64_t)t * C.o_token + head * C.o_head) ||
                      !__builtin_isfinite(C.lse[(int64_t)head * C.lse_stride + t]) || !(fabsf(P.delta[(int64_t)head * C.lse_stride + t]) < 0x1p100f);
            }
            if (__builtin_amdgcn_ballot_w64(odd) != 0)
                return true;
        }
        return false;
    };
    int f_min = 0, f_max = 0, l_min = 0, l_max = 0;
    edges(mine.there, first, end, &f_min, &f_max, &l_min, &l_max);
    const int front = lo + max(0, (f_min - lo) / GRAD_ROWS) * GRAD_ROWS, tiles = (l_max - lo + GRAD_ROWS - 1) / GRAD_ROWS;
    const int behind = tiles < B.tiles ? lo + tiles * GRAD_ROWS : hi;
    if (__builtin_amdgcn_ballot_w64((odd_k || odd_v) && large_row(v)) == 0 && !any_odd(front, min(f_max, hi)) && !any_odd(max(l_min, lo), behind))
        return;
#pragma unroll 1
    for (int values = 0; values < 2; ++values) {                     // dK, dV
        const bool odd = values ? odd_v : odd_k;
        if (__builtin_amdgcn_ballot_w64(odd) != 0)
            grad_again<true, TILES>(P, kvh, k, v, first, end, 0.0f, 0.0f, values, odd, values ? static_cast<__bf16 *>(P.dv) + (int64_t)mine.key * C.v_token + kvh * C.v_head
                                                                                       : static_cast<__bf16 *>(P.dk) + (int64_t)mine.key * C.k_token + kvh * C.k_head, tile);
    }
}

// What stands for rows behind a walk: a probability of 0 times anything else of them would be NaN where that is not finite.
__device__ const __attribute__((aligned(16))) char zero_row[ROWB] = {};

__global__ __launch_bounds__(256, 1) void attn_dkv_kernel(GradParams P)
{
    const CausalParams &C = P.c;
    constexpr int NT = 256, ROWS = GRAD_ROWS;
    constexpr int NB = 4;                                            // tiles in LDS: two that are multiplied, two that land
    __shared__ __attribute__((aligned(1024))) unsigned char smem[NB * 2 * TILE_BYTES];   // Q, dout
    __shared__ __attribute__((aligned(16))) float stat[NB][2][ROWS]; // lse, delta

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lh = lane >> 5;
    const int G = C.group;

    KeyBlock block(C);
    if (!my_item<NT, false>(C, block.blocks, LEAST_TILES, 1, block.bound(C), [&](int i) { return block.tiles_of(C, i); }, &block.it) || !block.look(C))
        return;
    const int kvh = block.it.kvh, split = block.it.split, splits = block.it.splits;
    const int lo = block.lo, hi = block.hi;
    int rt0, nrt;
    block.it.share(block.tiles, &rt0, &nrt);
    const GradKey mine(C, block);
    const int kk = mine.key, end = mine.end;
    const bool there = mine.there;
    const int from = kk * G, to = there ? end * G : from;            // the rows that see it
    int wr0 = rt0, wr1 = rt0, all_from = 0, all_to = 0;
    {
        int f_min, f_max, l_min, l_max;
        if (edges(there, from, to, &f_min, &f_max, &l_min, &l_max) && l_max > f_min) {
            all_from = f_max - lo;
            all_to = l_min - lo;
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
    // lse, wave 1 the deltas (and waves 2 and 3 the same once more, so that every wave has nine loads in flight).  Rows are (token, head) pairs that advance by 64 a tile: by step_t tokens and step_g
    // heads, and where those run over by a token more and a group of heads less.
    const unsigned lds_base = lds_address(smem), stat_base = lds_address(stat) + (wave & 1) * ROWS * 4;
    const int step_t = ROWS / G, step_g = ROWS - step_t * G;
    const int64_t q_step = 2 * (step_t * C.q_token + step_g * C.q_head), q_wrap = q_step + 2 * (C.q_token - G * C.q_head);
    const int64_t o_step = 2 * (step_t * C.o_token + step_g * C.o_head), o_wrap = o_step + 2 * (C.o_token - G * C.o_head);
    const int64_t l_step = 4 * (step_t + step_g * C.lse_stride), l_wrap = l_step + 4 * (1 - G * C.lse_stride);
    const char *qb = static_cast<const char *>(C.Q) + 2 * (int64_t)kvh * G * C.q_head, *gb = static_cast<const char *>(P.dout) + 2 * (int64_t)kvh * G * C.o_head;
    const char *lb = reinterpret_cast<const char *>(((wave & 1) == 0 ? C.lse : P.delta) + (int64_t)kvh * G * C.lse_stride);
    const int row_in = wave * 16 + (lane >> 4);                      // row inside a tile: row_in + 4 j; of the statistics: lane
    const char *q_at[4], *g_at[4], *l_at;
    int g_of[4], g_of_l;
#pragma unroll
    for (int j = 0; j < 5; ++j) {
        const unsigned row = (unsigned)(lo + rt0 * ROWS + (j < 4 ? row_in + 4 * j : lane));
        const int64_t t = row / (unsigned)G;
        const int g = (int)(row - (unsigned)t * G);
        if (j < 4) {
            const int chunk = ((lane & 15) ^ spread(j * 4 + (lane >> 4))) * 16;
            q_at[j] = qb + 2 * (t * C.q_token + g * C.q_head) + chunk;
            g_at[j] = gb + 2 * (t * C.o_token + g * C.o_head) + chunk;
            g_of[j] = g;
        } else {
            l_at = lb + 4 * (t + g * C.lse_stride);
            g_of_l = g;
        }
    }
    int rows_left = hi - lo - rt0 * ROWS;                            // of the walk, from the next tile to load on
    constexpr int LOADS = 9;                                         // of a wave and tile
    auto issue = [&](int b) __attribute__((always_inline)) {         // the next tile
        const char *q[4], *g[4], *l = l_at;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            q[j] = q_at[j];
            g[j] = g_at[j];
        }
        if (rows_left < ROWS) {                                      // uniform: rows behind the walk
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (row_in + 4 * j >= rows_left)
                    q[j] = g[j] = zero_row + (lane & 15) * 16;
            if (lane >= rows_left)
                l = zero_row;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            gather_load_16(q[j], lds_base + 2 * b * TILE_BYTES + wave * 4096 + j * 1024);
            gather_load_16(g[j], lds_base + (2 * b + 1) * TILE_BYTES + wave * 4096 + j * 1024);
        }
        gather_load_4(l, stat_base + b * 2 * ROWS * 4);
    };
    // ... and to the one after it, in five pieces (four rows, the statistics) that find their place among the MFMAs
    auto advance = [&](auto j_tag) __attribute__((always_inline)) {
        constexpr int j = decltype(j_tag)::value;
        int &g = j < 4 ? g_of[j & 3] : g_of_l;
        g += step_g;
        const bool over = g >= G;
        g -= over ? G : 0;
        if constexpr (j < 4) {
            q_at[j] += over ? q_wrap : q_step;
            g_at[j] += over ? o_wrap : o_step;
            asm volatile("" : "+v"(q_at[j]), "+v"(g_at[j]), "+v"(g));
        } else {
            l_at += over ? l_wrap : l_step;
            asm volatile("" : "+v"(l_at), "+v"(g));
            rows_left -= ROWS;
        }
    };
    auto advance_all = [&]() __attribute__((always_inline)) { each<0, 1>(advance, std::make_integer_sequence<int, 5>{}); };

    RowRead row_read;
    TransposedRead col_read;
    const float sl2 = C.scale * LOG2E;
    f32x16_t dk[DT], dv[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            dk[d][e] = dv[d][e] = 0.0f;

    // A pipeline of one unit's depth, a unit being 32 rows: under the exponentials of unit u the products of unit u + 1 with K and V
    // (segments 0 .. 15), and under the rest of them those of unit u with dout and Q (16 .. 31), one MFMA a segment, its fragment
    // requested three segments ahead.
    f32x4_t lse[4], del[4];                                          // of the unit's rows; -lse in units of log2(e)
    auto stats = [&](int b, int j) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            lse[q] = *reinterpret_cast<const f32x4_t *>(&stat[b][0][j * 32 + 8 * q + 4 * lh]);
            del[q] = *reinterpret_cast<const f32x4_t *>(&stat[b][1][j * 32 + 8 * q + 4 * lh]);
        }
    };
    auto products = [&](f32x16_t &s, f32x16_t &dp) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            s[e] = dp[e] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < DS; ++ks) {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_read.read(smem, 0, ks), kf[ks], s, 0, 0, 0);
            dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_read.read(smem, TILE_BYTES, ks), vf[ks], dp, 0, 0, 0);
        }
    };
    // unit (rt, J) from s, dp; the next, (bn, 1 - J), into sn, dpn.  row_read is at the next unit's tile, col_read at this one's.
    auto unit = [&](int rt, int bn, f32x16_t &s, f32x16_t &dp, f32x16_t &sn, f32x16_t &dpn, auto j_tag) __attribute__((always_inline)) {
        constexpr int J = decltype(j_tag)::value;
        constexpr int AHEAD = 6, RING = 8;
        constexpr int NOW = J * 32 * ROWB, THEN = (1 - J) * 32 * ROWB;
        if (rt * ROWS < all_from || (rt + 1) * ROWS > all_to) {      // border tiles, uniform
            float ninf = -INFINITY;
            asm volatile("" : "+v"(ninf));
            const unsigned row0 = (unsigned)(lo + rt * ROWS + J * 32 + 4 * lh - from), span = (unsigned)(to - from);
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (row0 + (unsigned)(8 * (e >> 2) + (e & 3)) >= span)
                    s[e] = ninf;
        }
        bf16x8_t frag[RING], pf[2], df[2];
        auto fetch = [&](auto s_tag) __attribute__((always_inline)) {
            constexpr int i = decltype(s_tag)::value;
            if constexpr (i < 16)
                frag[i % RING] = row_read.read(smem, THEN + (i & 1) * TILE_BYTES, i >> 1);
            else if constexpr (i < 32)
                frag[i % RING] = col_read.read(smem, NOW + (1 - (i & 1)) * TILE_BYTES + ((i - 16) >> 3) * 16 * ROWB, ((i - 16) >> 1) & 3);
        };
        float x[16];                                                 // arguments, then probabilities
        auto argument = [&](auto e_tag) __attribute__((always_inline)) {
            constexpr int e = decltype(e_tag)::value;
            x[e] = __builtin_fmaf(s[e], sl2, lse[e >> 2][e & 3]);
        };
        auto exponential = [&](auto e_tag) __attribute__((always_inline)) {
            constexpr int e = decltype(e_tag)::value;
            x[e] = __builtin_amdgcn_exp2f(x[e]);
            dp[e] -= del[e >> 2][e & 3];
        };
        auto product = [&](auto e_tag) __attribute__((always_inline)) {
            constexpr int e = decltype(e_tag)::value;
            dp[e] *= x[e];
            if constexpr (e & 1) {                                   // rounded in pairs
                pf[e >> 3][(e & 7) - 1] = (__bf16)x[e - 1];
                pf[e >> 3][e & 7] = (__bf16)x[e];
                df[e >> 3][(e & 7) - 1] = (__bf16)dp[e - 1];
                df[e >> 3][e & 7] = (__bf16)dp[e];
            }
        };
        constexpr f32x16_t zero = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        auto segment = [&](auto s_tag) __attribute__((always_inline)) {
            constexpr int i = decltype(s_tag)::value;
            fetch(std::integral_constant<int, i + AHEAD>{});
            if constexpr (i < 16) {
                if constexpr (i & 1)
                    dpn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i % RING], vf[i >> 1], i < 2 ? zero : dpn, 0, 0, 0);
                else
                    sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i % RING], kf[i >> 1], i < 2 ? zero : sn, 0, 0, 0);
            } else {
                constexpr int c = (i - 16) >> 3, d = ((i - 16) >> 1) & 3;
                if constexpr (i & 1)
                    dk[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i % RING], df[c], dk[d], 0, 0, 0);
                else
                    dv[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i % RING], pf[c], dv[d], 0, 0, 0);
            }
            stages<i>(argument, exponential, product);
            if constexpr (i == 24)
                stats(bn, 1 - J);
            if constexpr (i >= 28) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    lse[i - 28][c] *= -LOG2E;
                asm volatile("" : "+v"(lse[i - 28]));                // (here, not where it is used)
            }
            if constexpr (J == 0 && i >= 23 && i < 28)
                advance(std::integral_constant<int, i - 23>{});
            __builtin_amdgcn_sched_barrier(0);
        };
        each<0, 1>(fetch, std::make_integer_sequence<int, AHEAD>{});
        __builtin_amdgcn_sched_barrier(0);
        each<0, 1>(segment, std::make_integer_sequence<int, 32>{});
    };

    // (behind the walk's last tile rows are asked for once more, which nothing reads: the number of loads in flight stays the same)
    issue(0);
    advance_all();
    issue(1);
    advance_all();
    issue(2);
    advance_all();
    wait_vmcnt<LOADS>();
    __syncthreads();
    f32x16_t sa, da, sb, db2;
    int b = 0, rt = rt0;
    auto next_of = [](int i) { return (i + 1) & (NB - 1); };
    auto to_next = [&]() { return b == NB - 1 ? -2 * (NB - 1) * TILE_BYTES : 2 * TILE_BYTES; };
    // Tiles rt and rt + 1 have landed, rt + 2 is on its way, rt + 3 goes over tile rt - 1, which every wave is done with.
    auto load_ahead = [&]() __attribute__((always_inline)) { issue((b + 3) & (NB - 1)); };
    auto turn = [&]() __attribute__((always_inline)) {
        wait_vmcnt<LOADS>();
        __syncthreads();
        b = next_of(b);
        ++rt;
    };
    using first = std::integral_constant<int, 0>;
    using second = std::integral_constant<int, 1>;
    if (wr0 < wr1) {
        while (rt < wr0) {                                           // tiles of other waves only
            load_ahead();
            advance_all();
            turn();
        }
        row_read.move(2 * b * TILE_BYTES);
        col_read.move(2 * b * TILE_BYTES);
        products(sa, da);
        stats(b, 0);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                lse[q][c] *= -LOG2E;
        while (rt < wr1) {                                           // (behind the last tile the products of one more, unused: half the code)
            load_ahead();
            unit(rt, b, sa, da, sb, db2, first{});
            row_read.move(to_next());
            unit(rt, next_of(b), sb, db2, sa, da, second{});
            col_read.move(to_next());
            turn();
        }
    }
    while (rt < nrt) {
        load_ahead();
        advance_all();
        turn();
    }

    wait_vmcnt<0>();                                                 // (nothing lands behind the kernel's end)
    if (splits > 1) {
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            park<NT>(dk[d], part_of<NT>(C, 2 * DT * 16, block.it, split, d));
            park<NT>(dv[d], part_of<NT>(C, 2 * DT * 16, block.it, split, DT + d));
        }
        return;
    }
    __bf16 *out_k = static_cast<__bf16 *>(P.dk) + (int64_t)kk * C.k_token + kvh * C.k_head;
    __bf16 *out_v = static_cast<__bf16 *>(P.dv) + (int64_t)kk * C.v_token + kvh * C.v_head;
    bool odd_k = false, odd_v = false;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
        odd_k = store_tile(dk[d], C.scale, out_k, d, there) || odd_k;
        odd_v = store_tile(dv[d], 1.0f, out_v, d, there) || odd_v;
    }
    dkv_again<DT>(P, block, mine, kvh, odd_k, odd_v, 0);
}

// ... of dK and dV
__device__ __forceinline__ void join_dkv(const GradParams &P, int at, int *looked_at)
{
    const CausalParams &C = P.c;
    const int tile = at % (2 * DT), group = at / (2 * DT), kvh = group % C.kv_heads;
    KeyBlock block(C);
    block.it.kvh = kvh;
    block.it.block = group / C.kv_heads;
    Splits<256, false>(C, block.blocks, LEAST_TILES, 1, block.bound(C), [&](int i) { return block.tiles_of(C, i); }, looked_at).of_block(block.it.block, &block.it);
    if (block.it.splits < 2 || !block.look(C))
        return;
    const GradKey mine(C, block);
    const f32x16_t x = sum_of_parts<256>(C, 2 * DT * 16, block.it, tile);
    __bf16 *out = tile < DT ? static_cast<__bf16 *>(P.dk) + (int64_t)mine.key * C.k_token + kvh * C.k_head
                            : static_cast<__bf16 *>(P.dv) + (int64_t)mine.key * C.v_token + kvh * C.v_head;
    const bool odd = store_tile(x, tile < DT ? C.scale : 1.0f, out, tile & (DT - 1), mine.there);
    dkv_again<1>(P, block, mine, kvh, odd && tile < DT, odd && tile >= DT, tile & (DT - 1));
}

// Workgroups below `dkv_wgs`: dK and dV; the others dQ.  (Two launches, 6.3 and 10.1 us for a pack of 4096 tokens and four heads.)
static_assert(DQ_WAVES == 4, "one shape of workgroup for both");
__global__ __launch_bounds__(256, 4) void attn_grad_join_kernel(GradParams dkv, GradParams dq, int dkv_wgs)
{
    __shared__ int looked_at[MAX_BLOCKS];
    if ((int)blockIdx.x < dkv_wgs)
        join_dkv(dkv, blockIdx.x, looked_at);
    else
        join_dq(dq, (int)blockIdx.x - dkv_wgs, looked_at);
}

struct GradLaunches {
    CausalParams dq, dkv;
    int64_t row_blocks, key_blocks;      // of one key head
    int64_t dq_wgs, dkv_wgs;
    size_t bytes;                        // parked: a half of the workspace each
};
GradLaunches plan_grad(const CausalParams &c, int num_cu)
{
    GradLaunches g;
    g.dq = g.dkv = c;
    const size_t half = c.part_bytes / 2 & ~(size_t)255;
    g.dq.part_bytes = g.dkv.part_bytes = half;
    g.dkv.parts = c.parts == nullptr ? nullptr : c.parts + half / sizeof(float);
    const int64_t rows = (int64_t)c.tokens * c.group;
    g.row_blocks = (rows + DQ_ROWS - 1) / DQ_ROWS;
    g.key_blocks = (c.tokens + GRAD_KEYS - 1) / GRAD_KEYS;
    const size_t dq_part = (size_t)64 * 64 * DQ_WAVES * 4, dkv_part = (size_t)128 * 256 * 4;
    g.dq_wgs = plan_items(g.dq, g.row_blocks, (c.tokens + BKV - 1) / BKV, LEAST_TILES, dq_part, false, num_cu);
    g.dkv_wgs = plan_items(g.dkv, g.key_blocks, (rows + GRAD_ROWS - 1) / GRAD_ROWS, LEAST_TILES, dkv_part, false, num_cu);
    const size_t a = (size_t)g.dq.items * dq_part, b = (size_t)g.dkv.items * dkv_part;
    g.bytes = 2 * (((a > b ? a : b) + 255) & ~(size_t)255);
    return g;
}

}  // namespace

hipError_t launch_attn_prompt_grad(const GradParams &p, hipStream_t s, int num_cu)
{
    const GradLaunches g = plan_grad(p.c, num_cu);
    const int64_t most = (int64_t)1 << 24;                           // workgroups, of 256 threads
    const int64_t join_dq = g.dq.items > 0 ? g.row_blocks * p.c.kv_heads * DT : 0, join_dkv = g.dkv.items > 0 ? g.key_blocks * p.c.kv_heads * 2 * DT : 0;
    if (g.dq_wgs >= most || g.dkv_wgs >= most || join_dq + join_dkv >= most)
        return hipErrorInvalidValue;
    GradParams dq = p, dkv = p;
    dq.c = g.dq;
    dkv.c = g.dkv;
    hipLaunchKernelGGL(attn_dq_kernel, dim3((unsigned)g.dq_wgs), dim3(64 * DQ_WAVES), 0, s, dq);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(attn_dkv_kernel, dim3((unsigned)g.dkv_wgs), dim3(256), 0, s, dkv);
    e = hipGetLastError();
    if (e != hipSuccess || join_dq + join_dkv == 0)
        return e;
    hipLaunchKernelGGL(attn_grad_join_kernel, dim3((unsigned)(join_dkv + join_dq)), dim3(256), 0, s, dkv, dq, (int)join_dkv);
    return hipGetLastError();
}

size_t attn_grad_part_bytes(const CausalParams &p_in, int num_cu)
{
    CausalParams p = p_in;                                           // as if any workspace were there
    p.parts = reinterpret_cast<float *>(256);
    p.part_bytes = (size_t)1 << 48;
    p.max_counters = 1 << 30;
    return plan_grad(p, num_cu).bytes;
}

}  // namespace cf
