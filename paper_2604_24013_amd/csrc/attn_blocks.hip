// Causal attention of many rows for gfx950: packed prompts over their own keys, chunks of new tokens over a paged cache.
// bf16 MFMAs, fp32 online softmax.
//
// Rows.  A row is one token of one query head; the query heads that share a key head are neighbours (row = token * group +
// head in group), so that a workgroup's rows read the same key tiles and span few tokens -- under the causal mask few keys that
// only some of them see.  One workgroup = NW waves of 32 rows each; it walks over the keys in tiles of 64.
// Per tile and wave (as in the kernels of one query slice):
//   S^T = K Q^T      the key tile as the MFMA "A" operand, the wave's rows (in registers) as "B": a lane owns ONE row (lane & 31)
//                    and 16 of every 32 keys, so a row's statistics and its mask (keys first .. last) live in two lanes;
//   online softmax   P = exp2(S - m), m kept until a probability would exceed 2^8;
//   O^T += V^T P^T   P, rounded to bf16, is in the layout of an MFMA "B" operand when the 16 contraction slots are taken to mean
//                    the keys that the lane holds; V^T comes from the [key x feature] tile by the transposing LDS read.
// Mask.  A wave multiplies only the tiles from its rows' first key to their last; for the others of the workgroup's walk it moves its
// share of the loads.  Tiles on the border are masked by a select on the scores, so that what a row does not see has no weight --
// but zero times an infinite or NaN V is NaN: rows whose result is not finite are computed once more where hidden values can have
// been the reason (`rows_again`).
// Packed prompts: a workgroup takes consecutive rows whatever sequences they belong to; keys of the walk that belong to another
// sequence are masked like any others.
// Bound: the matrix pipe where rows fill the chip (8192 tokens, 32 heads of 4 key heads: 489 to 505 us with lse, 478 to 493 without, 1090 to 1120 and
// 1120 to 1150 TFLOP/s, where a library product of 8192 reaches 1232); else that a workgroup takes 10 us beside its tiles of 0.9 to 1.3 us each: 1 until
// kernel arguments and starts are there, 1.3 for the search of its piece, 1.5 to 2.5 for Q and the first tiles, 1.7 to park, and 4.5 for the
// last to arrive to merge.  4096 tokens, 4 heads: 33.6 us (511 TFLOP/s); 5 packed prompts of 8192 tokens, 8 heads of one key head: 73.4 us
// (712); 2381 new tokens over 13528 in e4m3, 8 heads of one key head: 76.6 us (668).
// With a window (a gap in the walk, tiles masked on both borders): 5 packed prompts of 16384 tokens, 8 heads of one key head, window 4096: 171 us (980);
// 2381 new tokens over 38528 in e4m3, window 4096 + 4: 70.3 us (492).
#include "attn_tiles.h"

namespace cf {
namespace {

// Tiles of a split at the least: about as long as a workgroup's start takes (1024 tokens, 8 heads of one key head 17.8 us; eight tiles 19.0, four
// 18.6).
constexpr int LEAST_TILES = 6;

constexpr int PARKED = DH / 32 * 16 + 4; // floats that a thread parks: its part of O, and m and l

template <int NW, int SRC, bool LSE, bool WIN>
__global__ __launch_bounds__(64 * NW, 2) void attn_blocks_kernel(CausalParams P)
{
    constexpr int NT = 64 * NW;          // threads per workgroup
    constexpr int BQ = NW * 32;          // rows per workgroup
    constexpr int KT = BKV / 32;         // 32-key MFMA tiles per key tile
    constexpr int DS = DH / 16;          // 16-wide feature slices (contraction of S^T)
    constexpr int DT = DH / 32;          // 32-wide feature tiles (rows of O^T)
    constexpr int LOADS = TILE_BYTES / 1024 / NW;   // wave-loads per wave of a bf16 K or V tile: four rows each
    constexpr int LOADS8 = LOADS / 2;               // of an e4m3 tile: eight rows each
    constexpr int V_BASE = 2 * TILE_BYTES;          // LDS: two K tiles, two V tiles

    __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * 2 * TILE_BYTES];

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lq = lane & 31, lh = lane >> 5;
    const int G = P.group;

    const int blocks = (int)(((SRC == PACKED ? (int64_t)P.tokens : (int64_t)P.max_q) * G + BQ - 1) / BQ);    // (paged: of one sequence)
    const Sequences seqs(P.starts, P.n_seqs);
    // A block's rows (tokens t_base .. t_last from row row0 of the first on) and walk over keys [lo, hi)
    struct Walk {
        int t_base, t_last, row0, lo, hi, shown;     // shown: keys that token t_base sees, less one (paged)
        const int32_t *table;
        bool any;
    };
    auto walk_of = [&](int block) {                  // of the lane's block; packed: but for lo
        Walk w;
        w.any = false;
        w.lo = w.shown = 0;
        w.table = nullptr;
        if constexpr (SRC == PACKED) {
            const int64_t r0 = (int64_t)(blocks - 1 - block) * BQ, all = (int64_t)P.tokens * G, r1 = r0 + BQ < all ? r0 + BQ : all;   // long blocks first
            w.t_base = (int)((unsigned)r0 / (unsigned)G);
            w.row0 = (int)(r0 - (int64_t)w.t_base * G);
            w.t_last = (int)((unsigned)(r1 - 1) / (unsigned)G);
            const int stop = seqs.end_of(P.n_seqs - 1);
            w.hi = w.t_last + 1 < stop ? w.t_last + 1 : stop;
            w.any = true;
        } else {
            const int seq = block % P.n_seqs, nth = blocks - 1 - block / P.n_seqs;
            const int q0 = P.starts[seq], q1 = P.starts[seq + 1];
            const int from = clamped(q0, P.tokens), m = clamped(q1, P.tokens) - from;
            int n = P.kv_len[seq];
            n = n < 0 ? 0 : n < P.max_kv ? n : P.max_kv;
            const int rows = m < P.max_q ? m : P.max_q;              // rows behind max_q are left as they were
            const int64_t r0 = (int64_t)nth * BQ, all = (int64_t)rows * G, r1 = r0 + BQ < all ? r0 + BQ : all;
            w.any = r0 < all;
            const int b0 = (int)((unsigned)r0 / (unsigned)G);
            w.row0 = (int)(r0 - (int64_t)b0 * G);
            const int last = w.any ? (int)((unsigned)(r1 - 1) / (unsigned)G) : 0;
            w.t_base = from + b0;
            w.t_last = from + last;
            w.shown = n - m + b0;
            w.hi = n - m + last + 1 > 0 ? n - m + last + 1 : 0;
            w.table = P.table + (int64_t)seq * P.max_pages;
        }
        return w;
    };
    // the gap of a walk whose first row's last key is `last`
    auto gap_of = [&](int lo, int hi, int last) { return WIN ? Gap<BKV>(P.sinks, lo, hi, window_from(P, lo, last)) : Gap<BKV>(); };
    Item it;
    const int all_blocks = SRC == PACKED ? blocks : blocks * P.n_seqs;
    int bound = SRC == PACKED && P.items > 0 && P.n_seqs <= 64 ? (seqs.longest() + BQ / G + 2 * BKV) / BKV : 0x7FFFFFFF;
    if constexpr (WIN)
        bound = (int)min((int64_t)bound, ((int64_t)P.window + P.sinks + BQ / G + 4 * BKV) / BKV);
    if (!my_item<NT, NW == 4>(P, all_blocks, LEAST_TILES, 1, bound, WIN && SRC != PACKED ? P.whole_from : 0, [&](int block) {
            Walk w = walk_of(block);
            if constexpr (SRC == PACKED) {
                int end;
                seqs.around(w.t_base, &w.lo, &end);
                w.lo = w.lo < 0 ? 0 : w.lo;
                if constexpr (WIN)
                    return w.lo < w.hi ? gap_of(w.lo, w.hi, w.t_base).tiles(w.lo, w.hi) : 0;
                return w.lo < w.hi ? (w.hi - w.lo + BKV - 1) / BKV : 0;
            } else {
                if constexpr (WIN)
                    return w.any ? max(1, gap_of(0, w.hi, w.shown).tiles(0, w.hi)) : 0;
                return w.any ? max(1, (w.hi + BKV - 1) / BKV) : 0;
            }
        }, &it))
        return;
    const int kvh = it.kvh, split = it.split, splits = it.splits;
    const Walk walk = walk_of(it.block);
    const int t_base = uniform(walk.t_base), t_last = uniform(walk.t_last), row0 = uniform(walk.row0), hi = uniform(walk.hi), shown = uniform(walk.shown);
    const int count = t_last - t_base + 1;
    const int32_t *table = uniform(walk.table);
    int lo = 0, seq_a = 0, seq_b = 0;
    if constexpr (SRC == PACKED) {
        seq_a = seqs.at(t_base);
        if (seq_a == P.n_seqs)
            return;                                  // behind the last sequence
        seq_b = seqs.at(t_last);
        lo = seqs.start_of(seq_a);
        lo = lo < 0 ? 0 : lo;
        if (lo >= hi)
            return;
    } else if (__builtin_amdgcn_readfirstlane(walk.any) == 0) {
        return;
    }

    // This workgroup's key tiles: [kt0, nkt) of the block's
    const Gap<BKV> gap = gap_of(lo, hi, SRC == PACKED ? t_base : shown);
    auto place_of = [&](int kt) __attribute__((always_inline)) { return WIN ? gap.key(kt) : kt * BKV; };   // a tile's first key, from lo on
    const int tiles = WIN ? gap.tiles(lo, hi) : (hi - lo + BKV - 1) / BKV;
    int kt0, nkt;
    it.share(tiles, &kt0, &nkt);

    // The lane's row
    const int r = row0 + wave * 32 + lq;
    const int token = r / G, g = r - token * G;      // token: from t_base on
    const int head = kvh * G + g;
    bool there = token < count;
    int first = 0, last;
    if constexpr (SRC == PACKED) {
        const int t = t_base + (there ? token : 0);
        int end;
        const int a = seqs.between(seq_a, seq_b, t, &first, &end);
        first = a < P.n_seqs ? first : t + 1;
        there = there && first <= t;
        first = there ? (first < 0 ? 0 : first) : t; // (a row of no sequence: any visible key will do, it is not stored)
        last = t;
    } else {
        last = shown + (there ? token : 0);
    }
    // ... and its wave's: tiles [wt0, wt1) have keys that a row of it sees; all see tiles that start at `all_from` or later and end at
    // `all_to` or earlier
    using Sees = std::conditional_t<WIN, SeesWindow, SeesUpTo>;
    const Sees sees = [&]() {
        if constexpr (WIN)
            return SeesWindow(P, first, last);
        else
            return SeesUpTo{first, last};
    }();
    int wt0 = kt0, wt1 = kt0, all_from = 0, all_to = 0;
    {
        int f_min, f_max, l_min, l_max;
        if constexpr (WIN) {
            int low, unused;                         // (rows that see first keys see those of their sequence, so that the lowest grows with the row)
            if (edges(there, sees.from, last, &f_min, &f_max, &l_min, &l_max) && l_max >= f_min) {
                edges(there, P.sinks > 0 ? first : sees.from, last, &low, &unused, &unused, &unused);
                all_from = f_max - lo;
                all_to = l_min - lo;
                wt0 = max(kt0, gap.tile(low - lo));
                wt0 -= (wt0 - kt0) & 1;
                wt1 = min(nkt, gap.tile(l_max - lo) + 1);
            }
        } else if (edges(there, first, last, &f_min, &f_max, &l_min, &l_max) && l_max >= f_min) {
            all_from = f_max - lo;
            all_to = l_min - lo;
            wt0 = max(kt0, (f_min - lo) / BKV);
            wt0 -= (wt0 - kt0) & 1;                  // (buffers and registers alternate together)
            wt1 = min(nkt, (l_max - lo) / BKV + 1);
        }
    }
    const bool busy = wt0 < wt1;
    const unsigned long long rows_there = __builtin_amdgcn_ballot_w64(there);

    const __bf16 *qrow = static_cast<const __bf16 *>(P.Q) + (int64_t)(t_base + (there ? token : 0)) * P.q_token + head * P.q_head;
    bf16x8_t qf[DS];
#pragma unroll
    for (int ks = 0; ks < DS; ++ks)
        qf[ks] = *reinterpret_cast<const bf16x8_t *>(qrow + ks * 16 + lh * 8);

    constexpr int E = SRC == PAGED_E4M3 ? 1 : 2;
    const int k_row = (int)(SRC == PACKED ? P.k_token : P.pool.token_stride) * E, v_row = (int)(SRC == PACKED ? P.v_token : P.pool.token_stride) * E;   // bytes
    const unsigned char *kb = static_cast<const unsigned char *>(SRC == PACKED ? P.K : P.pool.k) + kvh * (SRC == PACKED ? P.k_head : P.pool.head_stride) * E;
    const unsigned char *vb = static_cast<const unsigned char *>(SRC == PACKED ? P.V : P.pool.v) + kvh * (SRC == PACKED ? P.v_head : P.pool.head_stride) * E;
    const int shift = P.pool.page_shift, n_pages = (int)P.pool.n_pages;
    const int64_t page_bytes = P.pool.page_stride * E, exp_page = (int64_t)P.pool.kv_heads << shift;
    const uint8_t *ke = P.pool.k_exp + ((int64_t)kvh << shift), *ve = P.pool.v_exp + ((int64_t)kvh << shift);       // (e4m3)
    const unsigned lds_base = lds_address(smem);

    // Paged: the page table by windows of 64 entries, one a lane; `bad`: which of a window's pages do not exist.  The walk asks for V of
    // tile kt + 1, then for K of tile kt + 2, so that windows change upwards only, and a tile that is masked lies in the present
    // window or in the one before.
    int window = -1, entry = 0;
    unsigned long long bad = 0, bad_before = 0;
    auto window_of = [&](int kt) __attribute__((always_inline)) { return (place_of(kt) >> shift) >> 6; };
    auto page_of = [&](int key) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(entry, (key >> shift) & 63); };
    auto turn_to = [&](int kt) __attribute__((always_inline)) {
        const int w = window_of(kt);
        if (w != window) {
            const int i = w * 64 + lane;
            entry = i < P.max_pages ? table[i] : -1;
            bad_before = WIN || w == window + 1 ? bad : 0;           // (a gap may leave windows out)
            bad = __builtin_amdgcn_ballot_w64((unsigned)entry >= (unsigned)n_pages);
            window = w;
        }
    };

    // Loads of key tile `kt` into a K or V buffer.  bf16: wave-load j covers 4 rows of 256 bytes, straight into LDS.
    // K: the lane at LDS chunk position cp of row r fetches global chunk cp ^ (r & 15); V: the 64-byte groups of a row are XOR-ed
    // with (row & 3).  (The rows of a wave-load lie a multiple of sixteen from those of the wave's first.)  Rows behind the walk,
    // and those of pages that do not exist, read as zero and move no data.
    static_assert(NW * 4 % 16 == 0, "key rows of a wave-load");
    const int ld_row = wave * 4 + (lane >> 4), ld_cp = lane & 15;
    const unsigned k_off = (unsigned)((SRC == PACKED ? ld_row : lane >> 4) * k_row + ((ld_cp ^ (ld_row & 15)) << 4));
    const unsigned v_off = (unsigned)((SRC == PACKED ? ld_row : lane >> 4) * v_row + (((ld_cp >> 2) ^ (ld_row & 3)) << 6) + ((ld_cp & 3) << 4));
    auto issue = [&](int kt, const unsigned char *from, int row_bytes, unsigned off, unsigned lds) __attribute__((always_inline)) {
        if constexpr (SRC == PACKED) {                               // one buffer a tile
            const int key = lo + place_of(kt), left = hi - key < BKV ? hi - key : BKV;
            const i32x4_t rsrc = make_rsrc(from + (int64_t)key * row_bytes, left > 0 ? (unsigned)left * (unsigned)row_bytes : 0u);
#pragma unroll
            for (int j = 0; j < LOADS; ++j)
                direct_load_16(rsrc, off + (unsigned)(j * NW * 4) * (unsigned)row_bytes, lds + wave * 1024 + j * NW * 1024);
        } else {                                                     // one a wave-load, whose rows lie in one page
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const int key = place_of(kt) + wave * 4 + j * NW * 4, page = page_of(key);
                const int left = hi - key < 4 ? hi - key : 4;
                const bool some = left > 0 && (unsigned)page < (unsigned)n_pages;
                const unsigned char *at = from + (int64_t)page * page_bytes + (key & ((1 << shift) - 1)) * row_bytes;
                direct_load_16(make_rsrc(at, some ? (unsigned)(left * row_bytes) : 0u), off, lds + wave * 1024 + j * NW * 1024);
            }
        }
    };
    // e4m3: a lane fetches 16 codes of a row (eight lanes a row, eight rows a wave-load) and the row's exponent into registers, and
    // writes the bf16 values that they stand for where the direct loads would have put them.
    const int ld_row8 = wave * 8 + (lane >> 3), ld_c8 = lane & 7;
    u32x4_t code_k[LOADS8], code_v[LOADS8];
    int exp_k[LOADS8], exp_v[LOADS8];
    auto issue8 = [&](int kt, const unsigned char *from, const uint8_t *exponents, int row_bytes, u32x4_t (&code)[LOADS8], int (&ex)[LOADS8]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < LOADS8; ++j) {
            const int key = place_of(kt) + wave * 8 + j * NW * 8;
            const int left = hi - key < 8 ? hi - key : 8, page = page_of(key), in_page = key & ((1 << shift) - 1);
            const bool some = left > 0 && (unsigned)page < (unsigned)n_pages;
            const auto rows = plain_rsrc(from + (int64_t)page * page_bytes + in_page * row_bytes, some ? left * row_bytes : 0);
            const auto exps = plain_rsrc(exponents + page * exp_page + in_page, some ? left : 0);
            code[j] = __builtin_amdgcn_raw_buffer_load_b128(rows, (lane >> 3) * row_bytes + ld_c8 * 16, 0, 0);
            ex[j] = __builtin_amdgcn_raw_buffer_load_b8(exps, lane >> 3, 0, 0);
        }
    };
    auto put8 = [&](const u32x4_t (&code)[LOADS8], const int (&ex)[LOADS8], int base, bool is_v) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < LOADS8; ++j) {
            const float scale = __builtin_bit_cast(float, (unsigned)ex[j] << 23);
            u32x4_t out[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                out[i >> 1][2 * (i & 1)] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[j][i], scale, false));
                out[i >> 1][2 * (i & 1) + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[j][i], scale, true));
            }
            const int row = ld_row8 + j * NW * 8;
            unsigned char *to = smem + base + row * ROWB;
            const int at = is_v ? (((ld_c8 >> 1) ^ (row & 3)) << 6) + ((ld_c8 & 1) << 5) : ((2 * ld_c8) ^ (row & 15)) << 4;
            *reinterpret_cast<u32x4_t *>(to + at) = out[0];
            *reinterpret_cast<u32x4_t *>(to + (at ^ 16)) = out[1];
        }
    };

    // Fragment addresses inside a buffer.
    // K as "A" operand: lane (key = lq, lh) reads chunk (2 ks + lh) of its key row, swizzled.
    // V^T as "A" operand: transposing reads; the two reads of a slice start at key rows 4 lh + (i16 >> 2) and 8 more.
    int k_addr[DS];
#pragma unroll
    for (int ks = 0; ks < DS; ++ks)
        k_addr[ks] = lq * ROWB + (((2 * ks + lh) ^ (lq & 15)) << 4);
    const int blk = lane >> 4, i16 = lane & 15;
    const int v_kl = 4 * (blk >> 1) + (i16 >> 2);
    const int v_nl = (blk & 1) * 16 + (i16 & 3) * 4;
    int v_addr[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
        v_addr[t] = V_BASE + v_kl * ROWB + (((t) ^ (v_kl & 3)) << 6) + v_nl * 2;

    f32x16_t oacc[DT];
    float m_run = -3.402823466e38f;      // (finite: against -inf a tile whose scores are all -inf would give NaN)
    // Row sums of this lane's keys, and of a pair of tiles: of the rounded probabilities, which multiply V, so that the roundings of a row's
    // dominant key cancel; LSE: of the probabilities before rounding (rounded, the log-sum-exp of a row with one dominant key would be
    // off by up to 2^-9), and the output is divided by that.  Both sums would bring the output of a call with lse from 0.00212 to 0.00207 from 64
    // bits (scores of sigma 4: 0.00208 to 0.00183; rounded once, 0.0016), and cost 3 % of a full chip's time (504 to 520 us), 7 % of small launches'
    // (32.9 to 35.1 us, 74.2 to 79.5), as much as the sum over the rounded ones alone saves: a dot product of two, half the instructions.
    float l_run = 0.0f, l_pair = 0.0f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            oacc[d][e] = 0.0f;
    const float sl2 = P.scale * LOG2E;   // scores are kept in units of log2(e)

    auto scores = [&](int buf, f32x16_t (&sn)[KT]) __attribute__((always_inline)) {
        const unsigned char *st = smem + buf * TILE_BYTES;
#pragma unroll
        for (int j = 0; j < KT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                sn[j][e] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < DS; ++ks)
#pragma unroll
            for (int j = 0; j < KT; ++j) {
                const bf16x8_t kf = *reinterpret_cast<const bf16x8_t *>(st + k_addr[ks] + j * 32 * ROWB);
                sn[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks], sn[j], 0, 0, 0);
            }
    };
    auto maximum = [&](const f32x16_t (&sn)[KT]) __attribute__((always_inline)) {
        float mx = sn[0][0];
#pragma unroll
        for (int j = 0; j < KT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                mx = fmaxf(mx, sn[j][e]);
        return mx;
    };
    // Before a tile's scores are exponentiated: keys that a row does not see are masked (border tiles only), and the running reference
    // m is raised where the tile's maximum exceeds it by more than 2^RAISE (probabilities stay below 2^RAISE), so that the rescaling
    // of the accumulators is rare and sits in a wave-uniform branch.
    constexpr float RAISE = 8.0f;
    auto settle = [&](int kt, f32x16_t (&sn)[KT], float mx) __attribute__((always_inline)) {
        if (place_of(kt) < all_from || place_of(kt) + BKV - 1 > all_to) {    // uniform
            float ninf = -INFINITY;
            asm volatile("" : "+v"(ninf));                           // (keeps this a branch: not 32 selects in every tile)
            const int key0 = lo + place_of(kt) + 4 * lh;
            if constexpr (WIN) {
#pragma unroll
                for (int j = 0; j < KT; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (!sees(key0 + j * 32 + 8 * (e >> 2) + (e & 3)))
                            sn[j][e] = ninf;
            } else if constexpr (SRC == PACKED) {
                const unsigned at = (unsigned)(key0 - first), span = (unsigned)(last - first);
#pragma unroll
                for (int j = 0; j < KT; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (at + (unsigned)(j * 32 + 8 * (e >> 2) + (e & 3)) > span)
                            sn[j][e] = ninf;
            } else {
#pragma unroll
                for (int j = 0; j < KT; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (key0 + j * 32 + 8 * (e >> 2) + (e & 3) > last)
                            sn[j][e] = ninf;
            }
            mx = maximum(sn);
        }
        if constexpr (SRC != PACKED) {
            const unsigned long long none = window_of(kt) == window ? bad : bad_before;
            if (none != 0) {                                         // uniform
                const int key0 = place_of(kt) + 4 * lh;
#pragma unroll
                for (int j = 0; j < KT; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (none >> (((key0 + j * 32 + 8 * (e >> 2) + (e & 3)) >> shift) & 63) & 1)
                            sn[j][e] = -INFINITY;
                mx = maximum(sn);
            }
        }
        const float mxs = max_of_halves(mx) * sl2;                   // scale > 0: the maximum of the scaled scores
        if (__builtin_amdgcn_ballot_w64(mxs > m_run + RAISE) != 0) { // (not where all scores so far are -inf)
            const float m_new = fmaxf(m_run, mxs);
            float alpha = exp2f(m_run - m_new);                      // 0 on the first tile with a finite score
            asm volatile("" : "+v"(alpha));                          // (keeps this a branch, as above)
            m_run = m_new;
            l_run *= alpha;
            l_pair *= alpha;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    oacc[d][e] *= alpha;
        }
    };
    auto load_next = [&](int kt, int b) __attribute__((always_inline)) {   // into what the last barrier released
        if constexpr (SRC != PACKED)
            turn_to(kt + 1);
        if constexpr (SRC == PAGED_E4M3)
            issue8(kt + 1, vb, ve, v_row, code_v, exp_v);
        else
            issue(kt + 1, vb, v_row, v_off, lds_base + V_BASE + (1 - b) * TILE_BYTES);
        if constexpr (SRC != PACKED)
            turn_to(kt + 2);
        if constexpr (SRC == PAGED_E4M3)
            issue8(kt + 2, kb, ke, k_row, code_k, exp_k);
        else
            issue(kt + 2, kb, k_row, k_off, lds_base + b * TILE_BYTES);
    };
    auto put_v = [&](int b) __attribute__((always_inline)) { put8(code_v, exp_v, V_BASE + (1 - b) * TILE_BYTES, true); };
    auto put_k = [&](int b) __attribute__((always_inline)) { put8(code_k, exp_k, b * TILE_BYTES, false); };
    auto finish = [&](int b, bool put) __attribute__((always_inline)) {   // V of tile kt+1 and K of tile kt+2 have landed
        if constexpr (SRC == PAGED_E4M3) {
            if (put) {
                put_v(b);
                put_k(b);
            }
        } else {
            wait_vmcnt<0>();
        }
        __syncthreads();                                             // ... for every wave, and V of kt, K of kt+1 are read by all
    };
    // One tile: probabilities P = exp2(S - m) rounded to bf16, their row sums, O^T += V^T P^T; and under it, with NEXT, the scores of tile
    // kt + 1 and their maximum.  Thirty-two segments of one MFMA each -- sixteen of the scores, sixteen of V's
    // product --, the fragment of the third segment ahead requested in each, the 32 exponentials spread over segments 0 .. 22 and the
    // maximum over the last eight.
    bf16x2_t ones;
    ones[0] = ones[1] = (__bf16)1.0f;
    auto tile = [&](int kt, f32x16_t (&sc)[KT], f32x16_t (&sn)[KT], auto b_tag, auto next_tag) __attribute__((always_inline)) {
        constexpr int B = decltype(b_tag)::value;
        constexpr bool NEXT = decltype(next_tag)::value;
        constexpr int FIRST = NEXT ? 0 : 16;                         // first segment
        constexpr int AHEAD = 3;
        bf16x8_t frag[AHEAD + 1], pf[KT * 2];                        // pf: "B" fragments of the 16-key slices
        auto fetch = [&](auto s_tag) __attribute__((always_inline)) {
            constexpr int s = decltype(s_tag)::value;
            if constexpr (s < 16) {
                frag[s % (AHEAD + 1)] = *reinterpret_cast<const bf16x8_t *>(smem + k_addr[s >> 1] + (1 - B) * TILE_BYTES + (s & 1) * 32 * ROWB);
            } else if constexpr (s < 32) {
                const unsigned char *pv = smem + v_addr[s & 3] + B * TILE_BYTES + ((s - 16) >> 2) * 16 * ROWB;
                const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)(pv));
                const s16x4_t c = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)(pv + 8 * ROWB));
                frag[s % (AHEAD + 1)] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(a, c, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        };
        const float nm = -m_run;
        auto exponentials = [&](auto e_tag) __attribute__((always_inline)) {   // of elements e and e+1
            constexpr int e = decltype(e_tag)::value;
            bf16x2_t two;
#pragma unroll
            for (int i = 0; i < 2; ++i) {                            // bare v_exp_f32: arguments below -126 give 0
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e >> 4][(e & 15) + i], sl2, nm));
                if constexpr (LSE)
                    l_pair = (e == 0 && i == 0 && B == 0 ? 0.0f : l_pair) + p;
                two[i] = (__bf16)p;
            }
            pf[e >> 3][(e & 7)] = two[0];
            pf[e >> 3][(e & 7) + 1] = two[1];
            if constexpr (!LSE)
                l_pair = __builtin_amdgcn_fdot2_f32_bf16(two, ones, e == 0 && B == 0 ? 0.0f : l_pair, false);
            if constexpr (e == 30 && (B == 1 || !NEXT))
                l_run += l_pair;
        };
        float mx = -INFINITY;
        auto segment = [&](auto s_tag) __attribute__((always_inline)) {
            constexpr int s = decltype(s_tag)::value;
            fetch(std::integral_constant<int, s + AHEAD>{});
            if constexpr (s < 16) {
                if constexpr (s < 2)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        sn[s & 1][e] = 0.0f;
                sn[s & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[s % (AHEAD + 1)], qf[s >> 1], sn[s & 1], 0, 0, 0);
                if constexpr (s % 4 != 3)
                    exponentials(std::integral_constant<int, 2 * (s - s / 4)>{});
            } else {
                oacc[s & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[s % (AHEAD + 1)], pf[(s - 16) >> 2], oacc[s & 3], 0, 0, 0);
                if constexpr (NEXT && s < 24 && s % 2 == 0)
                    exponentials(std::integral_constant<int, 24 + (s - 16)>{});
                if constexpr (NEXT && s >= 24) {
                    constexpr int e0 = 4 * ((s - 24) & 3);
#pragma unroll
                    for (int e = e0; e < e0 + 4; ++e)
                        mx = fmaxf(mx, sn[(s - 24) >> 2][e]);
                    asm volatile("" : "+v"(mx));                     // (here, not where it is used)
                }
            }
            // (nobody reads these buffers any more; behind the last segment the conversions cost chunks of 2381 tokens 1.5 of 72 us)
            if constexpr (SRC == PAGED_E4M3 && NEXT && s == 27)
                put_v(B);
            if constexpr (SRC == PAGED_E4M3 && NEXT && s == 30)
                put_k(B);
            __builtin_amdgcn_sched_barrier(0);
        };
        const bool more = NEXT || kt + 1 < nkt;
        if (more)
            load_next(kt, B);
        fetch(std::integral_constant<int, FIRST>{});
        fetch(std::integral_constant<int, FIRST + 1>{});
        fetch(std::integral_constant<int, FIRST + 2>{});
        if constexpr (!NEXT)
            each<0, 2>(exponentials, std::make_integer_sequence<int, 16>{});
        __builtin_amdgcn_sched_barrier(0);
        each<FIRST, 1>(segment, std::make_integer_sequence<int, 32 - FIRST>{});
        if constexpr (NEXT)
            settle(kt + 1, sn, mx);
        if (more)
            finish(B, !NEXT);
    };

    if (nkt > kt0) {
        if constexpr (SRC != PACKED)
            turn_to(kt0);
        if constexpr (SRC == PAGED_E4M3) {
            issue8(kt0, kb, ke, k_row, code_k, exp_k);
            issue8(kt0, vb, ve, v_row, code_v, exp_v);
            put8(code_k, exp_k, 0, false);
        } else {
            issue(kt0, kb, k_row, k_off, lds_base);
            issue(kt0, vb, v_row, v_off, lds_base + V_BASE);
        }
        if constexpr (SRC != PACKED)
            turn_to(kt0 + 1);
        if constexpr (SRC == PAGED_E4M3) {
            issue8(kt0 + 1, kb, ke, k_row, code_k, exp_k);
            put8(code_v, exp_v, V_BASE, true);
            put8(code_k, exp_k, TILE_BYTES, false);
        } else {
            issue(kt0 + 1, kb, k_row, k_off, lds_base + TILE_BYTES);
            wait_vmcnt<0>();
        }
        __syncthreads();
        f32x16_t sa[KT], sb[KT];
        int kt = kt0;
        if (busy && wt0 == kt0) {
            scores(0, sa);
            settle(kt0, sa, maximum(sa));
        }
        __syncthreads();                                             // K of tile kt0 is read by all
        if (busy) {
            for (; kt < wt0; ++kt) {                                 // tiles of other waves only
                load_next(kt, (kt - kt0) & 1);
                if (kt + 1 == wt0) {
                    scores(0, sa);
                    settle(wt0, sa, maximum(sa));
                }
                finish((kt - kt0) & 1, true);
            }
            using buf0 = std::integral_constant<int, 0>;
            using buf1 = std::integral_constant<int, 1>;
            for (; kt + 2 < wt1; kt += 2) {
                tile(kt, sa, sb, buf0{}, std::true_type{});
                tile(kt + 1, sb, sa, buf1{}, std::true_type{});
            }
            if (kt + 2 == wt1) {
                tile(kt, sa, sb, buf0{}, std::true_type{});
                tile(kt + 1, sb, sa, buf1{}, std::false_type{});
                kt += 2;
            } else {
                tile(kt, sa, sb, buf0{}, std::false_type{});
                ++kt;
            }
        }
        for (; kt + 1 < nkt; ++kt) {
            load_next(kt, (kt - kt0) & 1);
            finish((kt - kt0) & 1, true);
        }
    }
    l_run = sum_of_halves(l_run);                                    // the whole row sums, in both lanes of the row

    // Key split: park (m, l, O) in the workspace, thread-major, sixteen bytes a lane; the workgroup that arrives last merges all
    // splits in split order, its own from its registers.  Device-coherent cache policy on exactly these accesses, relaxed agent-scope
    // atomics on the counter.
    if (splits > 1) {
        constexpr int COHERENT = 1 | 16;
        const size_t part = (size_t)PARKED * NT;
        const int group = it.block * P.kv_heads + kvh;
        auto part_rsrc = [&](int sp) {
            return __builtin_amdgcn_make_buffer_rsrc(parked_at(P, it, sp, part), 0, (int)(part * 4), 0x00020000);
        };
        {
            __amdgpu_buffer_rsrc_t rs = part_rsrc(split);
            auto park = [&](f32x4_t x, int i) __attribute__((always_inline)) {
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, x), rs, (i * NT + tid) * 16, 0, COHERENT);
            };
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    park(f32x4_t{oacc[d][e], oacc[d][e + 1], oacc[d][e + 2], oacc[d][e + 3]}, d * 4 + e / 4);
            park(f32x4_t{m_run, l_run, 0.0f, 0.0f}, DT * 4);
        }
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        unsigned *arrived = reinterpret_cast<unsigned *>(smem);       // the key tiles are no longer read
        if (tid == 0)
            *arrived = __hip_atomic_fetch_add(&P.counters[group], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (*arrived != (unsigned)(splits - 1))
            return;
        if (tid == 0)
            __hip_atomic_store(&P.counters[group], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        f32x16_t sum[DT];
        float m_all = -3.402823466e38f, l_all = 0.0f;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                sum[d][e] = 0.0f;
#pragma unroll 1
        for (int sp = 0; sp < splits; ++sp) {
            f32x16_t v[DT];
            float m = m_run, l = l_run;
            if (sp == split) {
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    v[d] = oacc[d];
            } else {
                __amdgpu_buffer_rsrc_t rs = part_rsrc(sp);
                auto ld = [&](int i) { return __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rs, (i * NT + tid) * 16, 0, COHERENT)); };
                const f32x4_t ml = ld(DT * 4);
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const f32x4_t x = ld(d * 4 + e / 4);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            v[d][e + k] = x[k];
                    }
                m = ml[0];
                l = ml[1];
            }
            const float m_new = fmaxf(m_all, m), back = exp2f(m_all - m_new), f = exp2f(m - m_new);   // (a row that sees no key of a split: nothing times a factor)
            m_all = m_new;
            l_all = l_all * back + l * f;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    sum[d][e] = sum[d][e] * back + v[d][e] * f;
        }
        m_run = m_all;
        l_run = l_all;
#pragma unroll
        for (int d = 0; d < DT; ++d)
            oacc[d] = sum[d];
    }

    // O = O^T / l, rounded to bf16; a row without a visible key is 0 and its log-sum-exp -inf.
    int nth = lane, per_token = G;
    asm volatile("" : "+v"(nth), "+s"(per_token));                   // (found anew: kept, they would take registers from the walk)
    const bool stored = rows_there >> nth & 1;
    const int r_out = row0 + wave * 32 + (nth & 31), of_token = r_out / per_token, of_head = kvh * G + r_out - of_token * G;
    const int64_t t = t_base + of_token;
    __bf16 *orow = static_cast<__bf16 *>(P.out) + t * P.o_token + of_head * P.o_head;
    const float inv = l_run == 0.0f ? 0.0f : 1.0f / l_run;
    float odd = 0.0f;                                                // NaN if a value is not finite
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            oacc[d][e] *= inv;
            odd = __builtin_fmaf(oacc[d][e], 0.0f, odd);
        }
    if (stored) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int gq = 0; gq < 4; ++gq) {
                bf16x4_t h;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    h[e] = (__bf16)oacc[d][4 * gq + e];
                *reinterpret_cast<u32x2_t *>(orow + d * 32 + 8 * gq + 4 * lh) = __builtin_bit_cast(u32x2_t, h);
            }
        if (LSE && lh == 0)
            P.lse[(int64_t)of_head * P.lse_stride + t] = l_run == 0.0f ? -INFINITY : (m_run + __log2f(l_run)) * LN2;
    }
    const unsigned long long odd_rows = __builtin_amdgcn_ballot_w64(stored && odd != 0.0f && l_run == l_run);   // (l is made of visible scores only)
    if (odd_rows != 0) {
        const bool again = (odd_rows | odd_rows >> 32) >> lq & 1;
        Keys<SRC> K, V;
        K.base = kb;
        K.row_bytes = k_row;
        K.table = table;
        K.exps = ke;
        K.page_bytes = page_bytes;
        K.n_pages = n_pages;
        K.exp_page = exp_page;
        K.shift = shift;
        V = K;
        V.base = vb;
        V.row_bytes = v_row;
        V.exps = ve;
        // The tiles of this wave, of all splits (the first may be one that no row sees); front .. f_max, l_min .. behind: keys that some rows do not see
        int f_min = 0, f_max = 0, l_min = 0, l_max = 0;
        int sinks_end = lo;                                          // (with a window the tiles with first keys too, of which rows see some)
        if constexpr (WIN) {
            edges(stored, sees.from, last, &f_min, &f_max, &l_min, &l_max);
            sinks_end = (int)min((int64_t)hi, lo + (int64_t)gap.front * BKV);
        } else {
            edges(stored, first, last, &f_min, &f_max, &l_min, &l_max);
        }
        const int front = lo + (WIN ? gap.key(gap.front) : max(0, (f_min - lo) / BKV - 1) * BKV), behind = min(hi, lo + ((l_max - lo) / BKV + 1) * BKV);
        if (any_large(V, front, min(f_max, hi)) || any_large(V, max(l_min + 1, lo), behind) || (WIN && any_large(V, lo, sinks_end))) {
            __builtin_amdgcn_s_waitcnt(0);                           // the rows' first results are written before their second
            rows_again<SRC>(K, V, static_cast<const __bf16 *>(P.Q) + (stored ? t : t_base) * P.q_token + of_head * P.q_head, sees, again, sl2, 0, 1, oacc,
                            &m_run, &l_run);
            if (again)
                store_fours(oacc, l_run == 0.0f ? 0.0f : 1.0f / l_run, orow);
        }
    }
}

template <int NW, int SRC, bool WIN>
hipError_t launch(const CausalParams &p, int64_t wgs, hipStream_t s)
{
    if (wgs * 64 * NW >= ((int64_t)1 << 32))
        return hipErrorInvalidValue;
    if (p.lse != nullptr)
        hipLaunchKernelGGL((attn_blocks_kernel<NW, SRC, true, WIN>), dim3((unsigned)wgs), dim3(64 * NW), 0, s, p);
    else
        hipLaunchKernelGGL((attn_blocks_kernel<NW, SRC, false, WIN>), dim3((unsigned)wgs), dim3(64 * NW), 0, s, p);
    return hipGetLastError();
}

size_t part_bytes(int waves) { return (size_t)PARKED * (64 * waves) * sizeof(float); }

// Four waves (128 rows) or eight; the launch's workgroups.
int choose_blocks(CausalParams &p, bool paged, int64_t rows, int64_t sequences, int64_t tiles, int num_cu, int64_t *wgs)
{
    const Tuning tn = tuning();
    // Eight waves share a tile's loads, and its conversion from e4m3; four make twice as many blocks.  us, four / eight: 8192 tokens x 32 heads
    // 545 / 525, 4096 x 4 in pieces of 20 and 12 tiles 33.5 / 38; 2381 tokens x 8 over 5 to 8 thousand in e4m3 106 / 81.
    const bool many = (rows + 255) / 256 * p.kv_heads * sequences >= 4 * num_cu;
    const int waves = tn.causal_waves ? tn.causal_waves : many || (paged && rows >= 256) ? 8 : 4;
    const int64_t blocks = (rows + waves * 32 - 1) / (waves * 32) * sequences, resident = (int64_t)num_cu * 8 / waves;
    if (!paged) {
        *wgs = plan_alike(p, blocks, tiles, LEAST_TILES, part_bytes(waves), true, num_cu, resident);
        return waves;
    }
    // Of a paged batch's blocks, `max_q` rows for every sequence, only the tables tell which have rows, so that with a window the kernel counts them and
    // decides what `plan_alike` does.  us, whole / cut: 1024 and 8 x 1 new tokens, 8 heads of one key head, over 9000, window 4096 + 4, 40 blocks in e4m3
    // 136 / 64 (of 8192 rows that there may be, 136 / 67); 512 and 15 x 1 over 30000, window 8192, 31 blocks 257 / 72; 4 x 2048 over 9000, 256 blocks
    // 153 / 169; 6 x 1024, 192 of them, 143 / 158.
    *wgs = plan_items(p, blocks, tiles, LEAST_TILES, part_bytes(waves), true, num_cu);
    p.whole_from = p.window == 0 || tn.causal_chunk ? 0 : (int)((3 * resident + 4 * p.kv_heads - 1) / (4 * p.kv_heads));
    return waves;
}

}  // namespace

int64_t plan_items(CausalParams &p, int64_t blocks, int64_t longest, int64_t least, size_t part, bool counted, int num_cu)
{
    // Four blocks a compute unit are not split.  Forward, 8192 tokens, 8 heads on each of 4 key heads: 522 us unsplit, 603 in pieces.  Gradient:
    // 8192 tokens of 32 heads on 4 2152 and 2228, 8 x 1024 tokens of 32 on 8 359 and 378, one of 6000 among 20 of 100 1123 and 1190.  Few rows of
    // like lengths: 128 sequences of 500 tokens, 8 key heads, 45 and 51 us, 512 of 100 to 1000 205 and 245, 256 of up to 4096, 4 key heads, 198 and
    // 201.  It is the wrong way round for one long context among many short ones, which only the tables on the device tell: 65536 among 127 of 500, 8
    // key heads, 733 and 110.
    const Tuning tn = tuning();
    const int64_t all = blocks * p.kv_heads;
    p.items = p.chunk = 0;
    p.num_cu = num_cu;
    if (p.parts == nullptr || blocks > 512 || all >= 4 * num_cu || (!p.paged && p.n_seqs > 64) || (counted && all > p.max_counters) ||
        longest <= (tn.causal_chunk ? 1 : least + least / 2) || blocks * longest > INT32_MAX)    // (the tiles of all walks are added up in 32 bits)
        return all;
    const int64_t rounds = (3 * all + 2 * num_cu - 1) / (2 * num_cu), fit = (int64_t)(p.part_bytes / part);
    int64_t items = tn.causal_chunk ? all * ((longest + tn.causal_chunk - 1) / tn.causal_chunk) : (rounds > 1 ? rounds : 1) * num_cu / p.kv_heads * p.kv_heads;
    if (items > fit) {
        if (tn.causal_chunk)
            return all;
        items = fit / p.kv_heads * p.kv_heads;
    }
    if (items <= all)
        return all;
    p.items = (int)items;
    p.chunk = tn.causal_chunk;
    return items;
}

int64_t plan_alike(CausalParams &p, int64_t blocks, int64_t longest, int64_t least, size_t part, bool counted, int num_cu, int64_t resident)
{
    // (8192 tokens, 8 heads of one key head, window 1024, forward and gradient: 512 blocks of rows left whole 221 us, in pieces 228.  128 of them, window
    // 512: in pieces 83, whole 88.  256 blocks of keys, 32768 tokens, the gradient: whole 530, in pieces 626.)
    const int64_t all = blocks * p.kv_heads;
    if (p.window == 0 || tuning().causal_chunk || 4 * all < 3 * resident)
        return plan_items(p, blocks, longest, least, part, counted, num_cu);
    p.items = p.chunk = 0;
    p.num_cu = num_cu;
    return all;
}

namespace {
// Tiles of a walk at the most, of `keys` keys.
int64_t longest_walk(const CausalParams &p, int64_t keys, int64_t rows)
{
    const int64_t all = (keys + BKV - 1) / BKV;
    if (p.window == 0)
        return all;
    const int64_t some = ((int64_t)p.window + p.sinks + (rows < 256 ? rows : 256) + 3 * BKV) / BKV;
    return some < all ? some : all;
}

template <int SRC>
hipError_t launch_as(const CausalParams &p, int waves, int64_t wgs, hipStream_t s)
{
    if (p.window > 0)
        return waves == 8 ? launch<8, SRC, true>(p, wgs, s) : launch<4, SRC, true>(p, wgs, s);
    return waves == 8 ? launch<8, SRC, false>(p, wgs, s) : launch<4, SRC, false>(p, wgs, s);
}

int choose_prompt(CausalParams &p, int num_cu, int64_t *wgs)
{
    const int64_t rows = (int64_t)p.tokens * p.group;
    return choose_blocks(p, false, rows, 1, longest_walk(p, p.tokens, rows), num_cu, wgs);
}
int choose_paged(CausalParams &p, int num_cu, int64_t *wgs)
{
    const int64_t rows = (int64_t)p.max_q * p.group;
    return choose_blocks(p, true, rows, p.n_seqs, longest_walk(p, p.max_kv, rows), num_cu, wgs);
}
}  // namespace

hipError_t launch_attn_prompt(const CausalParams &p_in, hipStream_t s, int num_cu)
{
    CausalParams p = p_in;
    int64_t wgs;
    const int waves = choose_prompt(p, num_cu, &wgs);
    return launch_as<PACKED>(p, waves, wgs, s);
}

hipError_t launch_attn_paged_blocks(const CausalParams &p_in, hipStream_t s, int num_cu)
{
    CausalParams p = p_in;
    int64_t wgs;
    const int waves = choose_paged(p, num_cu, &wgs);
    return p.pool.e4m3 ? launch_as<PAGED_E4M3>(p, waves, wgs, s) : launch_as<PAGED_BF16>(p, waves, wgs, s);
}

namespace {
size_t part_bytes_of(CausalParams p, int (*choose)(CausalParams &, int, int64_t *), int num_cu)
{
    p.parts = reinterpret_cast<float *>(256);                        // as if any workspace were there
    p.part_bytes = (size_t)1 << 48;
    p.max_counters = 1 << 30;
    int64_t wgs;
    const int waves = choose(p, num_cu, &wgs);
    return p.items > 0 ? (size_t)p.items * part_bytes(waves) : 0;
}
}  // namespace

size_t attn_paged_blocks_part_bytes(const CausalParams &p, int num_cu) { return part_bytes_of(p, choose_paged, num_cu); }

size_t attn_prompt_part_bytes(const CausalParams &p, int num_cu)
{
    const size_t f = part_bytes_of(p, choose_prompt, num_cu), g = attn_grad_part_bytes(p, num_cu);
    return f > g ? f : g;
}

}  // namespace cf
