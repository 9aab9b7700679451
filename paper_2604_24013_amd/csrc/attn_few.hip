// Attention of few rows over a paged cache for gfx950: decoded tokens, and a handful of new tokens at a time.
//
// Bound: HBM -- every visible key and value is read once for all rows of its key head.  So nothing of K or V goes through LDS and no
// wave waits for another: each wave walks over tiles of 32 keys of its own, straight from memory into the registers that the
// MFMAs read.
//   S^T = K Q^T     v_mfma_f32_16x16x32_bf16, 16 keys as "A" (a lane fetches 16 bytes of one key's row at a time), 16 rows as "B": a lane
//                   owns one row (lane & 15) and, with the keys of the two MFMA tiles interleaved by fours, the eight
//                   consecutive keys 8 (lane >> 4) .. + 7 of the tile;
//   O^T += V^T P^T  P, rounded to bf16, is in the layout of a "B" operand as it stands.  V: a lane fetches 8 features (8 l .. 8 l + 7, l =
//                   lane & 15) of each of those eight keys, whole rows by sixteen lanes; pairing the keys of a feature takes 32 byte
//                   permutes and gives the "A" operands of eight MFMAs, number n for the features 8 l + n.
// e4m3 codes become bf16 on the way in, with their row's power of two, which is exact.
// The next K tile is requested when the scores have taken the present one, the next V tile after its product; the page numbers two
// tiles ahead.  Keys behind the last are read from the last one's row and masked, those of pages that do not exist from page 0:
// every address is inside the pool.  The waves' (m, l, O) are merged in LDS, those of workgroups that share a sequence's keys in
// the workspace by the one that finishes last.
// Measured: 62 sequences of 33 to 4096 tokens, 4 heads of their own, bf16: 50 us, 4.4 TB/s of cache (a sum over memory reaches 4.0, a copy 4.7);
// eight contexts of 12 to 65 thousand, 8 heads of one key head, e4m3: 26.8 us, 3.7 TB/s; one of 1003: 8.9 us, of which 6 are the launch, the
// search and the merge.  With a window, whose walks leave out what nobody sees: 62 sequences of up to 16384 tokens, 4 heads of their own, bf16, window 2048 + 4:
// 51.9 us, 4.7 TB/s; the last 4096 + 4 of 100003 in e4m3, 8 heads of one key head: 11.2 us.
#include "attn_tiles.h"

namespace cf {
namespace {

constexpr int FEW_KEYS = 32;             // keys of a tile
constexpr int O_STRIDE = DH + 4;         // floats between rows of a parked O in LDS (the 16 rows of a store on different banks)

template <int NW, int QT, int SRC, bool WIN>
__global__ __launch_bounds__(64 * NW, 2) void attn_few_kernel(CausalParams P)
{
    constexpr int NT = 64 * NW;
    constexpr int ROWS = 16;             // rows of an MFMA tile
    constexpr bool E4M3 = SRC == PAGED_E4M3;

    __shared__ __attribute__((aligned(16))) float parked[NW * ROWS * O_STRIDE];
    __shared__ float stat_m[NW][ROWS], stat_l[NW][ROWS], stat_e[NW][ROWS];
    __shared__ unsigned arrived;
    __shared__ unsigned odd_rows[QT];    // whose result is not finite

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i = lane & 15, gq = lane >> 4;
    const int G = P.group;

    // Keys that a sequence's last row sees, over all of which its waves walk
    auto keys_of = [&](int seq) {
        const int q0 = P.starts[seq], q1 = P.starts[seq + 1];
        const int m = clamped(q1, P.tokens) - clamped(q0, P.tokens), some = m < P.max_q ? m : P.max_q;
        int n = P.kv_len[seq];
        n = (n < 0 ? 0 : n < P.max_kv ? n : P.max_kv) - m + some;
        return some <= 0 ? -1 : n > 0 ? n : 0;
    };
    // ... of which, with a window, some in the middle are seen by none: `rows` rows see `keys` keys, the last of them all
    auto gap_of = [&](int keys, int tokens) { return Gap<FEW_KEYS>(P.sinks, 0, keys, window_from(P, 0, keys - tokens)); };
    Item it;
    if (!my_item<NT, false>(P, P.n_seqs, NW, NW, 0x7FFFFFFF, 0, [&](int seq) {
            const int keys = keys_of(seq);
            if constexpr (WIN) {
                const int m = clamped(P.starts[seq + 1], P.tokens) - clamped(P.starts[seq], P.tokens);
                return keys < 0 ? 0 : max(1, gap_of(keys, m < P.max_q ? m : P.max_q).tiles(0, keys));
            }
            return keys < 0 ? 0 : max(1, (keys + FEW_KEYS - 1) / FEW_KEYS);
        }, &it))
        return;
    const int kvh = it.kvh, seq = it.block, split = it.split, splits = it.splits;
    const int group = seq * P.kv_heads + kvh;

    const int q0 = P.starts[seq], q1 = P.starts[seq + 1];
    const int from = clamped(q0, P.tokens), m = clamped(q1, P.tokens) - from;     // rows of the sequence
    int n = P.kv_len[seq];
    n = n < 0 ? 0 : n < P.max_kv ? n : P.max_kv;
    const int rows = (m < P.max_q ? m : P.max_q) * G;                // at most 16 QT
    if (rows <= 0)
        return;
    const int hi = n - m + (rows - 1) / G + 1 > 0 ? n - m + (rows - 1) / G + 1 : 0;   // keys that the last row sees
    const Gap<FEW_KEYS> gap = WIN ? gap_of(hi, (rows - 1) / G + 1) : Gap<FEW_KEYS>();
    auto place_of = [&](int tile) __attribute__((always_inline)) { return WIN ? gap.key(tile) : tile * FEW_KEYS; };      // a tile's first key
    const int tiles = WIN ? gap.tiles(0, hi) : (hi + FEW_KEYS - 1) / FEW_KEYS;
    int t0, t1;
    it.share(tiles, &t0, &t1);

    const int32_t *table = P.table + (int64_t)seq * P.max_pages;
    const int shift = P.pool.page_shift, n_pages = (int)P.pool.n_pages;
    constexpr int E = E4M3 ? 1 : 2;
    const int64_t page_bytes = P.pool.page_stride * E, row_bytes = P.pool.token_stride * E;
    const unsigned char *kb = static_cast<const unsigned char *>(P.pool.k) + kvh * P.pool.head_stride * E;
    const unsigned char *vb = static_cast<const unsigned char *>(P.pool.v) + kvh * P.pool.head_stride * E;
    const int64_t exp_page = (int64_t)P.pool.kv_heads << shift;
    const uint8_t *ke = E4M3 ? P.pool.k_exp + ((int64_t)kvh << shift) : nullptr;
    const uint8_t *ve = E4M3 ? P.pool.v_exp + ((int64_t)kvh << shift) : nullptr;

    // The lane's rows, one per row tile: their queries as "B" fragments.  Contraction slots: features 32 ks + 8 gq .. + 7 (bf16), or, so
    // that a lane's codes come in sixteens, 64 (ks >> 1) + 16 gq + 8 (ks & 1) .. + 7 (e4m3).
    bf16x8_t qf[QT][4];
    int last[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int r = t * ROWS + i < rows ? t * ROWS + i : 0;
        const int token = r / G;
        const __bf16 *q = static_cast<const __bf16 *>(P.Q) + (int64_t)(from + token) * P.q_token + (kvh * G + r - token * G) * P.q_head;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
            qf[t][ks] = *reinterpret_cast<const bf16x8_t *>(q + (E4M3 ? 64 * (ks >> 1) + 16 * gq + 8 * (ks & 1) : 32 * ks + 8 * gq));
        last[t] = n - m + token;
    }

    f32x4_t oacc[QT][8];
    float m_run[QT], l_run[QT], e_run[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        m_run[t] = -3.402823466e38f;
        l_run[t] = e_run[t] = 0.0f;
#pragma unroll
        for (int d = 0; d < 8; ++d)
            oacc[t][d] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const float sl2 = P.scale * LOG2E;
    constexpr float RAISE = 8.0f;
    bf16x2_t ones;
    ones[0] = ones[1] = (__bf16)1.0f;

    // K: rows of MFMA tile u, row i: key 8 (i >> 2) + 4 u + (i & 3) of the tile; V: keys 8 gq + j.
    const int k_eight = 8 * (i >> 2), v_eight = 8 * gq;
    struct Pages {
        int k, v;
    };
    auto key_of = [&](int tile, int eight) { const int key = place_of(tile) + eight; return key < hi ? key : hi - 1; };
    auto pages_of = [&](int tile) __attribute__((always_inline)) {
        Pages p;
        p.k = table[key_of(tile, k_eight) >> shift];
        p.v = table[key_of(tile, v_eight) >> shift];
        return p;
    };
    constexpr int KL = E4M3 ? 2 : 4;
    u32x4_t kc[2][KL], vc[E4M3 ? 4 : 8];                             // (e4m3: eight codes of V a row, two rows a register quadruple)
    float k_scale[2];
    u32x2_t v_exps;
    auto load_k = [&](int tile, const Pages &p) __attribute__((always_inline)) {
        const int page = (unsigned)p.k < (unsigned)n_pages ? p.k : 0;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int key = key_of(tile, k_eight + 4 * u + (i & 3));
            // (a key behind the last comes from the last one's row, which may lie in an earlier page than the eight that it stands in)
            const int in_page = key & ((1 << shift) - 1);
            const unsigned char *at = kb + page * page_bytes + in_page * row_bytes + gq * 16;
#pragma unroll
            for (int c = 0; c < KL; ++c)
                kc[u][c] = *reinterpret_cast<const u32x4_t *>(at + c * 64);
            if constexpr (E4M3)
                k_scale[u] = __builtin_bit_cast(float, (unsigned)ke[page * exp_page + in_page] << 23);
        }
    };
    auto load_v = [&](int tile, const Pages &p) __attribute__((always_inline)) {
        const int page = (unsigned)p.v < (unsigned)n_pages ? p.v : 0;
        const unsigned char *base = vb + page * page_bytes + i * (E4M3 ? 8 : 16);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int in_page = key_of(tile, v_eight + j) & ((1 << shift) - 1);
            if constexpr (E4M3) {
                const u32x2_t w = *reinterpret_cast<const u32x2_t *>(base + in_page * row_bytes);
                vc[j >> 1][2 * (j & 1)] = w[0];
                vc[j >> 1][2 * (j & 1) + 1] = w[1];
            } else {
                vc[j] = *reinterpret_cast<const u32x4_t *>(base + in_page * row_bytes);
            }
        }
        if constexpr (E4M3)
            v_exps = *reinterpret_cast<const u32x2_t *>(ve + page * exp_page + (key_of(tile, v_eight) & ((1 << shift) - 8)));
    };

    if (t0 + wave < t1) {
        int tile = t0 + wave;
        Pages now = pages_of(tile), next = pages_of(tile + NW);
        load_k(tile, now);
        load_v(tile, now);
        for (; tile < t1; tile += NW) {
            const bool more = tile + NW < t1;
            // scores: register 4 u + e is key 8 gq + 4 u + e
            bf16x8_t kf[2][4];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) {
                    if constexpr (E4M3) {
                        u32x4_t w;
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const unsigned code = kc[u][ks >> 1][2 * (ks & 1) + c];
                            w[2 * c] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code, k_scale[u], false));
                            w[2 * c + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code, k_scale[u], true));
                        }
                        kf[u][ks] = __builtin_bit_cast(bf16x8_t, w);
                    } else {
                        kf[u][ks] = __builtin_bit_cast(bf16x8_t, kc[u][ks]);
                    }
                }
            f32x4_t sc[QT][2];
#pragma unroll
            for (int t = 0; t < QT; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    sc[t][u] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        sc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[u][ks], qf[t][ks], sc[t][u], 0, 0, 0);
                }
            const bool none = (unsigned)now.v >= (unsigned)n_pages;  // the lane's eight keys are in no page
            Pages after = next;
            if (more) {
                after = pages_of(tile + 2 * NW);
                load_k(tile + NW, next);
            }
            __builtin_amdgcn_sched_barrier(0);

            bf16x8_t pf[QT];
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                const int key = place_of(tile) + v_eight;
                if constexpr (WIN) {
                    const SeesWindow sees(P, 0, last[t]);
                    if (__builtin_amdgcn_ballot_w64(none || key + 7 > last[t] || key < sees.from) != 0) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (none || !sees(key + e))
                                sc[t][e >> 2][e & 3] = -INFINITY;
                    }
                } else if (__builtin_amdgcn_ballot_w64(none || key + 7 > last[t]) != 0) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (none || key + e > last[t])
                            sc[t][e >> 2][e & 3] = -INFINITY;
                }
                float mx = sc[t][0][0];
#pragma unroll
                for (int e = 1; e < 8; ++e)
                    mx = fmaxf(mx, sc[t][e >> 2][e & 3]);
                mx *= sl2;
                if (__builtin_amdgcn_ballot_w64(mx > m_run[t] + RAISE) != 0) {
                    mx = fmaxf(mx, __shfl_xor(mx, 16));
                    mx = fmaxf(mx, __shfl_xor(mx, 32));
                    const float m_new = fmaxf(m_run[t], mx), alpha = exp2f(m_run[t] - m_new);
                    m_run[t] = m_new;
                    l_run[t] *= alpha;
                    e_run[t] *= alpha;
#pragma unroll
                    for (int d = 0; d < 8; ++d)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            oacc[t][d][e] *= alpha;
                }
                const float nm = -m_run[t];
                float es = 0.0f, ls = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    bf16x2_t two;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][(e + c) >> 2][(e + c) & 3], sl2, nm));
                        es += p;
                        two[c] = (__bf16)p;
                    }
                    ls = __builtin_amdgcn_fdot2_f32_bf16(two, ones, ls, false);
                    pf[t][e] = two[0];
                    pf[t][e + 1] = two[1];
                }
                e_run[t] += es;
                l_run[t] += ls;
            }

            if constexpr (E4M3) {                                    // exponents behind the last key may be anything
                const int real = hi - place_of(tile) - v_eight;
                if (place_of(tile) + FEW_KEYS > hi) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int have = real - 4 * c;
                        const unsigned keep = have >= 4 ? ~0u : have <= 0 ? 0u : (1u << 8 * have) - 1u;
                        v_exps[c] = (v_exps[c] & keep) | (0x7F7F7F7Fu & ~keep);
                    }
                }
            }
            // V of the eight keys, two features a register: then by feature, two keys a register
            unsigned v[8][4];
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    if constexpr (E4M3) {
                        const float scale = __builtin_bit_cast(float, (v_exps[j >> 2] >> (8 * (j & 3)) & 255u) << 23);
                        const unsigned code = vc[j >> 1][2 * (j & 1) + (c >> 1)];
                        v[j][c] = c & 1 ? __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code, scale, true))
                                        : __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code, scale, false));
                    } else {
                        v[j][c] = vc[j][c];
                    }
                }
#pragma unroll
            for (int d = 0; d < 8; ++d) {
                u32x4_t w;
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    w[c] = __builtin_amdgcn_perm(v[2 * c + 1][d >> 1], v[2 * c][d >> 1], d & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int t = 0; t < QT; ++t)
                    oacc[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w), pf[t], oacc[t][d], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (more)
                load_v(tile + NW, next);
            now = next;
            next = after;
        }
    }

    // Merge the waves, one row tile at a time; a thread takes four features of a row.
    const int64_t row_floats = DH + 4;                               // a parked row: O, m, l, e
    float *mine = P.parts == nullptr ? nullptr : parked_at(P, it, split, (size_t)QT * ROWS * row_floats);
    constexpr int COHERENT = 1 | 16;
    auto store_row = [&](int r, int c, const f32x4_t &o, float l) __attribute__((always_inline)) {
        const int token = r / G, head = kvh * G + r - token * G;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        bf16x4_t h;
        float odd = 0.0f;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const float y = o[x] * inv;
            odd = __builtin_fmaf(y, 0.0f, odd);
            h[x] = (__bf16)y;
        }
        *reinterpret_cast<u32x2_t *>(static_cast<__bf16 *>(P.out) + (int64_t)(from + token) * P.o_token + head * P.o_head + c * 4) = __builtin_bit_cast(u32x2_t, h);
        return odd != 0.0f && l == l;                                // (l is made of visible scores only)
    };
    auto finish_row = [&](int r, int c, const f32x4_t &o, float mm, float l, float e) __attribute__((always_inline)) {
        const int token = r / G, head = kvh * G + r - token * G;
        const bool odd = store_row(r, c, o, l);
        if (c == 0 && P.lse != nullptr)
            P.lse[(int64_t)head * P.lse_stride + from + token] = e == 0.0f ? -INFINITY : (mm + __log2f(e)) * LN2;
        return odd;
    };
    // Features 4 c .. 4 c + 3 of row r of what the waves parked in LDS.
    auto of_waves = [&](int r, int c, float *top, float *l, float *e) __attribute__((always_inline)) {
        float mm = -INFINITY, ll = 0.0f, ee = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w)
            mm = fmaxf(mm, stat_m[w][r]);
        f32x4_t a = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = exp2f(stat_m[w][r] - mm);                // (a wave that saw no key: nothing times a factor)
            const f32x4_t x = *reinterpret_cast<const f32x4_t *>(parked + (w * ROWS + r) * O_STRIDE + c * 4);
            ll += stat_l[w][r] * f;
            ee += stat_e[w][r] * f;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                a[k] += x[k] * f;
        }
        *top = mm;
        *l = ll;
        *e = ee;
        return a;
    };
    if (tid < QT)
        odd_rows[tid] = 0;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        if (t * ROWS >= rows)
            break;
        float l = l_run[t], e = e_run[t];
        l += __shfl_xor(l, 16);
        e += __shfl_xor(e, 16);
        l += __shfl_xor(l, 32);
        e += __shfl_xor(e, 32);
        if (t > 0)
            __syncthreads();                                         // the tile before has been read
        float *o = parked + (wave * ROWS + i) * O_STRIDE;
#pragma unroll
        for (int x = 0; x < 4; ++x) {                                // registers d = 0 .. 7 are features 8 (4 gq + x) + d
            *reinterpret_cast<f32x4_t *>(o + (4 * gq + x) * 8) = f32x4_t{oacc[t][0][x], oacc[t][1][x], oacc[t][2][x], oacc[t][3][x]};
            *reinterpret_cast<f32x4_t *>(o + (4 * gq + x) * 8 + 4) = f32x4_t{oacc[t][4][x], oacc[t][5][x], oacc[t][6][x], oacc[t][7][x]};
        }
        if (gq == 0) {
            stat_m[wave][i] = m_run[t];
            stat_l[wave][i] = l;
            stat_e[wave][i] = e;
        }
        __syncthreads();
        for (int u = tid; u < ROWS * DH / 4; u += NT) {
            const int r = u >> 5, c = u & 31, row = t * ROWS + r;
            if (row >= rows)
                continue;
            float mm, ll, ee;
            const f32x4_t a = of_waves(r, c, &mm, &ll, &ee);
            if (splits == 1) {
                if (finish_row(row, c, a, mm, ll, ee))
                    atomicOr(&odd_rows[t], 1u << r);
            } else {
                const auto rs = __builtin_amdgcn_make_buffer_rsrc(mine, 0, (int)(QT * ROWS * row_floats * 4), 0x00020000);
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, a), rs, (int)((row * row_floats + c * 4) * 4), 0, COHERENT);
                if (c == 0)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, f32x4_t{mm, ll, ee, 0.0f}), rs, (int)((row * row_floats + DH) * 4), 0, COHERENT);
            }
        }
    }
    if (splits > 1) {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (tid == 0)
            arrived = __hip_atomic_fetch_add(&P.counters[group], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (arrived != (unsigned)(splits - 1))
            return;
        if (tid == 0)
            __hip_atomic_store(&P.counters[group], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const int bytes = (int)(QT * ROWS * row_floats * 4);
        for (int u = tid; u < rows * 32; u += NT) {
            const int row = u >> 5, c = u & 31;
            f32x4_t a = {0.0f, 0.0f, 0.0f, 0.0f};
            float mm = -3.402823466e38f, ll = 0.0f, ee = 0.0f;
            constexpr int AT = 8;                                    // splits in flight (beyond the last: the last once more, unused)
            for (int sp0 = 0; sp0 < splits; sp0 += AT) {
                f32x4_t x[AT], st[AT];
#pragma unroll
                for (int k = 0; k < AT; ++k) {
                    const int sp = sp0 + k < splits ? sp0 + k : splits - 1;
                    const auto rs = __builtin_amdgcn_make_buffer_rsrc(parked_at(P, it, sp, (size_t)QT * ROWS * row_floats), 0, bytes, 0x00020000);
                    st[k] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)((row * row_floats + DH) * 4), 0, COHERENT));
                    x[k] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)((row * row_floats + c * 4) * 4), 0, COHERENT));
                }
                float top = mm;
#pragma unroll
                for (int k = 0; k < AT; ++k)
                    top = fmaxf(top, st[k][0]);
                const float back = exp2f(mm - top);
                mm = top;
                ll *= back;
                ee *= back;
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    a[y] *= back;
#pragma unroll
                for (int k = 0; k < AT; ++k) {
                    const float f = sp0 + k < splits ? exp2f(st[k][0] - mm) : 0.0f;
                    ll += st[k][1] * f;
                    ee += st[k][2] * f;
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        a[y] += sp0 + k < splits ? x[k][y] * f : 0.0f;
                }
            }
            if (finish_row(row, c, a, mm, ll, ee))
                atomicOr(&odd_rows[row / ROWS], 1u << (row % ROWS));
        }
    }
    // Rows whose result is not finite once more where what they do not see can have been the reason: the new tokens behind a row's own (a
    // single token's row sees all keys), the last key in the place of those behind it, or page 0 in the place of one that does not exist.  The waves
    // share the keys.
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    const unsigned odd = odd_rows[0] | (QT > 1 ? odd_rows[QT - 1] << 16 : 0u);
    if (odd == 0)
        return;
    Keys<SRC> Kk, Kv;
    Kk.base = kb;
    Kk.row_bytes = row_bytes;
    Kk.table = table;
    Kk.exps = ke;
    Kk.page_bytes = page_bytes;
    Kk.n_pages = n_pages;
    Kk.exp_page = exp_page;
    Kk.shift = shift;
    Kv = Kk;
    Kv.base = vb;
    Kv.exps = ve;
    bool unseen = false;                                             // values that no row sees may have been in the products
    auto pages_upto = [&](int keys) { return (int)(((unsigned)keys + (1u << shift) - 1) >> shift); };
    int in_front = 0, gone = 0;                                      // pages in front of a gap, and those in it, of which no key was in the products
    if constexpr (WIN) {
        in_front = pages_upto(gap.front * FEW_KEYS);
        gone = max(0, (place_of(gap.front) >> shift) - in_front);
    }
    for (int i = lane; i < pages_upto(hi) - gone; i += 64)
        unseen = unseen || (unsigned)table[WIN && i >= in_front ? i + gone : i] >= (unsigned)n_pages;
    if (SRC == PAGED_BF16 && hi % FEW_KEYS != 0) {                   // (the last key's V: NaN would be so in all rows that see it, infinite becomes NaN)
        int e;
        const unsigned char *row = Kv.row(hi - 1, &e);
        const unsigned w = row != nullptr ? reinterpret_cast<const unsigned *>(row)[lane] : 0;
        unseen = unseen || (w & 0x7FFFu) == 0x7F80 || (w >> 16 & 0x7FFFu) == 0x7F80;
    }
    // Keys of the walk that some rows do not see: those behind the first row's own; with a window those behind the first keys, and in front of the last
    // row's window.  (Of a single token's walk these are parts of two tiles.  With all keys behind the gap looked at, a feature of V that is infinite in its
    // window, of 4096 keys in e4m3, cost 204 us instead of 14.)
    auto hidden_is_large = [&]() {
        if (any_large(Kv, max(n - m + 1, 0), hi))
            return true;
        if constexpr (WIN) {
            const int front = min(hi, gap.front * FEW_KEYS);
            return any_large(Kv, min(P.sinks, front), front) || any_large(Kv, place_of(gap.front), min(hi, window_from(P, 0, hi - 1)));
        }
        return false;
    };
    if (__builtin_amdgcn_ballot_w64(unseen) == 0 && !hidden_is_large())
        return;
    const int lq = lane & 31, lh = lane >> 5, r = lq < rows ? lq : 0, token = r / G;
    f32x16_t acc[DH / 32];
    float m_row, l_row;
    const auto sees = [&]() {
        if constexpr (WIN)
            return SeesWindow(P, 0, n - m + token);
        else
            return SeesUpTo{0, n - m + token};
    }();
    rows_again<SRC>(Kk, Kv, static_cast<const __bf16 *>(P.Q) + (int64_t)(from + token) * P.q_token + (kvh * G + r - token * G) * P.q_head, sees,
                    odd >> lq & 1u, sl2, wave, NW, acc, &m_row, &l_row);
    for (int t = 0; t < QT; ++t) {
        __syncthreads();                                             // (the rows before have been read)
        if (lq >> 4 == t) {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                *reinterpret_cast<f32x4_t *>(parked + (wave * ROWS + (lq & 15)) * O_STRIDE + 4 * (8 * (e >> 2) + 4 * lh + (e & 3))) =
                    f32x4_t{acc[0][e], acc[1][e], acc[2][e], acc[3][e]};
            stat_m[wave][lq & 15] = m_row;
            stat_l[wave][lq & 15] = l_row;
        }
        __syncthreads();
        for (int u = tid; u < ROWS * DH / 4; u += NT)
            if (odd >> (t * ROWS + (u >> 5)) & 1u) {
                float mm, ll, ee;
                const f32x4_t a = of_waves(u >> 5, u & 31, &mm, &ll, &ee);
                store_row(t * ROWS + (u >> 5), u & 31, a, ll);
            }
    }
}

template <int NW, int QT, bool WIN>
hipError_t launch(const CausalParams &p, int64_t wgs, hipStream_t s)
{
    if (wgs * 64 * NW >= ((int64_t)1 << 32))
        return hipErrorInvalidValue;
    if (p.pool.e4m3)
        hipLaunchKernelGGL((attn_few_kernel<NW, QT, PAGED_E4M3, WIN>), dim3((unsigned)wgs), dim3(64 * NW), 0, s, p);
    else
        hipLaunchKernelGGL((attn_few_kernel<NW, QT, PAGED_BF16, WIN>), dim3((unsigned)wgs), dim3(64 * NW), 0, s, p);
    return hipGetLastError();
}

int choose_few(CausalParams &p, int num_cu, int64_t *wgs, size_t *part)          // 16-row tiles; the launch's workgroups
{
    const int qt = p.max_q * p.group <= 16 ? 1 : 2;
    *part = (size_t)(qt * 16) * (DH + 4) * sizeof(float);
    int64_t longest = (p.max_kv + FEW_KEYS - 1) / FEW_KEYS;
    if (p.window > 0 && ((int64_t)p.window + p.sinks + p.max_q + 3 * FEW_KEYS) / FEW_KEYS < longest)
        longest = ((int64_t)p.window + p.sinks + p.max_q + 3 * FEW_KEYS) / FEW_KEYS;
    *wgs = plan_items(p, p.n_seqs, longest, 8, *part, true, num_cu);
    return qt;
}

}  // namespace

bool attn_few_takes(const CausalParams &p) { return (int64_t)p.max_q * p.group <= 32; }

hipError_t launch_attn_few(const CausalParams &p_in, hipStream_t s, int num_cu)
{
    CausalParams p = p_in;
    int64_t wgs;
    size_t part;
    const bool one = choose_few(p, num_cu, &wgs, &part) == 1;
    if (p.window > 0)
        return one ? launch<8, 1, true>(p, wgs, s) : launch<8, 2, true>(p, wgs, s);
    return one ? launch<8, 1, false>(p, wgs, s) : launch<8, 2, false>(p, wgs, s);
}

size_t attn_few_part_bytes(const CausalParams &p_in, int num_cu)
{
    CausalParams p = p_in;                                           // as if any workspace were there
    p.parts = reinterpret_cast<float *>(256);
    p.part_bytes = (size_t)1 << 48;
    p.max_counters = 1 << 30;
    int64_t wgs;
    size_t part;
    choose_few(p, num_cu, &wgs, &part);
    return (size_t)p.items * part;
}

}  // namespace cf
