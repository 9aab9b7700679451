// Device helpers of the causal attention kernels: direct loads to LDS, fragment types, the search of a packed sequence.
#pragma once
#include "decoder_internal.h"

#include <cmath>
#include <type_traits>
#include <utility>

namespace cf {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));

constexpr int DH = 128;                  // head dimension these kernels are written for
constexpr int BKV = 64;                  // keys per tile
constexpr int ROWB = DH * 2;             // bytes of one key / value row in LDS (bf16)
constexpr int TILE_BYTES = BKV * ROWB;   // 16 KiB
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

template <typename T>
__device__ __forceinline__ T uniform(T v)
{
    if constexpr (sizeof(T) == 8) {
        const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
        const unsigned lo = __builtin_amdgcn_readfirstlane((int)(unsigned)u), hi = __builtin_amdgcn_readfirstlane((int)(unsigned)(u >> 32));
        return __builtin_bit_cast(T, ((unsigned long long)hi << 32) | lo);
    } else {
        return __builtin_bit_cast(T, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
    }
}

// A buffer of `bytes` bytes from a wave-uniform address: what lies behind it reads as zero.
__device__ __forceinline__ i32x4_t make_rsrc(const void *base, unsigned bytes)
{
    const unsigned long long a = reinterpret_cast<unsigned long long>(base);
    i32x4_t r;
    r[0] = __builtin_amdgcn_readfirstlane((int)(a & 0xFFFFFFFFull));
    r[1] = __builtin_amdgcn_readfirstlane((int)((a >> 32) & 0xFFFFull));
    r[2] = __builtin_amdgcn_readfirstlane((int)bytes);
    r[3] = 0x00020000;
    return r;
}

// The same for the compiler's own buffer accesses.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t plain_rsrc(const void *base, int bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(uniform(base)), 0, uniform(bytes), 0x00020000);
}

// Wave-wide 16-byte-per-lane load from global memory straight into LDS (lane L lands at lds_addr + 16 L).
__device__ __forceinline__ void direct_load_16(i32x4_t rsrc, unsigned voffset, unsigned lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\t"
                 "buffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(lds_addr), "v"(voffset), "s"(rsrc)
                 : "memory");
}

template <int N>
__device__ __forceinline__ void wait_vmcnt()
{
    __builtin_amdgcn_s_waitcnt((N & 0xF) | (0x7 << 4) | (0xF << 8) | ((N >> 4) << 14));
}

// f(FIRST), f(FIRST + STEP), ... as compile-time constants
template <int FIRST, int STEP, int... I, typename F>
__device__ __forceinline__ void each(F &f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, FIRST + STEP * I>{}), ...);
}

__device__ __forceinline__ unsigned lds_address(const void *p)
{
    return __builtin_amdgcn_readfirstlane((unsigned)(size_t)(__attribute__((address_space(3))) const unsigned char *)p);
}

// Maximum / sum over the two lanes (lane, lane ^ 32) that share a query.
__device__ __forceinline__ float max_of_halves(float x)
{
    const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const unsigned a = both[0], b = both[1];
    return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
__device__ __forceinline__ float sum_of_halves(float x)
{
    const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const unsigned a = both[0], b = both[1];
    return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}

// A start that a table holds, as a row of the tensor or the one behind its last, whatever it is.
__device__ __forceinline__ int clamped(int start, int tokens) { return start < 0 ? 0 : start < tokens ? start : tokens; }

// Inclusive sums over the wave's lanes.
__device__ __forceinline__ int scan(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // from 1, 2, 4, 8 lanes below in a row of 16
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // rows 1 and 3: the last lane of the row below
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // rows 2 and 3: lane 31
    return x;
}
__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(scan(x), 63); }
// The largest of the lanes' values, and zero.
__device__ __forceinline__ int wave_most(int x)
{
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
    return __builtin_amdgcn_readlane(x, 63);
}

// The packed sequences' starts, as every wave needs them: up to 64 sequences from one load, a start a lane; more from memory.
struct Sequences {
    const int32_t *starts;
    int n, first, mine;                  // starts[0]; starts[1 + lane] (behind the last: 2^31 - 1)
    __device__ __forceinline__ Sequences(const int32_t *s, int count) : starts(s), n(count)
    {
        const int lane = threadIdx.x & 63;
        first = s[0];
        mine = lane < n ? s[1 + lane] : 0x7FFFFFFF;
    }
    // starts[1 + i], i wave-uniform, in [0, n)
    __device__ __forceinline__ int end_of(int i) const { return n <= 64 ? __builtin_amdgcn_readlane(mine, i) : uniform(starts[1 + i]); }
    __device__ __forceinline__ int start_of(int i) const { return i == 0 ? uniform(first) : end_of(i - 1); }
    // how many of starts[1 ..] are <= t, for a wave-uniform t: sixty-four probes at a time
    __device__ __forceinline__ int at(int t) const
    {
        if (n <= 64)
            return __builtin_popcountll(__builtin_amdgcn_ballot_w64(mine <= t));
        const int lane = threadIdx.x & 63;
        int lo = 0, hi = n;
        while (lo < hi) {
            const int step = (hi - lo + 63) / 64, i = lo + lane * step;
            const int c = __builtin_popcountll(__builtin_amdgcn_ballot_w64(i < hi && starts[1 + (i < hi ? i : lo)] <= t));
            const int end = lo + c * step;
            hi = c == 0 ? lo : hi < end ? hi : end;
            lo = c == 0 ? lo : end - step + 1;
        }
        return uniform(lo);
    }
    // ... for a t of the lane's own, between two answers that enclose it (every lane takes part), and that sequence's two ends
    __device__ __forceinline__ int between(int a, int b, int t, int *start, int *end) const
    {
        while (__builtin_amdgcn_ballot_w64(a < b) != 0) {
            const int mid = (a + b) >> 1, s = n <= 64 ? __shfl(mine, mid & 63) : starts[1 + (mid < n ? mid : n - 1)];
            if (a < b) {
                if (s <= t)
                    a = mid + 1;
                else
                    b = mid;
            }
        }
        const int i = a < n ? a : n - 1;
        const int before = n <= 64 ? __shfl(mine, i > 0 ? i - 1 : 0) : starts[i];
        *end = n <= 64 ? __shfl(mine, i) : starts[1 + i];
        *start = i > 0 ? before : first;
        return a;
    }
    // tokens of the longest sequence; up to 64 sequences
    __device__ __forceinline__ int longest() const
    {
        const int lane = threadIdx.x & 63, before = __shfl_up(mine, 1);
        return wave_most(lane < n ? mine - (lane > 0 ? before : first) : 0);
    }
    // where the sequence of the lane's token t begins, and where it ends (2^31 - 1: t is behind the last); up to 64 sequences.  Every
    // lane takes part.
    __device__ __forceinline__ void around(int t, int *start, int *end) const
    {
        if (n <= 8) {
            *start = first;
            *end = 0x7FFFFFFF;
#pragma unroll 1
            for (int i = 0; i < n; ++i) {
                const int e = __builtin_amdgcn_readlane(mine, i);
                *start = e <= t ? e : *start;
                *end = e > t && e < *end ? e : *end;
            }
        } else {
            int i = 0;                   // how many are <= t
#pragma unroll 1
            for (int step = 32; step > 0; step /= 2)
                i += __shfl(mine, i + step - 1) <= t ? step : 0;
            i += __shfl(mine, i) <= t;
            const int before = __shfl(mine, (i - 1) & 63), e = __shfl(mine, i & 63);
            *start = i > 0 ? before : first;
            *end = i < n ? e : 0x7FFFFFFF;
        }
    }
};

// What a workgroup works on.  Walks under a causal mask are of all lengths, which only the tables on the device know, and a launch takes as
// long as its fullest compute unit.  So every workgroup looks at the walks of all blocks, a thread a block, and cuts them into splits of at most
// `chunk` tiles, the same for all, as few as make no more than P.items workgroups: as many as fit the chip a whole number of times.
// (Computed for one and eight heads, one sequence and several, workgroups one by one on the compute units: with 256 of 128 to 252
// workgroups each takes 33 us, with a quarter more than fit, 47.)  A grid of all blocks by the largest number of splits needs no
// search, but three workgroups of four then have nothing to do and hold up the others: dK and dV of 4096 tokens, 8 heads on one key
// head, took 148 us so.
constexpr int MAX_BLOCKS = 512;          // of one key head, that are looked at
struct Item {
    int kvh, block, split, splits;       // key heads innermost: neighbouring workgroups go to one XCD in turn, whose L2 holds few heads' keys
    int first;                           // the block's split 0 is this one of its key head's items
    // The split's share of `tiles`: [*from, *to)
    __device__ __forceinline__ void share(int tiles, int *from, int *to) const
    {
        const unsigned each = (unsigned)tiles / (unsigned)splits;
        const int over = tiles - (int)each * splits;
        *from = (int)each * split + (split < over ? split : over);
        *to = *from + (int)each + (split < over);
    }
};

// The splits of all blocks, by a workgroup of NT threads.  tiles_of(block): tiles of a lane's block (0: nothing to do), in the order of
// dispatch.  They lie in LDS and all loops are loops: unrolled, eight blocks a lane in registers, the same took 1 us more, much of it
// for fetching 14 KiB of instructions.
// PAIRED: two workgroups share a compute unit.
template <int NT, bool PAIRED>
struct Splits {
    const int *tiles;
    int chunk, blocks, items;
    // `grain`: a split takes a multiple of it, where a workgroup's waves take tiles in turn.  `bound`: no walk is longer.  Where that is not
    // worth a split (twice the least) the walks are not looked at: 16 prompts of 512 tokens 22.7 us, looked at 26.
    template <typename F>
    __device__ __forceinline__ Splits(const CausalParams &P, int count, int least, int grain, int bound, F &&tiles_of, int *lds) : tiles(lds), chunk(P.chunk), blocks(count)
    {
        const bool whole = chunk == 0 && bound <= 2 * least;
        const int lane = threadIdx.x & 63, up = (count + 63) & ~63;
#pragma unroll 1
        for (int b = threadIdx.x; b < up; b += NT) {                 // (whole waves)
            const int t = whole ? 1 : tiles_of(b < count ? b : count - 1);
            lds[b] = b < count ? t : 0;
        }
        __syncthreads();
        if (whole)
            chunk = 1;
        if (chunk > 0) {
            items = number();
            return;
        }
        int all = 0, some = 0;
#pragma unroll 1
        for (int b = lane; b < up; b += 64) {
            all += lds[b];
            some += lds[b] > 0;
        }
        const int total = wave_total(all), active = wave_total(some), most = P.items / P.kv_heads;
        const float wanted = fmaxf((float)most - 0.5f * active, 1.0f);           // a walk's last split is half as long as the others
        // (nor much less than a compute unit's share of all, or, paired, than 40 tiles: 512 blocks of 1 to 64 tiles took 82 us in pieces of 28 and
        // 74 in pieces of 40, 256 of them 52 in pieces of 26 and 49 of 40)
        const float share = (float)total * P.kv_heads / P.num_cu;
        chunk = max(max(least, (int)(total / wanted) + 1), PAIRED ? min((int)(1.2f * share), 40) : (int)(0.8f * share));
        chunk = (chunk + grain - 1) / grain * grain;
#pragma unroll 1
        while ((items = number()) > most)
            chunk += chunk / 16 / grain * grain + grain;
    }
    __device__ __forceinline__ int of(int t) const { return t <= 0 ? 0 : (int)((float)(t + chunk - 1) * __builtin_amdgcn_rcpf((float)chunk) * 1.0000002f); }
    __device__ __forceinline__ int number() const
    {
        int n = 0;
#pragma unroll 1
        for (int b = 0; b < blocks; b += 64)
            n += of(tiles[b + (threadIdx.x & 63)]);
        return wave_total(n);
    }
    // Item j of a key head: false: there are not so many.
    __device__ __forceinline__ bool item(int j, Item *it) const
    {
        int base = 0;
#pragma unroll 1
        for (int b = 0; b < blocks; b += 64) {
            const int n = of(tiles[b + (threadIdx.x & 63)]), end = base + scan(n);
            const unsigned long long behind = __builtin_amdgcn_ballot_w64(end > j);
            if (behind != 0) {
                const int lane = __builtin_ctzll(behind);
                it->splits = __builtin_amdgcn_readlane(n, lane);
                it->first = __builtin_amdgcn_readlane(end, lane) - it->splits;
                it->block = b + lane;
                it->split = j - it->first;
                return true;
            }
            base = __builtin_amdgcn_readlane(end, 63);
        }
        return false;
    }
    // The splits of a block, and the first of their items.
    __device__ __forceinline__ void of_block(int block, Item *it) const
    {
        int base = 0;
#pragma unroll 1
        for (int b = 0; b <= block; b += 64) {
            const int n = of(tiles[b + (threadIdx.x & 63)]), end = base + scan(n);
            it->splits = __builtin_amdgcn_readlane(n, block & 63);
            it->first = __builtin_amdgcn_readlane(end, block & 63) - it->splits;
            base = __builtin_amdgcn_readlane(end, 63);
        }
    }
};

// This workgroup's item; `blocks`: of one key head.
// PAIRED: two workgroups share a compute unit, those that are dispatched a whole chip apart.  The second half of the first two rounds is
// handed out backwards: items become shorter towards the end of a sequence's rows, and two of the same place would share.
template <int NT, bool PAIRED, typename F>
__device__ __forceinline__ bool my_item(const CausalParams &P, int blocks, int least, int grain, int bound, F &&tiles_of, Item *it)
{
    __shared__ int tiles[MAX_BLOCKS];
    int j = blockIdx.x / P.kv_heads;
    it->kvh = blockIdx.x - j * P.kv_heads;
    auto paired = [&](int number) {
        const int round = P.num_cu / P.kv_heads, end = number < 2 * round ? number : 2 * round;
        return PAIRED && j >= round && j < end ? round + end - 1 - j : j;
    };
    if (P.items == 0) {
        it->block = it->first = paired(gridDim.x / P.kv_heads);
        it->split = 0;
        it->splits = 1;
        return true;
    }
    const Splits<NT, PAIRED> splits(P, blocks, least, grain, bound, tiles_of, tiles);
    return splits.item(paired(splits.items), it);
}

// Smallest and largest of a wave's `first` and `last`, both of which grow with the row (lanes 0 .. 31, and the same in the others), over
// the rows that are there.  False: none is.
__device__ __forceinline__ bool edges(bool there, int first, int last, int *f_min, int *f_max, int *l_min, int *l_max)
{
    const unsigned rows = (unsigned)__builtin_amdgcn_ballot_w64(there);
    if (rows == 0)
        return false;
    const int a = __builtin_ctz(rows), b = 31 - __builtin_clz(rows);
    *f_min = __builtin_amdgcn_readlane(first, a);
    *f_max = __builtin_amdgcn_readlane(first, b);
    *l_min = __builtin_amdgcn_readlane(last, a);
    *l_max = __builtin_amdgcn_readlane(last, b);
    return true;
}
// Where item `first + split` of a block parks what it has: N floats a workgroup.
__device__ __forceinline__ float *parked_at(const CausalParams &P, const Item &it, int split, size_t floats)
{
    return P.parts + ((size_t)(it.first + split) * P.kv_heads + it.kvh) * floats;
}

enum { PACKED = 0, PAGED_BF16 = 1, PAGED_E4M3 = 2 };

// Where a sequence's (or the pack's) keys lie, for single rows: the pointer of key `key` (nullptr: its page does not exist), and its
// scale.
template <int SRC>
struct Keys {
    const unsigned char *base;       // packed: key 0 of this head
    int64_t row_bytes;
    const int32_t *table;            // paged: this sequence's row
    const uint8_t *exps;
    int64_t page_bytes, n_pages, exp_page;
    int shift;

    __device__ __forceinline__ const unsigned char *row(int key, int *e) const
    {
        if constexpr (SRC == PACKED) {
            return base + (int64_t)key * row_bytes;
        } else {
            const int64_t page = table[key >> shift];
            if ((uint64_t)page >= (uint64_t)n_pages)
                return nullptr;
            const int in_page = key & ((1 << shift) - 1);
            if constexpr (SRC == PAGED_E4M3)
                *e = (int)exps[page * exp_page + in_page] - 127;
            return base + page * page_bytes + in_page * row_bytes;
        }
    }
    __device__ __forceinline__ f32x2_t pair(const unsigned char *row, int i, int e) const    // features 2 i and 2 i + 1
    {
        if constexpr (SRC == PAGED_E4M3) {
            const f32x2_t v = __builtin_amdgcn_cvt_pk_f32_fp8((int)reinterpret_cast<const unsigned short *>(row)[i], false);
            return f32x2_t{ldexpf(v[0], e), ldexpf(v[1], e)};
        } else {
            const bf16x2_t v = reinterpret_cast<const bf16x2_t *>(row)[i];
            return f32x2_t{(float)v[0], (float)v[1]};
        }
    }
};

// Sums that are NaN in every lane stay so.  (Of inputs that are NaN throughout, 8192 keys for every row, one by one, would take some 40 ms by
// the count of instructions.)
__device__ __forceinline__ bool settled(float a, float b) { return __builtin_amdgcn_ballot_w64(a == a || b == b) == 0; }

// One row's attention by one wave, key by key, in two passes; lane i holds features 2 i and 2 i + 1.
template <int SRC>
__device__ __forceinline__ void careful_row(const Keys<SRC> &K, const Keys<SRC> &V, const __bf16 *q, __bf16 *out, int first, int last, float sl2)
{
    const int lane = threadIdx.x & 63;
    const float q0 = (float)q[2 * lane], q1 = (float)q[2 * lane + 1];
    float m = -INFINITY, l = 0.0f, o0 = 0.0f, o1 = 0.0f;
    for (int pass = 0; pass < 2; ++pass)
        for (int key = first; key <= last; ++key) {
            int e = 0;
            const unsigned char *k = K.row(key, &e);
            if (k == nullptr)
                continue;
            const f32x2_t kv = K.pair(k, lane, e);
            float s = q0 * kv[0] + q1 * kv[1];
#pragma unroll
            for (int d = 1; d < 64; d *= 2)
                s += __shfl_xor(s, d);
            s *= sl2;
            if (pass == 0) {
                m = fmaxf(m, s);
                if (!(s < INFINITY))                                 // this key's p is NaN, and so is everything
                    break;
            } else {
                const float p = exp2f(s - (m == -INFINITY ? 0.0f : m));
                const f32x2_t v = V.pair(V.row(key, &e), lane, e);
                l += p;
                o0 += p * v[0];
                o1 += p * v[1];
                if (settled(o0, o1))
                    break;
            }
        }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    bf16x2_t r;
    r[0] = (__bf16)(o0 * inv);
    r[1] = (__bf16)(o1 * inv);
    reinterpret_cast<bf16x2_t *>(out)[lane] = r;
}

}  // namespace
}  // namespace cf
