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
typedef unsigned short u16x8_t __attribute__((ext_vector_type(8)));

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

// Does a row of bf16 features hold a value that is not finite, or of 2^60 and more?
__device__ __forceinline__ bool large_row(const __bf16 *row)
{
    unsigned most = 0;
    for (int i = 0; i < DH / 8; ++i) {
        const u32x4_t w = reinterpret_cast<const u32x4_t *>(row)[i];
#pragma unroll
        for (int c = 0; c < 4; ++c)
            most = max(most, max(w[c] & 0x7FFFu, w[c] >> 16 & 0x7FFFu));
    }
    return most >= (127 + 60) << 7;
}

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
    __device__ __forceinline__ bf16x8_t eight(const unsigned char *row, int i, int e) const   // features 8 i .. 8 i + 7
    {
        if constexpr (SRC == PAGED_E4M3) {
            const u32x2_t code = reinterpret_cast<const u32x2_t *>(row)[i];
            const float scale = __builtin_bit_cast(float, (unsigned)(e + 127) << 23);
            u32x4_t w;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                w[2 * c] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[c], scale, false));
                w[2 * c + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[c], scale, true));
            }
            return __builtin_bit_cast(bf16x8_t, w);
        } else {
            return reinterpret_cast<const bf16x8_t *>(row)[i];
        }
    }
    __device__ __forceinline__ u32x2_t four(const unsigned char *row, int i, int e) const     // features 4 i .. 4 i + 3
    {
        if constexpr (SRC == PAGED_E4M3) {
            const unsigned code = reinterpret_cast<const unsigned *>(row)[i];
            const float scale = __builtin_bit_cast(float, (unsigned)(e + 127) << 23);
            return u32x2_t{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code, scale, false)),
                           __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code, scale, true))};
        } else {
            return reinterpret_cast<const u32x2_t *>(row)[i];
        }
    }
    // Does a row hold a value that is not finite, or of 2^60 and more?  (Products of 128 smaller ones do not overflow.)
    __device__ __forceinline__ bool large(const unsigned char *row, int e) const
    {
        if constexpr (SRC == PAGED_E4M3) {
            unsigned nan = 0;
            for (int i = 0; i < DH / 16; ++i) {
                const u32x4_t w = reinterpret_cast<const u32x4_t *>(row)[i];
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    nan |= (w[c] & 0x7F7F7F7Fu) + 0x01010101u;       // (0x7F is NaN)
            }
            return e > 50 || (nan & 0x80808080u) != 0;
        } else {
            return large_row(reinterpret_cast<const __bf16 *>(row));
        }
    }
};

// Results that are not finite.  The mask is a select on the scores, so that a hidden key has a probability of 0 -- but 0 times an infinite or
// NaN value of V is NaN.  Only the tiles on a wave's border hold keys that some of its rows see and others do not.  So a wave that finds a
// result that is not finite looks at the V rows of those tiles (64 keys at a time, a lane each).  If one of them is not finite, the wave walks over
// all keys once more, from memory, with such values taken out of the product and counted for the rows that see them; otherwise what is
// visible is not finite, and the result stays.  Bound by the latency of its loads: 3 us for 32 keys, about three times as long as an unsplit
// walk of the kernels takes.  6144 tokens, 4 heads of one key head: 70 us, with one infinite feature of V in an early token too, in a late one 572.
// Is one of the rows [from, to) large?
template <int SRC>
__device__ __forceinline__ bool any_large(const Keys<SRC> &K, int from, int to)
{
    for (; from < to; from += 64) {
        const int key = from + (int)(threadIdx.x & 63);
        int e = 0;
        const unsigned char *row = key < to ? K.row(key, &e) : nullptr;
        if (__builtin_amdgcn_ballot_w64(row != nullptr && K.large(row, e)) != 0)
            return true;
    }
    return false;
}

// acc[d] += a[d] w (an MFMA's "A" and "B" operands), d the feature tiles, where elements of `a` that are not finite count for the columns that see
// their index only (bit x of `seen`: slot x): they are taken out of `a`, and products of ones say which results they make +inf, -inf or NaN.
template <int TILES>
__device__ __forceinline__ void add_seen(f32x16_t (&acc)[TILES], bf16x8_t (&a)[TILES], bf16x8_t w, unsigned seen)
{
    u16x8_t most = {};
#pragma unroll
    for (int d = 0; d < TILES; ++d)
        most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x8_t, a[d]) & (unsigned short)0x7FFF);
    bool finite = true;
#pragma unroll
    for (int x = 0; x < 8; ++x)
        finite = finite && most[x] < 0x7F80;
    if (__builtin_amdgcn_ballot_w64(!finite) != 0) {
        constexpr unsigned short ONE = 0x3F80;
        u16x8_t plus, minus;                                         // what they are multiplied by
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const bool sees = seen >> x & 1, negative = (float)w[x] < 0.0f;
            plus[x] = sees && !negative ? ONE : 0;
            minus[x] = sees && negative ? ONE : 0;
        }
#pragma unroll 1
        for (int i = 0; i < 2 * (TILES); ++i) {                    // (the code is there once) tile i / 2: what makes it +inf, what makes it -inf
            u16x8_t bits = __builtin_bit_cast(u16x8_t, a[0]), up, down;
#pragma unroll
            for (int d = 1; d < TILES; ++d)
                bits = i >> 1 == d ? __builtin_bit_cast(u16x8_t, a[d]) : bits;
            const unsigned short sign = i & 1 ? 0x8000 : 0;
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const bool nan = (bits[x] & 0x7FFF) > 0x7F80;
                up[x] = nan || bits[x] == (0x7F80 | sign) ? ONE : 0;
                down[x] = nan || bits[x] == (0xFF80 ^ sign) ? ONE : 0;
            }
            const f32x16_t zero = {};
            f32x16_t n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, up), __builtin_bit_cast(bf16x8_t, plus), zero, 0, 0, 0);
            n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, down), __builtin_bit_cast(bf16x8_t, minus), n, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float more = n[e] > 0.0f ? (i & 1 ? -INFINITY : INFINITY) : 0.0f;
#pragma unroll
                for (int d = 0; d < TILES; ++d)
                    acc[d][e] += i >> 1 == d ? more : 0.0f;
            }
        }
#pragma unroll
        for (int d = 0; d < TILES; ++d) {
            const u16x8_t bits = __builtin_bit_cast(u16x8_t, a[d]);
            u16x8_t kept;
#pragma unroll
            for (int x = 0; x < 8; ++x)
                kept[x] = (bits[x] & 0x7FFF) < 0x7F80 ? bits[x] : 0;
            a[d] = __builtin_bit_cast(bf16x8_t, kept);
        }
    }
#pragma unroll
    for (int d = 0; d < TILES; ++d)
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[d], w, acc[d], 0, 0, 0);
}

__device__ __forceinline__ bool none_finite(const f32x16_t &x)
{
    bool finite = false;
#pragma unroll
    for (int e = 0; e < 16; ++e)
        finite = finite || __builtin_isfinite(x[e]);
    return !finite;
}
// Smallest / largest of the wave's values.
__device__ __forceinline__ int least_of(int x)
{
    for (int d = 1; d < 64; d *= 2)
        x = min(x, __shfl_xor(x, d));
    return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ int most_of(int x) { return -least_of(-x); }
// What lanes at + 4 (lane / 32) hold, for a constant `at`: of the rows 0 .. 31 that lanes 0 .. 31 look up, those that an MFMA operand's slots stand for.
__device__ __forceinline__ int of_slot(int x, int at)
{
    const int low = __builtin_amdgcn_readlane(x, at), high = __builtin_amdgcn_readlane(x, at + 4);
    return threadIdx.x & 32 ? high : low;
}
template <typename T>
__device__ __forceinline__ const T *of_slot(const T *p, int at)
{
    const unsigned long long u = reinterpret_cast<unsigned long long>(p);
    const unsigned lo = of_slot((int)(unsigned)u, at), hi = of_slot((int)(unsigned)(u >> 32), at);
    return reinterpret_cast<const T *>((unsigned long long)hi << 32 | lo);
}

// "A" operands of the transposed product: four features 4 n .. 4 n + 3 of rows 2 i and 2 i + 1, n = lane & 31, go to slots 2 i and 2 i + 1 of the four
// feature tiles, so that register e of tile d of the result is feature 4 (8 (e >> 2) + 4 half + (e & 3)) + d.
__device__ __forceinline__ void put_pair(bf16x8_t (&a)[DH / 32], int i, u32x2_t even, u32x2_t odd)
{
#pragma unroll
    for (int d = 0; d < DH / 32; ++d) {
        u32x4_t w = __builtin_bit_cast(u32x4_t, a[d]);
        w[i] = __builtin_amdgcn_perm(odd[d >> 1], even[d >> 1], d & 1 ? 0x07060302u : 0x05040100u);
        a[d] = __builtin_bit_cast(bf16x8_t, w);
    }
}
// A lane's row of such a result, times `factor`, as bf16.
__device__ __forceinline__ void store_fours(const f32x16_t (&acc)[DH / 32], float factor, __bf16 *row)
{
    const int lh = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        bf16x4_t h;
#pragma unroll
        for (int d = 0; d < DH / 32; ++d)
            h[d] = (__bf16)(acc[d][e] * factor);
        *reinterpret_cast<u32x2_t *>(row + 4 * (8 * (e >> 2) + 4 * lh + (e & 3))) = __builtin_bit_cast(u32x2_t, h);
    }
}

// Attention of up to 32 rows by one wave, from memory: lane (row = lane & 31, and the same in the other half) sees keys first .. last; results where
// `wanted`: m, l, and O^T as `put_pair` has it.  The wave takes units of 32 keys nth, nth + step, ... from the first that is seen on.
template <int SRC>
__device__ __forceinline__ void rows_again(const Keys<SRC> &K, const Keys<SRC> &V, const __bf16 *q, int first, int last, bool wanted, float sl2, int nth, int step,
                                           f32x16_t (&acc)[DH / 32], float *max_score, float *sum)
{
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));                                   // (nothing made of it is kept over the walk before)
    const int lq = lane & 31, lh = lane >> 5;
    const int from = least_of(wanted ? first : 0x7FFFFFFF), to = most_of(wanted ? last : -1);
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            acc[d][i] = 0.0f;
    float m = -3.402823466e38f, l = 0.0f;
#pragma unroll 1
    for (int64_t at0 = (from & ~31) + 32 * (int64_t)nth; at0 <= to; at0 += 32 * step) {
        const int key0 = (int)at0, mine = key0 + lq < from ? from : key0 + lq < to ? key0 + lq : to;
        int ek = 0, ev = 0;
        const unsigned char *kr = K.row(mine, &ek), *vr = V.row(mine, &ev);
        const unsigned absent = (unsigned)__builtin_amdgcn_ballot_w64(kr == nullptr);
        if (kr == nullptr) {                                         // (not seen)
            kr = K.base;
            vr = V.base;
        }
        u32x2_t four[16];                                            // of the keys that a lane's sixteen slots stand for
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            const int at = 8 * (x >> 2) + (x & 3);
            four[x] = V.four(of_slot(vr, at), lq, SRC == PAGED_E4M3 ? of_slot(ev, at) : 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        f32x16_t s = {};
        asm volatile("" : "+v"(q));                                  // (the row is read in every unit: 32 registers)
#pragma unroll
        for (int ks = 0; ks < DH / 16; ++ks)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(K.eight(kr, 2 * ks + lh, ek), reinterpret_cast<const bf16x8_t *>(q)[2 * ks + lh], s, 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        unsigned seen = 0;                                           // of the lane's sixteen keys
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int at = 8 * (i >> 2) + 4 * lh + (i & 3), key = key0 + at;
            const bool sees = key >= first && key <= last && !(absent >> at & 1);
            seen |= (unsigned)sees << i;
            s[i] = sees ? s[i] * sl2 : -INFINITY;
            mx = fmaxf(mx, s[i]);
        }
        const float m_new = fmaxf(m, max_of_halves(mx)), alpha = exp2f(m - m_new);
        m = m_new;
        l *= alpha;
        bf16x8_t p[2];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            p[i >> 3][i & 7] = (__bf16)__builtin_amdgcn_exp2f(s[i] - m);
            l += (float)p[i >> 3][i & 7];
        }
#pragma unroll
        for (int d = 0; d < DH / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                acc[d][i] *= alpha;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            bf16x8_t v[DH / 32];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                put_pair(v, i, four[8 * c + 2 * i], four[8 * c + 2 * i + 1]);
            add_seen(acc, v, p[c], seen >> 8 * c);
        }
        if ((key0 & 0xE0) == 0) {                                    // now and then: does anything that follows matter?
            bool done = true;
#pragma unroll
            for (int d = 0; d < DH / 32; ++d)
                done = done && none_finite(acc[d]);
            if (__builtin_amdgcn_ballot_w64(wanted && !done) == 0)
                break;
        }
    }
    *max_score = m;
    *sum = sum_of_halves(l);
}

}  // namespace
}  // namespace cf
