// A serving step's tables from the lengths of its requests: where each sequence's rows begin, how many tokens its cache holds, the pages that
// it takes from the stack of free ones (after what finished requests give back has been put onto it), each new token's position and slot.
//
// Bound by latency: some KB are read and written, each step needs sums over all sequences of what the one before made, and a trip to memory
// takes most of a microsecond.  So one workgroup does it all: it asks for all lengths at once, adds up in LDS, and takes a thread a page or token,
// found by a search over those sums.  A token whose page has just been taken looks at the stack, not at the table, so that no access waits for a
// store.  Tokens of more than ROWS_HERE are left to a second launch over all compute units.
// Measured (us): 64 decoding sequences 5.5 traced, 6.0 back to back; 512 with 24 prompts among them, 22 thousand tokens, 14.4 and 4.0 for the second launch, 17.6
// back to back.  Tried: searches by 64-ary steps of a wave 6.7 and 17.2, neighbouring pages and tokens on one thread 9.1 and 22.3, all of a thread's searches side by
// side without branches 7.3 and 23.2.
#include "decoder_internal.h"

namespace cf {
namespace {

constexpr int ROWS_HERE = 8192;

// Sums of whole numbers from 0 to 2^32 - 1, where they end.
__device__ __forceinline__ unsigned add(unsigned x, unsigned y) { return __builtin_elementwise_add_sat(x, y); }
__device__ __forceinline__ unsigned scan_wave(unsigned x)            // inclusive, over the lanes
{
#define FROM(control, rows) add(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, control, rows, 0xf, false))
    x = FROM(0x111, 0xf);                                            // from 1, 2, 4, 8 lanes below in a row of 16
    x = FROM(0x112, 0xf);
    x = FROM(0x114, 0xf);
    x = FROM(0x118, 0xf);
    x = FROM(0x142, 0xa);                                            // rows 1 and 3: the last lane of the row below
    x = FROM(0x143, 0xc);                                            // rows 2 and 3: lane 31
#undef FROM
    return x;
}

// How many of ends[0 .. n) (ascending) are <= t.
__device__ __forceinline__ int count_upto(const int *ends, int n, int t)
{
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (ends[mid] <= t)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int at_least_0(int x) { return x < 0 ? 0 : x; }
// Pages of a row of the table that `tokens` tokens take.
__device__ __forceinline__ int pages_upto(const TableParams &P, int64_t tokens)
{
    const int64_t p = (tokens + (1 << P.page_shift) - 1) >> P.page_shift;
    return (int)(p < P.max_pages ? p : P.max_pages);
}
__device__ __forceinline__ void put_token(const TableParams &P, int t, int64_t position, int page)
{
    const bool real = position >> P.page_shift < P.max_pages && (unsigned)page < (unsigned)P.n_pages;
    P.positions[t] = (int32_t)(position < INT32_MAX ? position : INT32_MAX);
    P.slots[t] = real ? ((int64_t)page << P.page_shift) + (position & ((1 << P.page_shift) - 1)) : -1;
}
__device__ __forceinline__ void put_padding(const TableParams &P, int t)
{
    P.positions[t] = 0;
    P.slots[t] = -1;
}

// CHUNKS sequences a thread at the most; AT_ONCE pages or tokens of a thread are on their way together.
template <int NT, int CHUNKS, int AT_ONCE>
__global__ __launch_bounds__(NT) void step_tables_kernel(TableParams P)
{
    constexpr int NW = NT / 64;
    __shared__ int a[NT * CHUNKS], b[NT * CHUNKS], had[NT * CHUNKS];
    static_assert(AT_ONCE * NW <= 64 && CHUNKS * NW <= 64, "what the waves count is a lane each");
    __shared__ unsigned wave_sums[2][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = P.n_seqs;
    int parity = 0;
    // Of what the waves left in wave_sums, `count` of them: sums up to every one, a lane each, and what comes before place `at`.  (Added up by every thread
    // for itself, sixteen waves' counts took a fifth of the time.)
    auto sums_upto = [&](int number) { return scan_wave(lane < number ? wave_sums[parity][lane] : 0); };
    auto before_of = [&](unsigned sums, int at) { return at > 0 ? (unsigned)__builtin_amdgcn_readlane((int)sums, at - 1) : 0u; };

    // The lengths, all asked for at once
    const bool backs = P.back_from != nullptr;
    int count = *P.free_count, held[CHUNKS], fresh[CHUNKS], from[CHUNKS], to[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int s = c * NT + tid;
        held[c] = fresh[c] = from[c] = to[c] = 0;
        if (s < n) {
            held[c] = P.held[s];
            fresh[c] = P.new_tokens[s];
            if (backs) {
                from[c] = P.back_from[s];
                to[c] = P.back_to[s];
            }
        }
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        held[c] = at_least_0(held[c]);
        fresh[c] = at_least_0(fresh[c]);
        from[c] = at_least_0(from[c]);
        to[c] = to[c] < P.max_pages ? to[c] : P.max_pages;
        had[c * NT + tid] = held[c];
    }
    count = count < 0 ? 0 : count < P.n_pages ? count : P.n_pages;

    // Inclusive sums of x over the sequences into `sums` and x, no more than `most`; their total.  (One barrier: buffers alternate.)
    auto add_up = [&](unsigned (&x)[CHUNKS], int *sums, unsigned most) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            x[c] = scan_wave(x[c]);
            if (lane == 63)
                wave_sums[parity][c * NW + wave] = x[c];
        }
        __syncthreads();
        const unsigned upto = sums_upto(CHUNKS * NW), total = before_of(upto, CHUNKS * NW);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const unsigned all = add(before_of(upto, c * NW + wave), x[c]);
            x[c] = all < most ? all : most;
            if (c * NT + tid < n)
                sums[c * NT + tid] = (int)x[c];
        }
        parity ^= 1;
        return (int)(total < most ? total : most);
    };

    // Pages that come back: entries [from, to) of each row that name a page, in the order of the batch.
    if (backs) {
        unsigned x[CHUNKS];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            x[c] = to[c] > from[c] ? to[c] - from[c] : 0;
            if (c * NT + tid < n)
                b[c * NT + tid] = from[c];
        }
        const int entries = add_up(x, a, INT32_MAX);
        __syncthreads();
        for (int64_t i0 = 0; i0 < entries; i0 += NT * AT_ONCE) {
            int page[AT_ONCE];
            int64_t at[AT_ONCE];
            unsigned long long real[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int64_t i = i0 + u * NT + tid;
                page[u] = -1;
                at[u] = 0;
                if (i < entries) {
                    const int s = count_upto(a, n, (int)i);
                    at[u] = (int64_t)s * P.max_pages + b[s] + (int)i - (s > 0 ? a[s - 1] : 0);
                    page[u] = P.page_table[at[u]];
                }
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                real[u] = __builtin_amdgcn_ballot_w64((unsigned)page[u] < (unsigned)P.n_pages);
                if (lane == 0)
                    wave_sums[parity][u * NW + wave] = __builtin_popcountll(real[u]);
            }
            __syncthreads();
            const unsigned upto = sums_upto(AT_ONCE * NW);
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int place = count + (int)before_of(upto, u * NW + wave) + __builtin_popcountll(real[u] & ((1ull << lane) - 1));
                if (real[u] >> lane & 1) {
                    if (place < P.n_pages)
                        P.free_pages[place] = page[u];
                    if (P.clear_back)
                        P.page_table[at[u]] = -1;
                }
            }
            const int all = count + (int)before_of(upto, AT_ONCE * NW);
            count = all < P.n_pages ? all : P.n_pages;
            parity ^= 1;
        }
        __syncthreads();                                             // the stack is written, and a and b are read
    }

    // Rows: sequence s has [a[s - 1], a[s]) of them, all together no more than there is room for.
    unsigned ends[CHUNKS], pages[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
        ends[c] = (unsigned)fresh[c];
    const int rows = add_up(ends, a, (unsigned)P.max_tokens);
    __syncthreads();
    // Pages that are taken: of sequence s [b[s - 1], b[s]) of all, in the order of the batch; number i is the i-th from the top of the stack.
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int s = c * NT + tid;
        pages[c] = 0;
        if (s < n) {
            const int64_t len = (int64_t)held[c] + ends[c] - (s > 0 ? a[s - 1] : 0);
            P.q_start[s + 1] = (int)ends[c];
            P.kv_len[s] = (int32_t)(len < INT32_MAX ? len : INT32_MAX);
            pages[c] = pages_upto(P, len) - pages_upto(P, held[c]);
        }
    }
    const int taken = add_up(pages, b, INT32_MAX);
    if (tid == 0) {
        P.q_start[0] = 0;
        *P.free_left = count - taken;
    }
    __syncthreads();
    auto from_stack = [&](int i) { return i < count ? P.free_pages[count - 1 - i] : -1; };
    for (int64_t i0 = 0; i0 < taken; i0 += NT * AT_ONCE) {
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int64_t i = i0 + u * NT + tid;
            if (i < taken) {
                const int page = from_stack((int)i), s = count_upto(b, n, (int)i);
                P.page_table[(int64_t)s * P.max_pages + pages_upto(P, had[s]) + (int)i - (s > 0 ? b[s - 1] : 0)] = page;
            }
        }
    }
    if (P.max_tokens > ROWS_HERE)
        return;
    for (int t0 = 0; t0 < P.max_tokens; t0 += NT * AT_ONCE) {
        int64_t position[AT_ONCE];
        int page[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int t = t0 + u * NT + tid;
            position[u] = page[u] = -1;
            if (t < rows) {
                const int s = count_upto(a, n, t), have = had[s], i_taken = pages_upto(P, have);
                position[u] = (int64_t)have + t - (s > 0 ? a[s - 1] : 0);
                const int64_t i = position[u] >> P.page_shift;
                if (i < P.max_pages)
                    page[u] = i < i_taken ? P.page_table[(int64_t)s * P.max_pages + i] : from_stack((s > 0 ? b[s - 1] : 0) + (int)i - i_taken);
            }
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int t = t0 + u * NT + tid;
            if (t < P.max_tokens) {
                if (position[u] >= 0)
                    put_token(P, t, position[u], page[u]);
                else
                    put_padding(P, t);
            }
        }
    }
}

// Tokens of a large step, from the finished table.
__global__ __launch_bounds__(256) void step_slots_kernel(TableParams P)
{
    __shared__ int ends[MAX_TABLE_SEQS];
    for (int s = threadIdx.x; s < P.n_seqs; s += 256)
        ends[s] = P.q_start[s + 1];
    __syncthreads();
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t >= P.max_tokens)
        return;
    const int s = count_upto(ends, P.n_seqs, t);
    if (s == P.n_seqs) {
        put_padding(P, t);
        return;
    }
    const int64_t position = (int64_t)at_least_0(P.held[s]) + t - (s > 0 ? ends[s - 1] : 0), i = position >> P.page_shift;
    put_token(P, t, position, i < P.max_pages ? P.page_table[(int64_t)s * P.max_pages + i] : -1);
}

}  // namespace

hipError_t launch_step_tables(const TableParams &p, hipStream_t s)
{
    // (a small batch's barriers are cheaper among four waves)
    if (p.n_seqs <= 256 && p.max_tokens <= 1024)
        hipLaunchKernelGGL((step_tables_kernel<256, 1, 1>), dim3(1), dim3(256), 0, s, p);
    else if (p.n_seqs <= 1024)
        hipLaunchKernelGGL((step_tables_kernel<1024, 1, 4>), dim3(1), dim3(1024), 0, s, p);
    else
        hipLaunchKernelGGL((step_tables_kernel<1024, MAX_TABLE_SEQS / 1024, 4>), dim3(1), dim3(1024), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.max_tokens <= ROWS_HERE)
        return e;
    hipLaunchKernelGGL(step_slots_kernel, dim3((unsigned)(((int64_t)p.max_tokens + 255) / 256)), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace cf
