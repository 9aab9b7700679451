// A serving step's tables from the lengths of its requests: where each sequence's rows begin, how many tokens its cache holds, the pages that
// it takes from the stack of free ones (after what finished requests give back has been put onto it), each new token's position and slot.
//
// Bound by latency: some KB are read and written, each step needs sums over all sequences of what the one before made, and the first access to
// memory of a chain costs about a microsecond.  So one workgroup does it all, with the sums over sequences in LDS and a thread a page (or token),
// found by a search over those sums.  Tokens of more than ROWS_HERE are left to a second launch over all compute units.
#include "decoder_internal.h"

namespace cf {
namespace {

constexpr int NT = 1024, NW = NT / 64;
constexpr int ROWS_HERE = 8 * NT;

// How many of ends[0 .. n) (ascending) are <= t.
template <typename P>
__device__ __forceinline__ int count_upto(P ends, int n, int t)
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

// Token t's position and slot; `ends`: starts[1 ..] of the sequences.
template <typename E>
__device__ __forceinline__ void token_slot(const TableParams &P, E ends, int t)
{
    const int seq = count_upto(ends, P.n_seqs, t);
    int64_t slot = -1, position = 0;
    if (seq < P.n_seqs) {
        position = (int64_t)at_least_0(P.held[seq]) + t - (seq > 0 ? ends[seq - 1] : 0);
        const int64_t i = position >> P.page_shift;
        if (i < P.max_pages) {
            const int page = P.page_table[(int64_t)seq * P.max_pages + i];
            if ((unsigned)page < (unsigned)P.n_pages)
                slot = ((int64_t)page << P.page_shift) + (position & ((1 << P.page_shift) - 1));
        }
    }
    P.positions[t] = (int32_t)(position < INT32_MAX ? position : INT32_MAX);
    P.slots[t] = slot;
}

__global__ __launch_bounds__(NT) void step_tables_kernel(TableParams P)
{
    __shared__ int a[MAX_TABLE_SEQS], b[MAX_TABLE_SEQS], wave_sums[2][NW];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = P.n_seqs;

    // Inclusive sums of value(s) over the sequences into `to`, no more than `most`; their total.
    auto sums_of = [&](int *to, int64_t most, auto value) {
        int64_t base = 0;
        for (int s0 = 0; s0 < n; s0 += NT) {
            const int s = s0 + tid;
            // (each value is cut off at `most`, so that the sums of 64 of them fit 64 bits, and of what is left 31)
            int64_t x = s < n ? value(s) : 0;
            x = x < most ? x : most;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int64_t y = __shfl_up((long long)x, d);
                x += lane >= d ? y : 0;
            }
            x = x < most ? x : most;
            if (lane == 63)
                wave_sums[0][wave] = (int)x;
            __syncthreads();
            int64_t before = base, all = base;
            for (int w = 0; w < NW; ++w) {
                before += w < wave ? wave_sums[0][w] : 0;
                all += wave_sums[0][w];
            }
            const int64_t mine = before + x;
            if (s < n)
                to[s] = (int)(mine < most ? mine : most);
            base = all < most ? all : most;
            __syncthreads();
        }
        return (int)base;
    };

    int count = *P.free_count;
    count = count < 0 ? 0 : count < P.n_pages ? count : P.n_pages;
    // Pages that come back: entries [from, to) of each row that name a page, in the order of the batch.
    if (P.back_from != nullptr) {
        auto from_of = [&](int s) { return at_least_0(P.back_from[s]); };
        const int entries = sums_of(a, INT32_MAX, [&](int s) {
            const int from = from_of(s), to = P.back_to[s] < P.max_pages ? P.back_to[s] : P.max_pages;
            return to > from ? to - from : 0;
        });
        for (int64_t i0 = 0; i0 < entries; i0 += NT) {
            const int64_t i = i0 + tid;
            int page = -1;
            if (i < entries) {
                const int s = count_upto(a, n, (int)i);
                page = P.page_table[(int64_t)s * P.max_pages + from_of(s) + (int)i - (s > 0 ? a[s - 1] : 0)];
            }
            const bool real = (unsigned)page < (unsigned)P.n_pages;
            const unsigned long long all = __builtin_amdgcn_ballot_w64(real);
            int *sums = wave_sums[i0 / NT & 1];
            if (lane == 0)
                sums[wave] = __builtin_popcountll(all);
            __syncthreads();                                         // (the other half is written before the next one of these)
            int before = __builtin_popcountll(all & ((1ull << lane) - 1)), total = 0;
            for (int w = 0; w < NW; ++w) {
                before += w < wave ? sums[w] : 0;
                total += sums[w];
            }
            if (real && count + before < P.n_pages)
                P.free_pages[count + before] = page;
            count = count + total < P.n_pages ? count + total : P.n_pages;
        }
        __syncthreads();
    }

    // Rows: sequence s has [start, a[s]) of them, all together no more than there is room for.
    const int rows = sums_of(a, P.max_tokens, [&](int s) { return at_least_0(P.new_tokens[s]); });
    __syncthreads();
    auto rows_of = [&](int s) { return a[s] - (s > 0 ? a[s - 1] : 0); };
    const int mask = (1 << P.page_shift) - 1;
    auto pages_upto = [&](int64_t tokens) {                          // of a row of the table
        const int64_t p = (tokens + mask) >> P.page_shift;
        return (int)(p < P.max_pages ? p : P.max_pages);
    };
    for (int s = tid; s < n; s += NT) {
        const int64_t len = (int64_t)at_least_0(P.held[s]) + rows_of(s);
        P.q_start[s + 1] = a[s];
        P.kv_len[s] = (int32_t)(len < INT32_MAX ? len : INT32_MAX);
    }
    if (tid == 0)
        P.q_start[0] = 0;

    // Pages that are taken: number i of all, in the order of the batch, is the i-th from the top of the stack.
    const int taken = sums_of(b, INT32_MAX, [&](int s) {
        const int held = at_least_0(P.held[s]);
        return pages_upto((int64_t)held + rows_of(s)) - pages_upto(held);
    });
    __syncthreads();
    for (int64_t i = tid; i < taken; i += NT) {
        const int s = count_upto(b, n, (int)i);
        const int entry = pages_upto(at_least_0(P.held[s])) + (int)i - (s > 0 ? b[s - 1] : 0);
        P.page_table[(int64_t)s * P.max_pages + entry] = i < count ? P.free_pages[count - 1 - (int)i] : -1;
    }
    if (tid == 0)
        *P.free_left = count - taken;
    if (P.max_tokens > ROWS_HERE)
        return;
    __syncthreads();                                                 // the table's new entries are written
    for (int t = tid; t < P.max_tokens; t += NT)
        token_slot(P, (const int *)a, t);
}

__global__ __launch_bounds__(256) void step_slots_kernel(TableParams P)
{
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t < P.max_tokens)
        token_slot(P, (const int32_t *)P.q_start + 1, t);
}

}  // namespace

hipError_t launch_step_tables(const TableParams &p, hipStream_t s)
{
    hipLaunchKernelGGL(step_tables_kernel, dim3(1), dim3(NT), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.max_tokens <= ROWS_HERE)
        return e;
    hipLaunchKernelGGL(step_slots_kernel, dim3((unsigned)(((int64_t)p.max_tokens + 255) / 256)), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace cf
