// The end of a step over a cache whose attention is windowed: past and start move on, and pages that no later row sees leave
// the page table.
//
// The next row stands at slot n = past + len and sees slots 0 .. sinks - 1 and those from n - window + 1 on, later rows no
// earlier ones: page e leaves where sinks <= e ps and (e + 1) ps <= n - window + 1.  The pages that left are listed in the
// order of their entries: a warp's ballot gives an entry its place among 32, sums over the warps before the rest.
//
// A block per sequence.  A table is a few kilobytes, so all of it is latency: one round of loads, one barrier, one round of
// stores (32 tables of 129 pages 3.2 us, 256 tables of 2,048 pages 3.7 us a call from Python: the launch rate).
#include "paged.cuh"

namespace a2sf {

A2SF_DEBUG_TRANSLATION_UNIT(paged_slide)

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kEntries = 4;                  // of a thread and round

__global__ void __launch_bounds__(kThreads)
paged_slide_kernel(const __grid_constant__ PagedView pv, const __grid_constant__ SlideArgs a)
{
    __shared__ int counts[2][kEntries * kWarps];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, b = blockIdx.x;
    dependency_wait();
    dependents_may_start();
    const SeqState st = seq_state(pv, b);
    const int start = pv.start ? pv.start[b] : st.past;
    const int32_t *table = pv.table + (size_t)b * pv.max_pages;
    int32_t *out = a.table_out + (size_t)b * pv.max_pages;
    int32_t *freed = a.freed ? a.freed + (size_t)b * pv.max_pages : nullptr;
    const int n = st.past + st.len;
    const int first = (a.sinks + pv.ps - 1) >> pv.ps_shift, end = max(0, n - a.window + 1) >> pv.ps_shift;
    // in place, only the entries that may leave are touched
    const bool whole = a.table_out != pv.table;
    const int e0 = whole ? 0 : first, e1 = whole ? pv.max_pages : end;
    int listed = 0;
    for (int base = e0, round = 0; base < e1; base += kThreads * kEntries, ++round) {
        int page[kEntries];
        unsigned before[kEntries];
        bool gone[kEntries];
#pragma unroll
        for (int x = 0; x < kEntries; ++x) {
            const int e = base + x * kThreads + tid;
            page[x] = e < e1 && A2SF_IN_RANGE(e, pv.max_pages, kDbgPagedSlide) ? table[e] : -1;
        }
#pragma unroll
        for (int x = 0; x < kEntries; ++x) {
            const int e = base + x * kThreads + tid;
            const bool leaves = e >= first && e < end && page[x] >= 0;
            gone[x] = leaves && page[x] < pv.num_pages;
            if (leaves && !gone[x]) *pv.status = A2SF_ERR_INVALID_ARG;       // no page: it leaves the table unlisted
            if (e < e1 && (whole || leaves)) out[e] = leaves ? -1 : page[x];
            const unsigned all = __ballot_sync(0xffffffffu, gone[x]);
            before[x] = __popc(all & ((1u << lane) - 1));
            if (lane == 0) counts[round & 1][x * kWarps + warp] = __popc(all);
        }
        __syncthreads();
        // the sums over all warps before: 64 counts, two a lane, in every warp
        const int c0 = counts[round & 1][2 * lane], c1 = counts[round & 1][2 * lane + 1];
        int incl = c0 + c1;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
#pragma unroll
        for (int x = 0; x < kEntries; ++x) {
            const int k = x * kWarps + warp;
            const int upto = __shfl_sync(0xffffffffu, incl, k >> 1), odd = __shfl_sync(0xffffffffu, c1, k >> 1), even = __shfl_sync(0xffffffffu, c0, k >> 1);
            const int at = listed + upto - odd - (k & 1 ? 0 : even) + (int)before[x];
            if (freed && gone[x] && A2SF_IN_RANGE(at, pv.max_pages, kDbgPagedSlide)) freed[at] = page[x];
        }
        listed += __shfl_sync(0xffffffffu, incl, 31);
    }
    __syncthreads();                                        // past and start have been read
    if (tid == 0) {
        if (a.freed_count) a.freed_count[b] = listed;
        a.past_out[b] = n;
        a.start_out[b] = start + st.len;
    }
}

}  // namespace

cudaError_t launch_slide(const PagedView &pv, const SlideArgs &a, cudaStream_t s)
{
    static_assert(kEntries * kWarps == 64, "two counts a lane");
    const cudaError_t e = launch_chained(paged_slide_kernel, (unsigned)pv.B, kThreads, 0, s, pv, a);
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace a2sf
