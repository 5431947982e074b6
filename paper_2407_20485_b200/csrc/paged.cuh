// The cache in pages: what its kernels share (device view, page lookups, division of work).
#pragma once

#include <cuda.h>

#include "common.cuh"

namespace a2sf {

struct PagedView {
    char *k, *v;                 // [num_pages][H][ps][d] elements
    // Windowed attention uses neither scores nor positions, and the others no window: one place for both, since 16 bytes more of
    // arguments are 0.35 us more for every launch of the rotary kernel.
    union {
        struct {
            float *scores;       // [num_pages][H][ps]
            int32_t *positions;
        };
        struct {
            int window, sinks, sink_end;              // see Near; sink_end is sinks in whole grains
        };
    };
    const int32_t *table;        // [B][max_pages]
    const int32_t *past, *start; // [B]; start may be nullptr (past)
    const int32_t *lens;         // [B] or nullptr (c)
    int *status;                 // sticky status word of the paged kernels
    int B, H, G, d, ps, ps_shift, max_pages, num_pages, c;
    float sl2;                   // scale * log2(e)
};

struct SeqState {
    int past, len;               // slots before the chunk, new tokens
};

// Lengths live on the device: whatever they hold, past + len stays within the page table.
__device__ __forceinline__ SeqState seq_state(const PagedView &a, int b)
{
    SeqState s;
    const int cap = a.max_pages << a.ps_shift;
    s.past = a.past[b];
    s.len = a.lens ? min(a.lens[b], a.c) : a.c;
    if (s.past < 0 || s.len < 0 || s.past > cap - s.len) {
        *a.status = A2SF_ERR_INVALID_ARG;
        s.past = min(max(s.past, 0), cap);
        s.len = min(max(s.len, 0), cap - s.past);
    }
    return s;
}

// Page of slot `s` of sequence b for reading: a bad entry is reported and page 0 stands in.
__device__ __forceinline__ int page_for_read(const PagedView &a, const int32_t *row, int s)
{
    if (!A2SF_IN_RANGE(s >> a.ps_shift, a.max_pages, kDbgPagedRow)) return 0;
    const int p = row[s >> a.ps_shift];
    if ((unsigned)p < (unsigned)a.num_pages) return p;
    *a.status = A2SF_ERR_INVALID_ARG;
    return 0;
}
// ... and for writing: -1, and the write is left out.
__device__ __forceinline__ int page_for_write(const PagedView &a, const int32_t *row, int s)
{
    if (!A2SF_IN_RANGE(s >> a.ps_shift, a.max_pages, kDbgPagedRow)) return -1;
    const int p = row[s >> a.ps_shift];
    if ((unsigned)p < (unsigned)a.num_pages) return p;
    *a.status = A2SF_ERR_INVALID_ARG;
    return -1;
}
// Index of a slot's row within the pool (times d: its K and V row; alone: score and position).
__device__ __forceinline__ int64_t pool_row(const PagedView &a, int page, int h, int s)
{
    const int64_t row = (((int64_t)page * a.H + h) << a.ps_shift) + (s & ((1 << a.ps_shift) - 1));
    return A2SF_IN_RANGE(row, ((int64_t)a.num_pages * a.H) << a.ps_shift, kDbgPagedRow) && A2SF_IN_RANGE(h, a.H, kDbgPagedRow) ? row : 0;
}

// ---- windowed attention (template parameter Win): what is seen, as a list without a gap ----------------
// The row at slot p sees slots j < sinks and p - window < j <= p.  Of the rows from token i0 of the chunk on none sees a slot
// between the sinks and  lo = past + i0 + 1 - window.  So their slots are numbered along a list: the grains (16 slots of one
// page) that hold the sinks, then those from lo's on; `skip` slots, whole grains, lie between and are neither read nor looked up.
// In these numbers a row's place is past - skip + i, and the rule above holds as it stands: a slot of the sinks' grains is
// below every window if anything is skipped.  Without a window nothing is skipped, and near numbers are slots.
// A grain is also one box of a copy.  It is the smallest page, so that no page is smaller and least is read that nobody sees; larger ones would
// make fewer boxes and gain or lose little (us with 16, 32 and 64: one token, 32 heads, window 205: 6.5, 7.0, 6.9; 32 x 40 windows of 2048:
// 204, 202, 205; four tokens, window 4096: 29.3, 29.5, 29.5; 8 prompts, window 512: 51.4, 50.6, 51.7; 2048 tokens, window 4096: 167 all).
constexpr int kGrain = 16;

struct Near {
    int past, skip;              // near slots before the chunk; slots left out
    int dead;                    // near slots sinks .. dead-1 are seen by none of the rows: they may hold anything
};

template <bool Win> __device__ __forceinline__ Near near_slots(const PagedView &a, int past, int i0)
{
    Near n = {past, 0, 0};
    if (Win) {
        const int lo = max(0, past + i0 + 1 - a.window);
        n.skip = max(0, (lo & -kGrain) - a.sink_end);
        n.past = past - n.skip;
        n.dead = lo - n.skip;
    }
    return n;
}
template <bool Win> __device__ __forceinline__ int real_slot(const PagedView &a, const Near &n, int s)
{
    return Win && s >= a.sink_end ? s + n.skip : s;
}
// Rows of one TMA box: what lies together in a page and in the list.
template <bool Win> __device__ __forceinline__ int box_rows(const PagedView &a, int tile) { return min(Win ? kGrain : a.ps, tile); }

// Lengths of sequence b with past in near numbers, for all rows of the chunk.
template <bool Win> __device__ __forceinline__ SeqState near_state(const PagedView &a, int b, Near &n)
{
    SeqState s = seq_state(a, b);
    n = near_slots<Win>(a, s.past, 0);
    s.past = n.past;
    return s;
}

// Near slots that `rows` consecutive tokens can see at most (host): the capacity without a window.
__host__ inline int near_capacity(const PagedView &a, bool windowed, int rows)
{
    const long long cap = (long long)a.max_pages << a.ps_shift;
    if (!windowed) return (int)cap;
    const long long most = (long long)a.sink_end + a.window - 1 + rows + kGrain - 1;
    return (int)(most < cap ? most : cap);
}

// alpha^age in fp32, with 0^0 = 1 (nl2a = -log2 alpha, +inf for alpha = 0)
__device__ __forceinline__ float age_exponent(int age, float nl2a) { return age == 0 ? 0.f : (float)age * nl2a; }

__host__ inline float neg_log2(float alpha) { return alpha > 0.f ? -log2f(alpha) : INFINITY; }

// The reference (what is subtracted before the exponential, log2 units) of a row whose largest logit is `mx`: kBelow under it, but
// nowhere by more than 15 -- large logits round the difference -- so that fp16 holds the largest probability.
template <int kBelow> __device__ __forceinline__ float reference(float mx)
{
    if (kBelow == 0) return mx;
    const float m = mx - (float)kBelow;
    return mx - m <= 15.f ? m : mx;                      // -inf stays -inf
}

// First row (token of the chunk) whose weight alpha^(len-1-i) is not below 2^-126, the smallest normal
// fp32 number: a probability is at most 1, and the exponential of what lies below is flushed to zero.
__device__ __forceinline__ int first_weighted_token(int len, float nl2a)
{
    if (!(nl2a > 0.f)) return 0;
    const float span = 126.f / nl2a;
    return span >= (float)len ? 0 : max(0, len - 1 - (int)span);
}

// ---- the tiles of all (sequence, K/V head) units as one list ---------------------------------------
struct Where {            // position in the list: unit (b, h), tile t of its `tiles`
    int b, h, t, tiles;
};

// Tiles of one head of sequence b; none where it takes no part in the call.
template <int Tile, bool Win = false> __device__ __forceinline__ int seq_tiles(const PagedView &pv, int b)
{
    Near near;
    const SeqState st = near_state<Win>(pv, b, near);
    return st.len > 0 ? (st.past + st.len + Tile - 1) / Tile : 0;
}

// prefix[0 .. B] of the sequences' tiles, by one warp
template <int Tile, bool Win = false> __device__ __forceinline__ void tile_prefix(int32_t *prefix, const PagedView &pv)
{
    const int lane = threadIdx.x & 31;
    int run = 0;
    for (int b0 = 0; b0 < pv.B; b0 += 32) {
        const int b = b0 + lane;
        int incl = b < pv.B ? seq_tiles<Tile, Win>(pv, b) : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        if (b < pv.B) prefix[b + 1] = run + incl;
        run += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) prefix[0] = 0;
}

__device__ __forceinline__ Where locate(const int32_t *prefix, int B, int H, long long w)
{
    int lo = 0, hi = B - 1;                        // last b with H * prefix[b] <= w
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((long long)H * prefix[mid] <= w) lo = mid;
        else hi = mid - 1;
    }
    Where x;
    x.b = lo;
    x.tiles = prefix[lo + 1] - prefix[lo];
    const long long rest = w - (long long)H * prefix[lo];
    x.h = (int)(rest / x.tiles);
    x.t = (int)(rest - (long long)x.h * x.tiles);
    return x;
}

__device__ __forceinline__ void next_unit(Where &x, const int32_t *prefix, int B, int H)
{
    x.t = 0;
    if (++x.h < H) return;
    x.h = 0;
    do ++x.b; while (x.b < B && prefix[x.b + 1] == prefix[x.b]);
    x.tiles = x.b < B ? prefix[x.b + 1] - prefix[x.b] : 0;
}

// ---- kernels of one call follow each other by programmatic launch ----------------------------------
// A kernel is resident, its barriers and descriptors set up, while its predecessor drains; it waits
// with dependency_wait() before it touches anything that any earlier kernel wrote.  Every kernel waits, and
// lets its followers start only after that, so behind a kernel that has waited lie all its predecessors, not
// only the last one.  The first kernel of a call waits before it reads anything (what runs before it in the
// stream may be anybody's); the following ones may read what no kernel of the call writes without waiting.
__device__ __forceinline__ void dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void dependents_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename... Params, typename... Args>
cudaError_t launch_clusters(void (*kernel)(Params...), unsigned grid, unsigned cluster, unsigned threads, size_t smem, cudaStream_t s, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}
template <typename... Params, typename... Args>
cudaError_t launch_chained(void (*kernel)(Params...), unsigned grid, unsigned threads, size_t smem, cudaStream_t s, Args... args)
{
    return launch_clusters(kernel, grid, 1, threads, smem, s, args...);
}

// ---- launchers -------------------------------------------------------------------------------
int *paged_status_word();        // device address on the current device (nullptr on failure)
int read_and_clear_paged_status(cudaStream_t s);

struct RotaryArgs {
    // heads [0, Hq): x -> y rotated; then (append) Hk keys rotated into pages and Hk values copied
    const void *x, *k, *v;
    void *y;
    Strides sx, sy, skv;
    const int32_t *positions;    // [B][n] or nullptr; with several axes [axes][B][n]
    const int32_t *start;        // [B] or nullptr (0, or past in append)
    const int32_t *lens;
    int B, n, d, Hq, Hk, transpose;
};
cudaError_t launch_rotary(int dtype, const a2sf_rotary_plan *plan, const RotaryArgs &r, const PagedView *pages,
                          cudaStream_t s);

cudaError_t launch_rotary_axes(int dtype, const a2sf_rotary_axes_plan *plan, const RotaryArgs &r, const PagedView *pages,
                               cudaStream_t s);

struct AttendArgs {
    PagedView pv;
    const void *q;
    void *out;
    float *lse;                  // [B][H*G][c] or nullptr
    Strides sq, so;
    float alpha, nl2a;           // nl2a = -log2(alpha)
    bool scores, windowed;
    void *ws;
};
// Tensor map of a pool: rows of d elements, boxes of 128 bytes x box_rows rows, 128-byte swizzle.
bool make_pool_map(CUtensorMap *map, int dtype, const void *pool, const PagedView &pv, int box_rows);

// few rows (len * G <= kFewRows): the cache is read once, split evenly over the device
constexpr int kFewRows = 16;
size_t attend_few_ws_bytes(int dtype, const PagedView &pv, bool windowed);
cudaError_t launch_attend_few(int dtype, const AttendArgs &a, cudaStream_t s);

// many rows, 16-bit storage: tcgen05
bool make_query_map(CUtensorMap *map, int dtype, const void *q, const PagedView &pv, const Strides &st);
size_t attend_tc_ws_bytes(const PagedView &pv);
cudaError_t launch_attend_tc(int dtype, const AttendArgs &a, cudaStream_t s);
size_t window_tc_ws_bytes(const PagedView &pv);               // windowed
cudaError_t launch_window_tc(int dtype, const AttendArgs &a, cudaStream_t s);

// 32-bit storage, and small calls of 16-bit storage
size_t attend_mma_ws_bytes(int dtype, const PagedView &pv, bool windowed);
cudaError_t launch_attend_mma(int dtype, const AttendArgs &a, cudaStream_t s);

cudaError_t launch_evict(int elem_bytes, const PagedView &pv, int budget, int recent, const int32_t *dst_table,
                         int dst_max_pages, int32_t *past_out, int32_t *start_out, void *ws, cudaStream_t s);
size_t evict_ws_bytes(size_t units, int budget);

struct SlideArgs {
    int32_t *table_out, *freed, *freed_count, *past_out, *start_out;      // freed, freed_count may be nullptr
    int window, sinks;
};
cudaError_t launch_slide(const PagedView &pv, const SlideArgs &a, cudaStream_t s);

}  // namespace a2sf
