// Attention of a chunk through a sliding window, with sinks, over a paged cache for 16-bit storage (TMA + tcgen05 + TMEM).
//
// As in the chunk attention without a window the G query heads of a K/V head and the chunk's tokens are folded into rows, a row
// tile ("stream") is 128/G tokens x G heads, and an item is a pair of row tiles, which share every K/V tile.  An item walks over
// the near slots of its rows (see Near) in tiles of 128: the sinks, and from the window of its first row on.
//
//   S = Q K^T -> TMEM;  P, rounded to the storage type, replaces its logits in TMEM and is the A operand of O += P V.
//   One thread has one row, so nothing is exchanged between threads, and each stream has four softmax warps and an issuing warp
//   of its own: while one stream waits for products the other's exponentials run.  P goes to the products in halves of 64 keys.
//   A row's reference (what is subtracted before the exponential) stays where it is unless a row sum shows that a probability
//   may have left fp16's range: then the half is done again against the row's maximum and the accumulator rescaled.  Until
//   a row has seen a slot its reference is unset, +inf.  A half of which no row of a warp sees anything costs it no exponential.
//
//   All items of a call are about as long as the window, so they are dealt in turn.  Where there are few, their tiles are one list, of
//   which every CTA takes an equal part, and a part that begins or ends inside an item leaves partial results that the merge kernel
//   joins.  The list is not written down: a CTA sums the lengths itself and finds its own place.
//
// What binds: one exponential per logit, 16 a clock and SM, and 128 x 128 x d x 4 operations of a tile at 8192 a clock: 2048 clocks
// each for a pair of tiles, d = 128, which takes 3,500 to 3,900: of 1,730 for half a tile of one stream 1,120 are its exponentials,
// which the other stream's slow down, 200 the wait for logits, the rest latencies between (S as one product of 128 columns, after all of
// P: 5,200).  The tensor pipe is active for 50 % of the time, the special-function unit for 49 % (2048 tokens, window 4096).  Long runs
// are held by the board's power: 156 us in the first 20 ms, 168 us at 1000 W and 1.6 GHz.  A CTA's first item waits 5,000 to 7,000
// clocks for its first logits, and an epilogue takes 5,000, most of it the first pass through its instructions, so code is kept short:
// short items are bound by these (8 prompts of 2048 and 125 to 265 tokens, window 512: 49 us, of which a CTA's 10 to 15 tiles take
// 20 to 27).
// P as one term of the storage type, as in the tcgen05 form without a window: a product is off by half a step at most, which adds to
// what rounding the output costs (error against 64 bits, of the output's norm: 2048 tokens, window 4096, bf16 1.69e-3 where rounding alone is
// 1.65e-3; 8 prompts, window 512, fp16 2.20e-4 and 2.04e-4).  A second term behind the first in tensor memory, as the forms for
// fewer rows have it, brings the error down to the rounding's and takes 167 -> 214 us and 51 -> 59.
#include <type_traits>

#include "paged_tc.cuh"

namespace a2sf {

A2SF_DEBUG_TRANSLATION_UNIT(paged_window_tc)

namespace {

using namespace paged_tc;

constexpr int kSms = 148;
constexpr int kThreads = 352;                // producer warp, an issuing warp and four softmax warps for each stream
constexpr int kFirstSoftmaxWarp = 3;
constexpr int kKStages = 3, kVStages = 2;
constexpr float kOptimisticLimit = 32768.f;  // a row sum below this keeps every probability < 2^15
constexpr float kRescaleThreshold = 8.0f;    // log2 units above the reference; beyond that limit one of 64 is 9 above
// A new reference lies so far below the row's maximum (log2 units): fp16 holds all bits of a probability down to 2^-14 and none below
// 2^-24, so with 8 these are 2^-22 and 2^-32 of the maximum, and 64 logits that all equal it have half of the limit.
template <typename T> constexpr float kBelow = std::is_same<T, __half>::value ? 8.f : 0.f;

// Division of the list, in tiles: what an item costs beside its own (set-up, epilogue), what cutting must gain, how near an end of an
// item a cut goes to that end instead, and what a part has at least.  The merge kernel takes the time of 3 to 4 tiles, but SMs that
// idle in the last round leave power to the others (us, cut and whole, in long runs under the power cap: 256 items of 35 tiles 178 and
// 168; 192 of 34: 119 and 150; 160 of 18: 67 and 85).
constexpr int kItemCost = 2, kMergeCost = 10, kSnap = 2;
constexpr int kMinPart = 6;                   // of the list
constexpr int kItemSlots = kItemCost * kBlk + kBlk / 2;      // with what rounding to whole tiles adds
constexpr int kCutBelow = 6 * kSms;          // items of a call (by its capacity) from which none is cut: the last round is short

struct Desc {                                // of the item that CTA k cuts and began: its pieces, 0 where there is none
    int b, h, pair, pieces;
};
struct WinWs {
    Desc *desc;           // [kSms]
    float2 *part_ml;      // [2 * kSms][2 * kBlk] reference, sum.  2k: the piece that begins an item, 2k + 1: one that continues it
    float *part_o;        // [2 * kSms][d/4][2 * kBlk][4]: a warp stores 32 rows' four columns as 512 bytes
    int pair_tokens;
    bool cut;             // whether items may be cut
};

// ---- the list of items ---------------------------------------------------------------------------------
__device__ __forceinline__ int pair_count(const SeqState &st, int pair_tokens) { return (st.len + pair_tokens - 1) / pair_tokens; }
__device__ __forceinline__ int pair_tiles(const PagedView &pv, const SeqState &st, int pair, int pair_tokens)
{
    const Near near = near_slots<true>(pv, st.past, pair * pair_tokens);
    return (near.past + min((pair + 1) * pair_tokens, st.len) + kBlk - 1) / kBlk;
}

// The list's lengths are estimates in slots, so that sums over a sequence's pairs are closed forms.  A pair whose window is full has
// C near slots, but for its place in a grain; the E pairs before have all slots up to their own last.
struct Lengths {
    long long past, full;        // full: C
    int pair_tokens, pairs, early, tail;                     // tail: tokens that the last pair lacks

    __device__ Lengths(const PagedView &pv, const SeqState &st, int pt) : past(st.past), full((long long)pt + pv.window - 1 + pv.sink_end + kGrain / 2), pair_tokens(pt)
    {
        pairs = pair_count(st, pt);
        const long long e = (full - 1 - past) / pt;
        early = full - 1 < past ? 0 : (int)min(e, (long long)pairs);
        tail = pairs * pt - st.len;
    }
    // of the first p pairs of one head
    __device__ long long sum(int p) const
    {
        const long long e = min(p, early);
        return e * past + pair_tokens * (e * (e + 1) / 2) + (p - e) * full + (long long)p * kItemSlots - (p == pairs ? tail : 0);
    }
};

// prefix[0 .. B] of the lengths of one head, and the number of its items, by the whole block
__device__ __forceinline__ void sum_lengths(long long *prefix, int *items, const PagedView &pv, int pair_tokens)
{
    for (int b = threadIdx.x; b < pv.B; b += blockDim.x) {
        const SeqState st = seq_state(pv, b);
        const Lengths x(pv, st, pair_tokens);
        prefix[b + 1] = st.len > 0 ? x.sum(x.pairs) : 0;
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        long long run = 0;
        int count = 0;
        for (int b0 = 0; b0 < pv.B; b0 += 32) {
            const int b = b0 + lane;
            long long incl = b < pv.B ? prefix[b + 1] : 0;
            if (b < pv.B) count += pair_count(seq_state(pv, b), pair_tokens);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long x = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += x;
            }
            if (b < pv.B) prefix[b + 1] = run + incl;
            run += __shfl_sync(0xffffffffu, incl, 31);
        }
        count = __reduce_add_sync(0xffffffffu, count);
        if (lane == 0) {
            prefix[0] = 0;
            *items = count;
        }
    }
    __syncthreads();
}

// Where a CTA's part begins: tile t of an item (t = its tiles: the next item).
struct Place {
    int b, h, pair, t;
    long long w, item;           // place in the list, and the item's
};

// Tile of the item that a cut `in` slots behind its place goes through.
__device__ __forceinline__ int tile_at(long long in) { return (int)((in - kItemSlots) >> 7); }
static_assert(kBlk == 128, "tile_at");

// The cut before part k of the list.
__device__ __forceinline__ Place cut_before(const long long *prefix, const PagedView &pv, int pair_tokens, int k, int parts)
{
    const long long total = pv.H * prefix[pv.B], w = total * k / parts;
    if (k >= parts) return Place{pv.B, 0, 0, 0, total, total};
    int lo = 0, hi = pv.B - 1;                               // last b with H * prefix[b] <= w
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (pv.H * prefix[mid] <= w) lo = mid;
        else hi = mid - 1;
    }
    const SeqState st = seq_state(pv, lo);
    const Lengths x(pv, st, pair_tokens);
    const long long rest = w - pv.H * prefix[lo], each = prefix[lo + 1] - prefix[lo];
    int h = (int)__fdividef((float)rest, (float)each);       // nearly
    while (h * each > rest) --h;
    while ((h + 1) * each <= rest) ++h;
    const long long at = rest - h * each;                    // among the head's items
    int p = 0, last = x.pairs - 1;                           // last pair with sum(p) <= at
    while (p < last) {
        const int mid = (p + last + 1) >> 1;
        if (x.sum(mid) <= at) p = mid;
        else last = mid - 1;
    }
    const long long in = at - x.sum(p), length = x.sum(p + 1) - x.sum(p);
    const int tiles = pair_tiles(pv, st, p, pair_tokens), t = tile_at(in);
    Place y = {lo, h, p, 0, w - in, w - in};
    if (t > kSnap) {
        const bool end = tiles - t <= kSnap;
        y.t = end ? tiles : t;
        y.w = end ? w - in + length : w;
    }
    return y;
}

struct Job {
    int b, h, pair, i0, past, used, skip;    // i0: the pair's first token; past, used in its near slots
    int tiles, t0, t1;                       // key tiles of the item, those of this piece
    int from[2], to[2];                      // ... of each stream: it sees nothing before and behind
};

// Walks over a CTA's items: its part of the list, or one of every gridDim, in rounds of alternating direction.
struct Walk {
    const PagedView &pv;
    Place end;
    int pair_tokens, tile_tokens, b, h, pair, t, pairs;
    SeqState st;
    bool more, inside, back;     // back: the next round runs backwards

    // whole items, dealt in turn
    __device__ Walk(const PagedView &v, int pt) : pv(v), end{}, pair_tokens(pt), tile_tokens(kBlk / v.G), b(-1), h(0), pair(0), t(0), inside(false), back(true)
    {
        sequence();
        skip(blockIdx.x);
    }
    // a part of the list
    __device__ Walk(const PagedView &v, int pt, const Place &at, const Place &e) : pv(v), end(e), pair_tokens(pt), tile_tokens(kBlk / v.G), b(at.b), h(at.h), pair(at.pair), t(at.t), more(at.w < e.w), inside(true), back(false)
    {
        st = b < pv.B ? seq_state(pv, b) : SeqState{0, 0};
        pairs = pair_count(st, pair_tokens);
        if (more && t >= pair_tiles(pv, st, pair, pair_tokens)) skip(1);
    }
    // the next sequence that has a part in the call, 32 at a time
    __device__ void sequence()
    {
        const int lane = threadIdx.x & 31;
        for (int b0 = b + 1; b0 < pv.B; b0 += 32) {
            SeqState s = {0, 0};
            if (b0 + lane < pv.B) s = seq_state(pv, b0 + lane);
            const unsigned any = __ballot_sync(0xffffffffu, s.len > 0);
            if (!any) continue;
            const int f = __ffs(any) - 1;
            b = b0 + f;
            st.past = __shfl_sync(0xffffffffu, s.past, f);
            st.len = __shfl_sync(0xffffffffu, s.len, f);
            pairs = pair_count(st, pair_tokens);
            more = true;
            return;
        }
        more = false;
    }
    // so many items on
    __device__ void skip(int items)
    {
        t = 0;
        unsigned at = (unsigned)h * pairs + pair + items;    // the launch sees to it that a call's items are a 31-bit number
        while (more && at >= (unsigned)pv.H * pairs) {
            at -= (unsigned)pv.H * pairs;
            sequence();
        }
        if (!more) return;
        h = (int)(at / (unsigned)pairs);
        pair = (int)at - h * pairs;
    }
    __device__ bool next(Job &j)
    {
        if (!more) return false;
        j.b = b; j.h = h; j.pair = pair;
        j.i0 = pair * pair_tokens;
        const Near near = near_slots<true>(pv, st.past, j.i0);
        j.past = near.past; j.used = near.past + st.len; j.skip = near.skip;
        const int tokens = min(pair_tokens, st.len - j.i0);
        j.tiles = (j.past + j.i0 + tokens + kBlk - 1) / kBlk;
        j.t0 = t;
        const bool last = inside && b == end.b && h == end.h && pair == end.pair;
        j.t1 = last ? min(j.tiles, end.t) : j.tiles;
        if (j.t1 <= t) {
            more = false;
            return false;
        }
        // stream 0 sees no slot beyond its own last token's; stream 1, where no sinks are, none before its first one's window
        const int end0 = (j.past + j.i0 + min(tokens, tile_tokens) + kBlk - 1) / kBlk;
        const int begin1 = pv.sinks ? 0 : max(0, j.past + j.i0 + tile_tokens + 1 - pv.window) / kBlk;
        j.from[0] = j.t0;
        j.to[0] = min(j.t1, end0);
        j.from[1] = max(j.t0, begin1);
        j.to[1] = tokens > tile_tokens ? j.t1 : 0;
        if (last) more = false;
        else      skip(inside ? 1 : back ? 2 * (int)(gridDim.x - blockIdx.x) - 1 : 2 * (int)blockIdx.x + 1);
        back = !back;
        return true;
    }
};

// ---- attn ------------------------------------------------------------------------------------------------
// What the other warps have to know of a job.
struct JobInfo {
    int t0, t1;                              // key tiles; t1 < 0: there are no more jobs
    int from[2], to[2];                      // of each stream
    int top, used, dead;                     // end of what the pair's first row sees, and of the sequence; no row sees sinks .. dead - 1
    int b, h, i0, part;                      // part: -1 for a whole item
};
constexpr int kJobs = 4;
constexpr int kJobReaders = 10;              // issuing and softmax warps

struct Shared {
    uint64_t q_full[2], q_empty[2], k_full[kKStages], k_empty[kKStages], v_full[kVStages], v_empty[kVStages];
    uint64_t s_full[2][2], p_full[2][2], o_done[2][2];      // per stream and half: logits, probabilities, products with values
    uint64_t job_full[kJobs], job_empty[kJobs];
    uint32_t tmem_base;
    int abort_flag, items, inside;
    Place cut[2];
    JobInfo jobs[kJobs];
};

template <int D> constexpr size_t smem_bytes() { return (size_t)Tile<D>::kBytes * (2 + kKStages + kVStages) + sizeof(Shared); }
static_assert(smem_bytes<128>() <= 227 * 1024, "shared memory");
static_assert((A2SF_PAGED_MAX_SEQUENCES + 1) * sizeof(long long) <= 2 * Tile<64>::kBytes, "the sums over the sequences stand in the queries' place");

// The wait for loads from tensor memory, with the registers that it is for: nothing that uses them moves before it.
__device__ __forceinline__ void tmem_wait_ld_of(uint32_t (&a)[32], uint32_t (&b)[32])
{
#define A2SF_R8(v, i) "+r"(v[i]), "+r"(v[i + 1]), "+r"(v[i + 2]), "+r"(v[i + 3]), "+r"(v[i + 4]), "+r"(v[i + 5]), "+r"(v[i + 6]), "+r"(v[i + 7])
    asm volatile("tcgen05.wait::ld.sync.aligned;" : A2SF_R8(a, 0), A2SF_R8(a, 8), A2SF_R8(a, 16), A2SF_R8(a, 24)::"memory");
    asm volatile("" : A2SF_R8(b, 0), A2SF_R8(b, 8), A2SF_R8(b, 16), A2SF_R8(b, 24)::"memory");
#undef A2SF_R8
}

__device__ __forceinline__ uint64_t twice(float x) { return pack_f32x2(__float_as_uint(x), __float_as_uint(x)); }

// Probabilities of 64 logits into tensor memory, packed, and their sum.
template <typename T>
__device__ __forceinline__ float probabilities(uint32_t dst, const uint32_t (&v)[2][32], uint64_t sl2x2, uint64_t nmx2)
{
    uint64_t rs2[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        uint32_t p[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            float x0, x1;
            unpack_f32x2(fma_f32x2(pack_f32x2(v[c][2 * e], v[c][2 * e + 1]), sl2x2, nmx2), x0, x1);
            const float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
            rs2[e & 3] = add_f32x2(rs2[e & 3], pack_f32x2(__float_as_uint(p0), __float_as_uint(p1)));
            p[e] = pack2<T>(p0, p1);
        }
        tmem_st16(dst + c * 16, p);
    }
    float a, b;
    unpack_f32x2(add_f32x2(add_f32x2(rs2[0], rs2[1]), add_f32x2(rs2[2], rs2[3])), a, b);
    return a + b;
}

// -inf for the logits whose bit is not set
__device__ __forceinline__ void mask(uint32_t (&v)[32], uint32_t bits)
{
#pragma unroll
    for (int x = 0; x < 32; ++x) v[x] = bits & (1u << x) ? v[x] : 0xff800000u;
}
// bits 0 .. n-1
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1; }

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1)
paged_window_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                       const __grid_constant__ CUtensorMap map_v, const __grid_constant__ AttendArgs a, const __grid_constant__ WinWs ws)
{
    constexpr int kTileBytes = Tile<D>::kBytes;
    constexpr int kFmt = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t *Qs = smem, *Ks = Qs + 2 * kTileBytes, *Vs = Ks + kKStages * kTileBytes;
    Shared *sh = reinterpret_cast<Shared *>(Vs + kVStages * kTileBytes);
    const PagedView &pv = a.pv;
    const int G = pv.G, tile_tokens = kBlk / G, tile_rows = tile_tokens * G;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &sh->abort_flag;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kKStages; ++s) { mbar_init(&sh->k_full[s], 1); mbar_init(&sh->k_empty[s], 2); }
        for (int s = 0; s < kVStages; ++s) { mbar_init(&sh->v_full[s], 1); mbar_init(&sh->v_empty[s], 2); }
        for (int s = 0; s < kJobs; ++s) { mbar_init(&sh->job_full[s], 1); mbar_init(&sh->job_empty[s], kJobReaders); }
        for (int x = 0; x < 2; ++x) {
            mbar_init(&sh->q_full[x], 1);
            mbar_init(&sh->q_empty[x], 1);
            for (int h = 0; h < 2; ++h) {
                mbar_init(&sh->s_full[x][h], 1);
                mbar_init(&sh->p_full[x][h], kBlk);
                mbar_init(&sh->o_done[x][h], 1);
            }
        }
        sh->abort_flag = smem_u32(smem) & 1023u ? 1 : 0;    // the swizzled tiles need this alignment
        sh->inside = 0;
        fence_mbar_init();
        prefetch_tmap(&map_q); prefetch_tmap(&map_k); prefetch_tmap(&map_v);
    }
    if (warp == 1) {
        tmem_alloc(&sh->tmem_base, 512);
        tmem_relinquish();
    }
    dependency_wait();
    if (ws.cut) {
        // the CTA's part of the list
        long long *prefix = reinterpret_cast<long long *>(smem);
        sum_lengths(prefix, &sh->items, pv, ws.pair_tokens);
        const long long total = pv.H * prefix[pv.B];
        const int parts = (int)max(1ll, min((long long)kSms, total / (kMinPart * kBlk)));
        const float n = (float)pv.H * (float)sh->items, mean = n > 0.f ? (float)total / n : 0.f;
        const bool inside = (float)total / parts + (kItemCost + kMergeCost) * kBlk < fminf(ceilf(n / kSms) * mean, (float)total / kSms + mean);
        if (inside && lane == 0 && warp < 2) sh->cut[warp] = cut_before(prefix, pv, ws.pair_tokens, blockIdx.x + warp, parts);
        __syncthreads();                                     // the sums have been read
        if (threadIdx.x == 0) {
            // The item that this part ends inside, if it began here: it goes on in the following parts whose own cuts lie inside it.
            Desc d = {0, 0, 0, 0};
            const Place end = sh->cut[1];
            if (inside && end.b < pv.B && end.t > 0 && end.item >= sh->cut[0].w) {
                const int tiles = pair_tiles(pv, seq_state(pv, end.b), end.pair, ws.pair_tokens);
                if (end.t < tiles) {
                    d = Desc{end.b, end.h, end.pair, 2};
                    for (int k = blockIdx.x + 2; k < parts && tiles - tile_at(total * k / parts - end.item) > kSnap; ++k) ++d.pieces;
                }
            }
            ws.desc[blockIdx.x] = d;
            sh->inside = inside;
        }
    }
    // rows that no query copy fills (G does not divide 128) are zero, so that their logits stay finite
    for (int x = threadIdx.x; x < 2 * Tile<D>::kHalves * (kBlk - tile_rows) * 8; x += kThreads) {
        const int piece = x & 7, row = tile_rows + (x >> 3) % (kBlk - tile_rows), half = (x >> 3) / (kBlk - tile_rows);
        *reinterpret_cast<uint4 *>(Qs + half * Tile<D>::kHalfBytes + row * 128 + piece * 16) = make_uint4(0, 0, 0, 0);
    }
    fence_async_smem();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    dependents_may_start();
    const uint32_t tmem_base = sh->tmem_base;

    // A failed wait poisons the CTA: later waits return at once, loops keep their shape.
    auto wait = [&](uint64_t *bar, uint32_t parity) -> bool {
        if (mbar_try_wait(bar, parity)) return true;
        if (*abort_flag) return false;
        return mbar_wait(bar, parity, abort_flag);
    };
    // For jobs: the next one is made known, and an old one's place free, only when the one before is done, which may be long.
    auto wait_job = [&](uint64_t *bar, uint32_t parity) -> bool {
        if (mbar_try_wait(bar, parity)) return true;
        if (*abort_flag) return false;
        return mbar_wait(bar, parity, abort_flag, 64 * kWaitCycles);
    };

    if (warp == 0) {
        // ---- TMA producer: lane i copies box i -----------------------------------------------------
        Walk walk = sh->inside ? Walk(pv, ws.pair_tokens, sh->cut[0], sh->cut[1]) : Walk(pv, ws.pair_tokens);
        Job j;
        int kt = 0, n[2] = {0, 0}, jobs = 0, ok = 1;        // tiles so far, items of each stream, items
        // tells the others; behind the last job that there is none
        auto publish = [&](bool any) {
            if (lane == 0) {
                const int slot = jobs % kJobs;
                ok = jobs < kJobs || wait_job(&sh->job_empty[slot], ((jobs / kJobs) & 1) ^ 1) ? 1 : 0;
                if (ok) {
                    JobInfo &x = sh->jobs[slot];
                    x.t1 = -1;
                    if (any) {
                        x.t0 = j.t0; x.t1 = j.t1;
                        x.from[0] = j.from[0]; x.from[1] = j.from[1]; x.to[0] = j.to[0]; x.to[1] = j.to[1];
                        x.top = j.past + j.i0 + 1; x.used = j.used; x.dead = max(0, x.top - pv.window);
                        x.b = j.b; x.h = j.h; x.i0 = j.i0;
                        x.part = j.t0 == 0 && j.t1 == j.tiles ? -1 : 2 * (int)blockIdx.x + (j.t0 > 0);
                    }
                    mbar_arrive(&sh->job_full[slot]);
                }
            }
            ok = __shfl_sync(0xffffffffu, ok, 0);
            ++jobs;
        };
        auto queries = [&](int X) {
            if (lane == 0) {
                ok = n[X] == 0 || wait(&sh->q_empty[X], (n[X] - 1) & 1) ? 1 : 0;
                if (ok) {
                    mbar_arrive_expect_tx(&sh->q_full[X], (uint32_t)(tile_rows * 128 * Tile<D>::kHalves));
                    copy_query_tile<D>(Qs + X * kTileBytes, &map_q, &sh->q_full[X], j.h * G, j.i0 + X * tile_tokens, j.b);
                }
            }
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (ok) ++n[X];
        };
        while (ok && walk.next(j)) {
            const int32_t *table = pv.table + (size_t)j.b * pv.max_pages;
            publish(true);
            if (ok && j.from[0] < j.to[0]) queries(0);
            for (int t = j.t0; ok && t < j.t1; ++t, ++kt) {
                const int ks = kt % kKStages, vs = kt % kVStages;
                const PageTile p = page_tile<true>(pv, t, j.used);
                const int slot = t * kBlk + lane * p.box;
                int row = 0;
                if (lane < p.boxes) {
                    const int real = real_slot<true>(pv, Near{0, j.skip, 0}, slot);
                    row = (int)pool_row(pv, page_for_read(pv, table, real), j.h, real);
                }
                const uint32_t bytes = (uint32_t)(p.boxes * p.box * 128 * Tile<D>::kHalves);
                if (lane == 0) {
                    if (kt >= kKStages) ok = wait(&sh->k_empty[ks], ((kt / kKStages) & 1) ^ 1) ? 1 : 0;
                    if (ok) mbar_arrive_expect_tx(&sh->k_full[ks], bytes);
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (!ok) break;
                copy_page_tile<D>(Ks + ks * kTileBytes, &map_k, &sh->k_full[ks], p, row);
                if (t == j.t0 && j.from[1] < j.to[1]) queries(1);
                if (ok && lane == 0) {
                    if (kt >= kVStages) ok = wait(&sh->v_empty[vs], ((kt / kVStages) & 1) ^ 1) ? 1 : 0;
                    if (ok) mbar_arrive_expect_tx(&sh->v_full[vs], bytes);
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (!ok) { ++kt; break; }                   // K of this tile is on its way
                copy_page_tile<D>(Vs + vs * kTileBytes, &map_v, &sh->v_full[vs], p, row);
            }
        }
        if (ok) publish(false);
        if (lane == 0 && *abort_flag) {
            // copies still in flight get a bounded chance to land before the CTA exits
            int dummy = 0;
            for (int k = max(0, kt - kKStages); k < kt; ++k) mbar_wait(&sh->k_full[k % kKStages], (k / kKStages) & 1, &dummy);
            for (int k = max(0, kt - kVStages); k < kt; ++k) mbar_wait(&sh->v_full[k % kVStages], (k / kVStages) & 1, &dummy);
            for (int X = 0; X < 2; ++X)
                if (n[X] > 0) mbar_wait(&sh->q_full[X], (n[X] - 1) & 1, &dummy);
        }
    } else if (warp < kFirstSoftmaxWarp) {
        // ---- MMA issuer of stream X (lane 0; the warp stays together to clear values that no row sees) ----
        const int X = warp - 1;
        const uint32_t idesc_qk = make_idesc(kFmt, kBlk, kBlk / 2, 0, 0);
        const uint32_t idesc_pv = make_idesc(kFmt, kBlk, D, 0, 1);        // V is MN-major
        // descriptors of the first buffers; the others lie whole tiles behind (16-byte units)
        const uint64_t step = kTileBytes >> 4;
        const uint64_t q_desc = kmajor_desc(smem_u32(Qs + X * kTileBytes)), k_desc = kmajor_desc(smem_u32(Ks));
        // V as an MN-major operand: 64-wide halves 16 KB apart, 8-key groups 1024 bytes apart
        const uint64_t v_desc = make_sdesc_sw128(smem_u32(Vs), Tile<D>::kHalfBytes, 1024);
        const uint32_t sp = tmem_base + X * 2 * kBlk, o = sp + kBlk;
        auto clear = [&](uint8_t *V, int r0, int r1) {
            for (int x = lane; x < Tile<D>::kHalves * (r1 - r0) * 8; x += 32) {
                const int piece = x & 7, row = r0 + (x >> 3) % (r1 - r0), half = (x >> 3) / (r1 - r0);
                *reinterpret_cast<uint4 *>(V + half * Tile<D>::kHalfBytes + row * 128 + piece * 16) = make_uint4(0, 0, 0, 0);
            }
            fence_async_smem();
            __syncwarp();
        };
        int kt = 0, n = 0, cnt = 0;                         // tiles of all, items and tiles of this stream
        for (int jobs = 0;; ++jobs) {
            const int slot = jobs % kJobs;
            if (__any_sync(0xffffffffu, !wait_job(&sh->job_full[slot], (jobs / kJobs) & 1))) break;
            const JobInfo &j = sh->jobs[slot];
            const int t0 = j.t0, t1 = j.t1, from = j.from[X], to = j.to[X], used = j.used, dead = j.dead;
            if (t1 < 0) break;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->job_empty[slot]);
            // half h of S of tile t: keys 64h .. 64h+63, in columns 64h .. (lane 0)
            auto logits = [&](int t, int k, int h) {
#pragma unroll
                for (int x = 0; x < D / 16; ++x) {
                    const uint64_t off = (uint64_t)(((x >> 2) * Tile<D>::kHalfBytes + (x & 3) * 32) >> 4);
                    umma_ss(sp + 64 * h, q_desc + off, k_desc + k % kKStages * step + off + (uint64_t)(h * 8192 >> 4), idesc_qk, x > 0);
                }
                umma_commit(&sh->s_full[X][h]);
                if (h == 1) {
                    umma_commit(&sh->k_empty[k % kKStages]);
                    if (t + 1 == to) umma_commit(&sh->q_empty[X]);
                }
            };
            for (int t = t0; t < t1; ++t, ++kt) {
                const int ks = kt % kKStages, vs = kt % kVStages;
                if (t < from || t >= to) {                  // the other stream's alone; once it is here, it has been waited for
                    wait(&sh->k_full[ks], (kt / kKStages) & 1);
                    if (lane == 0) mbar_arrive(&sh->k_empty[ks]);
                    wait(&sh->v_full[vs], (kt / kVStages) & 1);
                    if (lane == 0) mbar_arrive(&sh->v_empty[vs]);
                    __syncwarp();
                    continue;
                }
                if (t == from) {
                    wait(&sh->q_full[X], n++ & 1);
                    wait(&sh->k_full[ks], (kt / kKStages) & 1);
                    tc_fence_after_sync();
                    if (lane == 0) { logits(t, kt, 0); logits(t, kt, 1); }
                    __syncwarp();
                }
                const bool more = t + 1 < to;
                wait(&sh->v_full[vs], (kt / kVStages) & 1);
                if (more) wait(&sh->k_full[(kt + 1) % kKStages], ((kt + 1) / kKStages) & 1);
                // Slots behind the sequence, and those between the sinks and the window of the pair's first row, may hold
                // anything, NaN included: 0 * NaN must not reach O.  Both issuing warps write the same zeros.
                uint8_t *V = Vs + vs * kTileBytes;
                const int tile0 = t * kBlk, valid = used - tile0;
                if (valid < kBlk) clear(V, valid, kBlk);
                const int r0 = max(pv.sinks - tile0, 0), r1 = min(dead - tile0, kBlk);
                if (r0 < r1) clear(V, r0, r1);
                // 16 keys per step: 8 columns of packed P, two 8-key groups of V.  Keys 64h .. 64h+63 have their P at columns
                // 64h .. 64h+31, over logits that their threads have read; the next logits take its place behind the products.
                const uint64_t vd = v_desc + vs * step;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    wait(&sh->p_full[X][h], cnt & 1);
                    tc_fence_after_sync();
                    if (lane == 0) {
#pragma unroll
                        for (int k = 4 * h; k < 4 * h + 4; ++k)
                            umma_ts(o, sp + 64 * (k >> 2) + 8 * (k & 3), vd + (uint64_t)(k * 2048 >> 4), idesc_pv, t != from || k > 0);
                        // Before the next logits are asked for: who has seen those of a tile has then seen its predecessor's
                        // products end, and a wait for o_done cannot take the phase before for the one that it means.
                        umma_commit(&sh->o_done[X][h]);
                        if (more) logits(t + 1, kt + 1, h);
                        if (h == 1) umma_commit(&sh->v_empty[vs]);
                    }
                    __syncwarp();
                }
                ++cnt;
            }
        }
    } else {
        // ---- softmax + epilogue: a thread per row -------------------------------------------------------
        const int X = (warp - kFirstSoftmaxWarp) >> 2;
        const int quarter = warp & 3;                      // TMEM lanes this warp may touch
        const int r = quarter * 32 + lane;                 // row in the tile = TMEM lane
        const unsigned per = 65536u / G + 1;               // x / G = x * per >> 16 for a row x
        auto token_of = [&](int x) { return (int)(x * per >> 16); };
        const uint32_t sp0 = tmem_base + X * 2 * kBlk + ((uint32_t)(quarter * 32) << 16), to = sp0 + kBlk;
        int cnt = 0;                                        // tiles of this stream so far
        for (int jobs = 0;; ++jobs) {
            const int slot = jobs % kJobs;
            if (__any_sync(0xffffffffu, !wait_job(&sh->job_full[slot], (jobs / kJobs) & 1))) break;
            const JobInfo &j = sh->jobs[slot];
            if (j.t1 < 0) break;
            const int from = j.from[X], end = j.to[X], part = j.part;
            const int tok0 = X * tile_tokens;               // the stream's first token in the pair
            const bool live = r < tile_rows && j.top + tok0 + token_of(r) <= j.used;
            if (from >= end) {
                // a piece of the keys that holds nothing this stream sees: an empty partial result
                if (part >= 0) ws.part_ml[(size_t)part * 2 * kBlk + X * kBlk + r] = make_float2(-INFINITY, 0.f);
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh->job_empty[slot]);
                continue;
            }
            // near slots that the row sees: top - window .. top - 1 and the sinks; rows behind the chunk see what its last one does
            const int top = min(j.top + tok0 + token_of(r), j.used);
            const int top_first = __shfl_sync(0xffffffffu, top, 0), top_last = __shfl_sync(0xffffffffu, top, 31);
            float m = INFINITY, l = 0.f;
            bool set = false;                               // every row of the warp has a reference
            const uint64_t sl2x2 = twice(pv.sl2);
#pragma unroll 1
            for (int s0 = from * kBlk; s0 < end * kBlk; s0 += 64) {
                const int h = s0 >> 6 & 1;
                const uint32_t sp = sp0 + h * 64;
                wait(&sh->s_full[X][h], cnt & 1);
                tc_fence_after_sync();
                const bool unseen = s0 >= top_last || (s0 + 64 <= top_first - pv.window && s0 >= pv.sinks);      // by every row of the warp
                uint32_t v[2][32];
                float rowsum;
                if (__builtin_expect(unseen, 0)) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[0][e] = 0u;
                    tmem_st32(sp, v[0]);
                } else {
                    tmem_ld32(sp, v[0]);
                    tmem_ld32(sp + 32, v[1]);
                    tmem_wait_ld_of(v[0], v[1]);
                    if (__builtin_expect(s0 + 64 > top_first || s0 < top_last - pv.window, 0)) {
                        const int e1 = top - s0, e0 = e1 - pv.window, sinks = pv.sinks - s0;
                        mask(v[0], low_bits(e1) & (~low_bits(e0) | low_bits(sinks)));
                        mask(v[1], low_bits(e1 - 32) & (~low_bits(e0 - 32) | low_bits(sinks - 32)));
                    }
                    bool exact = !set;
                    if (__builtin_expect(set, 1)) {
                        rowsum = probabilities<T>(sp, v, sl2x2, twice(-m));
                        // rows behind the chunk hold anything: they must not decide when the others' references move
                        exact = __any_sync(0xffffffffu, live && !(rowsum <= kOptimisticLimit));      // also NaN
                    }
                    if (__builtin_expect(exact, 0)) {
                        float smax = __uint_as_float(v[0][0]), factor = 1.f;
#pragma unroll
                        for (int x = 1; x < 32; ++x) smax = fmaxf(smax, __uint_as_float(v[0][x]));
#pragma unroll
                        for (int x = 0; x < 32; ++x) smax = fmaxf(smax, __uint_as_float(v[1][x]));
                        bool grow = false;
                        if (m == INFINITY) {
                            if (smax != -INFINITY) m = __fmaf_ru(smax, pv.sl2, -kBelow<T>);      // what it has summed are zeros
                        } else if (fmaf(smax, pv.sl2, -m) > kRescaleThreshold) {
                            grow = true;
                            const float before = m;
                            m = __fmaf_ru(smax, pv.sl2, -kBelow<T>);
                            factor = ex2_approx(before - m);
                        }
                        if (__any_sync(0xffffffffu, grow)) {
                            // O holds all halves before: the last one's products are waited for
                            if (h == 1) wait(&sh->o_done[X][0], cnt & 1);
                            else        wait(&sh->o_done[X][1], (cnt - 1) & 1);
                            tc_fence_after_sync();
#pragma unroll 1
                            for (int c = 0; c < D / 32; ++c) {
                                uint32_t o[32];
                                tmem_ld32(to + c * 32, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int x = 0; x < 32; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * factor);
                                tmem_st32(to + c * 32, o);
                            }
                        }
                        set = !__any_sync(0xffffffffu, live && m == INFINITY);
                        l *= factor;
                        rowsum = probabilities<T>(sp, v, sl2x2, twice(-m));
                    }
                    l += rowsum;
                }
                tmem_wait_st();
                tc_fence_before_sync();
                mbar_arrive(&sh->p_full[X][h]);
                cnt += h;
            }
            // ---- epilogue: the row, normalised, or handed on.  The next products into O wait for the next P, which comes after.
            const float inv = 1.f / l;
            const bool done = wait(&sh->o_done[X][1], (cnt - 1) & 1);
            tc_fence_after_sync();
            if (part < 0) {
                // This lane stores piece lane & 3 of rows r0 .. r0 + 3
                T *orow[4];
                const int r0 = r & ~3;
                int tk = token_of(r0), gk = r0 - tk * G;
                tk += tok0;
                T *base = static_cast<T *>(a.out) + (int64_t)j.b * a.so.b + (lane & 3) * 8;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const bool in = r0 + k < tile_rows && j.top + tk <= j.used && done && A2SF_IN_RANGE(j.i0 + tk, pv.c, kDbgWindowTc);
                    orow[k] = in ? base + (int64_t)(j.h * G + gk) * a.so.h + (int64_t)(j.i0 + tk) * a.so.t : nullptr;
                    if (++gk == G) { gk = 0; ++tk; }
                }
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    tmem_ld32(to + c * 32, o);
                    tmem_wait_ld();
                    uint4 w[4];
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) {
                        uint32_t x[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = pack2<T>(__uint_as_float(o[q4 * 8 + 2 * e]) * inv, __uint_as_float(o[q4 * 8 + 2 * e + 1]) * inv);
                        w[q4] = make_uint4(x[0], x[1], x[2], x[3]);
                    }
                    transpose4(w);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (orow[k]) *reinterpret_cast<uint4 *>(orow[k] + c * 32) = w[k];
                }
                if (a.lse && live && done) a.lse[(((size_t)j.b * pv.H + j.h) * G + r - token_of(r) * G) * pv.c + j.i0 + tok0 + token_of(r)] = (m + log2f(l)) * 0.6931471805599453f;
            } else if (A2SF_IN_RANGE(part, 2 * kSms, kDbgWindowTc)) {
                float4 *po = reinterpret_cast<float4 *>(ws.part_o) + (size_t)part * (D / 4) * (2 * kBlk) + X * kBlk + r;
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    tmem_ld32(to + c * 32, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int q8 = 0; q8 < 8; ++q8)
                        if (live && done)
                            po[(c * 8 + q8) * 2 * kBlk] = make_float4(__uint_as_float(o[q8 * 4]), __uint_as_float(o[q8 * 4 + 1]), __uint_as_float(o[q8 * 4 + 2]),
                                                                      __uint_as_float(o[q8 * 4 + 3]));
                }
                if (live && done) ws.part_ml[(size_t)part * 2 * kBlk + X * kBlk + r] = make_float2(l > 0.f ? m : -INFINITY, l);
            }
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->job_empty[slot]);
        }
    }

    tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, 512);
    }
    if (threadIdx.x == 0 && sh->abort_flag) *pv.status = A2SF_ERR_TIMEOUT;
}

// ---- merge: a block per 32 rows of a cut item; lane = row, a warp takes every eighth group of four columns --------
constexpr int kMergeThreads = 256;
constexpr int kRowBlocks = 2 * kBlk / 32;

template <typename T, int D>
__global__ void __launch_bounds__(kMergeThreads)
paged_window_merge_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ WinWs ws)
{
    constexpr int NG = D / 4 / 8;                            // column groups of a warp
    constexpr int LD = D + 8;                                // halfwords of a staged row
    __shared__ __align__(16) T stage[32][LD];
    const PagedView &pv = a.pv;
    const int G = pv.G, tile_tokens = kBlk / G, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int k = blockIdx.x / kRowBlocks, pr0 = blockIdx.x % kRowBlocks * 32, pr = pr0 + lane;
    dependency_wait();
    dependents_may_start();
    const Desc d = ws.desc[k];
    if (d.pieces == 0) return;
    const SeqState st = seq_state(pv, d.b);
    auto token = [&](int row) {                              // of the chunk, or -1 for a row that is none
        const int X = row / kBlk, r = row - X * kBlk, tok = X * tile_tokens + r / G;
        const int i = d.pair * ws.pair_tokens + tok;
        return r < tile_tokens * G && i < st.len ? i : -1;
    };
    auto piece = [&](int s) { return (size_t)(s == 0 ? 2 * k : 2 * (k + s) + 1); };
    const int i = token(pr);
    if (!A2SF_IN_RANGE(k + d.pieces - 1, kSms, kDbgWindowTc)) return;
    // pieces that hold nothing the row sees have weight 0; what lies there is not used
    float mx = -INFINITY, l = 0.f;
    for (int s = 0; s < d.pieces; ++s) {
        const float2 ml = i >= 0 ? ws.part_ml[piece(s) * 2 * kBlk + pr] : make_float2(0.f, 0.f);
        mx = fmaxf(mx, ml.y > 0.f ? ml.x : -INFINITY);
    }
    float4 o[NG];
#pragma unroll
    for (int e = 0; e < NG; ++e) o[e] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
    for (int s = 0; s < d.pieces; ++s) {
        const float2 ml = i >= 0 ? ws.part_ml[piece(s) * 2 * kBlk + pr] : make_float2(0.f, 0.f);
        const float f = ml.y > 0.f ? exp2f(ml.x - mx) : 0.f;
        l = fmaf(f, ml.y, l);
        const float4 *src = reinterpret_cast<const float4 *>(ws.part_o) + piece(s) * (D / 4) * (2 * kBlk) + pr;
#pragma unroll
        for (int e = 0; e < NG; ++e) {
            const float4 v = f > 0.f ? src[(size_t)(warp + 8 * e) * (2 * kBlk)] : make_float4(0.f, 0.f, 0.f, 0.f);
            o[e].x = fmaf(f, v.x, o[e].x); o[e].y = fmaf(f, v.y, o[e].y);
            o[e].z = fmaf(f, v.z, o[e].z); o[e].w = fmaf(f, v.w, o[e].w);
        }
    }
    const float inv = 1.f / l;
#pragma unroll
    for (int e = 0; e < NG; ++e)
        *reinterpret_cast<uint2 *>(&stage[lane][(warp + 8 * e) * 4]) = make_uint2(pack2<T>(o[e].x * inv, o[e].y * inv), pack2<T>(o[e].z * inv, o[e].w * inv));
    if (warp == 0 && i >= 0 && a.lse) a.lse[(((size_t)d.b * pv.H + d.h) * G + (pr % kBlk) % G) * pv.c + i] = (mx + log2f(l)) * 0.6931471805599453f;
    __syncthreads();
    for (int e = threadIdx.x; e < 32 * (D / 8); e += kMergeThreads) {
        const int row = e / (D / 8), ch = e % (D / 8), ir = token(pr0 + row), g = ((pr0 + row) % kBlk) % G;
        if (ir >= 0)
            *reinterpret_cast<uint4 *>(static_cast<T *>(a.out) + (int64_t)d.b * a.so.b + (int64_t)(d.h * G + g) * a.so.h + (int64_t)ir * a.so.t + ch * 8) =
                *reinterpret_cast<const uint4 *>(&stage[row][ch * 8]);
    }
}

size_t pad(size_t x) { return (x + 255) / 256 * 256; }

WinWs carve(const PagedView &pv, void *mem, size_t *bytes)
{
    WinWs w;
    w.pair_tokens = 2 * (kBlk / pv.G);
    const long long items = (long long)pv.B * pv.H * ((pv.c + w.pair_tokens - 1) / w.pair_tokens);
    w.cut = items < kCutBelow;
    char *base = static_cast<char *>(mem);
    size_t off = 0;
    const size_t parts = w.cut ? 2 * kSms : 0;
    w.desc = reinterpret_cast<Desc *>(base + off); off += pad(kSms * sizeof(Desc));
    w.part_ml = reinterpret_cast<float2 *>(base + off); off += pad(parts * 2 * kBlk * 8);
    w.part_o = reinterpret_cast<float *>(base + off); off += pad(parts * 2 * kBlk * pv.d * 4);
    if (bytes) *bytes = off;
    return w;
}

template <typename T, int D>
cudaError_t launch(int dtype, const AttendArgs &a, cudaStream_t s)
{
    cudaError_t e = allow_dynamic_smem<paged_window_tc_kernel<T, D>>(smem_bytes<D>());
    if (e != cudaSuccess) return e;
    CUtensorMap mq, mk, mv;
    if (!make_query_map(&mq, dtype, a.q, a.pv, a.sq) || !make_pool_map(&mk, dtype, a.pv.k, a.pv, kGrain) ||
        !make_pool_map(&mv, dtype, a.pv.v, a.pv, kGrain))
        return cudaErrorInvalidValue;
    const WinWs ws = carve(a.pv, a.ws, nullptr);
    if ((long long)a.pv.B * a.pv.H * ((a.pv.c + ws.pair_tokens - 1) / ws.pair_tokens) > 0x7fffffff - 2 * kSms) return cudaErrorInvalidValue;
    if ((e = launch_chained(paged_window_tc_kernel<T, D>, kSms, kThreads, smem_bytes<D>(), s, mq, mk, mv, a, ws)) != cudaSuccess) return e;
    count_launch();
    if (!ws.cut) return cudaSuccess;
    if ((e = launch_chained(paged_window_merge_kernel<T, D>, kSms * kRowBlocks, kMergeThreads, 0, s, a, ws)) != cudaSuccess) return e;
    count_launch();
    return cudaSuccess;
}

}  // namespace

size_t window_tc_ws_bytes(const PagedView &pv)
{
    size_t bytes = 0;
    carve(pv, nullptr, &bytes);
    return bytes;
}

cudaError_t launch_window_tc(int dtype, const AttendArgs &a, cudaStream_t s)
{
    const bool wide = a.pv.d == 128;
    if (dtype == A2SF_BF16) return wide ? launch<__nv_bfloat16, 128>(dtype, a, s) : launch<__nv_bfloat16, 64>(dtype, a, s);
    return wide ? launch<__half, 128>(dtype, a, s) : launch<__half, 64>(dtype, a, s);
}

}  // namespace a2sf
