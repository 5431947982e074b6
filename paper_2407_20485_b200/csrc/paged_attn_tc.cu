// Attention of a chunk over a paged cache for 16-bit storage (TMA + tcgen05 + TMEM).
//
// The G query heads of a K/V head and the chunk's tokens are folded into rows: a row tile is
// 128/G tokens x G heads (128 rows, or a few less when G does not divide 128), so K and V are read once
// for the whole group and the mask is a bound on the slot that grows with the row.
//
//   plan    one CTA, from the lengths on the device: an item is a pair of row tiles of one (sequence, K/V
//           head) and the key tiles it sees.  When there are too few items for the device's SMs (a short
//           chunk behind a long cache) items are cut along the keys.  Sorted, longest first.
//   attn    persistent CTAs take items in that order.  Two row tiles ("streams") share every K/V tile and
//           take turns: while one's rows are in the softmax warps, the other's products run.
//             S = Q K^T -> TMEM;  P, rounded to the storage type, replaces its logits in TMEM and is the A
//             operand of O += P V;  V is read MN-major from its TMA tile.
//           A row's reference (what is subtracted before the exponential) stays where it is unless a
//           row sum shows that a probability may have left fp16's range: then the tile is done again
//           against the row's maximum and the accumulator rescaled.  (fp16: against 2^8 less, see kBelow.)
//   merge   joins the items that were cut.
//   score   S_j <- alpha^len S_j + sum_r exp2(s_rj - c_r), c_r = lse_r + age * (-log2 alpha): K tile x Q
//           tiles transposed, so a slot is a TMEM lane and its sum is made by two threads in row order.
//           Rows whose weight is below fp32's normal numbers are not visited (alpha = 0.9: all but the last
//           830 tokens).  The (key tile, row tile) pairs of the call are one list, cut into equal shares; a
//           key tile that a cut goes through is summed in parts, which the join kernel adds in order.
//
// What binds: one exponential per logit in attn and one in score, 16 a clock and SM, and 128 x 128 x d x 4
// operations of a tile at 8192 a clock, 1024 clocks each for d = 128.  They overlap in part: the special-function unit runs at
// 45 % of its rate in attn and at 53 % in score, the tensor pipe at 41 % and 21 %, and neither is full (a chunk of 2048 tokens
// behind 14,336, 8 heads, bf16); a pair of tiles takes 2.2 to 2.3 us.
// P as one term of the storage type: every product is off by at most half a step, the output by that of sum P |V|.  Two terms,
// as in the other forms, would cost 1,612 -> 2,022 us for the chunk behind 30,720 slots and 138 -> 155 us for ragged prompts
// (half as many products again, and twice the packing), and leave the error against 64 bits, which is the output's rounding for
// the most part, at 1.7e-3 of the outputs' norm (bf16) and at 2.0e-4 where one term has 2.2e-4 (fp16).
#include <type_traits>

#include "paged_tc.cuh"

namespace a2sf {

A2SF_DEBUG_TRANSLATION_UNIT(paged_attn_tc)

namespace {

using namespace paged_tc;

constexpr int kSms = 148;
constexpr int kSplitBelow = 4 * kSms;        // items of a call from which none is cut
constexpr int kPieces = 4 * kSms;            // pieces that cutting makes at most, next to one per item
constexpr int kMinPiece = 4;                 // key tiles of a piece at least
// Sequences of at most so many key tiles need no plan: no item is long, so none is cut.  Such a call is attn and score alone (12 heads, 244 tokens: 27 us with plan, merge and join, 16 us without).
constexpr int kDirectTiles = 8;
// Up to so many row tiles a key tile's sum is left whole: at most 5 us for one CTA, what the join kernel costs.
constexpr int kWholeRows = 4;
constexpr int kMaxParts = kSplitBelow + kPieces;   // sum of ceil(T / piece) <= total / piece + items
constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;
constexpr int kCandidates = 32;
constexpr int kPlanCache = 4096;             // items whose length fits in the plan's shared memory
constexpr int kLevels = 8;                   // the list is sorted by length in this many steps
constexpr int kItemCost = 3;                 // what an item costs beside its tiles (set-up, epilogue), in tiles
constexpr int kScoreCtas = 2 * kSms;

struct Item {                                // of one head; all heads have the same
    int b, pair, t0, t1;                     // key tiles t0 .. t1-1
    int part;                                // -1: whole; else index of its partial result
    int past, len, pad;                      // of its sequence
};
struct Merge {
    int b, pair, n, part;                    // partial results part .. part + n - 1
};
struct PlanHead {
    int level[kLevels + 1];                  // first item of each step, longest first
    int merges;
};

struct TcWs {
    float *lse2;          // [B*H][c*G] log-sum-exp, log2 units
    PlanHead *head;
    Item *items;          // [max_items]
    Merge *merges;        // [B * pairs]
    float2 *part_ml;      // [kMaxParts][part_rows]
    float *part_o;        // [kMaxParts][d/4][part_rows][4]: a warp stores 32 rows' four columns as 512 bytes
    float *score_parts;   // [2 * kScoreCtas][kBlk] sums of key tiles that two CTAs or more share
    int max_items, part_rows, pairs, pair_tokens, parts;
    bool direct, whole_scores;
};

__device__ __forceinline__ int pair_key_tiles(const SeqState &st, int pair, int pair_tokens)
{
    return (st.past + min((pair + 1) * pair_tokens, st.len) + kBlk - 1) / kBlk;
}

// The item list.  Cutting items into pieces of p tiles makes sum(ceil(T / p)) of them; CTAs take them in
// rounds, so a call takes about  max(ceil(pieces / SMs) * (mean length + kItemCost), longest + kItemCost):
// lengths between a quarter and one and a half of an SM's even share are tried, and no cut at all.
__global__ void __launch_bounds__(kPlanThreads)
paged_plan_kernel(const __grid_constant__ PagedView pv, const __grid_constant__ TcWs ws)
{
    __shared__ int tiles[kPlanCache], level[kLevels], warp_cnt[kPlanWarps], warp_max_[kPlanWarps], cand_piece[kCandidates], n_parts, n_merges;
    __shared__ float cand_cost[kCandidates], warp_work[kPlanWarps];
    __shared__ SeqState seqs[A2SF_PAGED_MAX_SEQUENCES];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    dependency_wait();
    dependents_may_start();
    if (tid < kLevels) level[tid] = 0;
    if (tid == 0) { n_parts = 0; n_merges = 0; }
    const int all = pv.B * ws.pairs;
    for (int b = tid; b < pv.B; b += kPlanThreads) seqs[b] = seq_state(pv, b);
    __syncthreads();
    auto measure = [&](int x) -> int {
        const int b = x / ws.pairs, p = x - b * ws.pairs;
        const SeqState st = seqs[b];
        return p * ws.pair_tokens < st.len ? pair_key_tiles(st, p, ws.pair_tokens) : 0;
    };
    auto item_tiles = [&](int x) -> int { return x < kPlanCache ? tiles[x] : measure(x); };
    float sum = 0.f;                                         // of tiles: only the choice below uses it
    int cnt = 0, mx = 0;
    for (int x = tid; x < all; x += kPlanThreads) {
        const int t = measure(x);
        if (x < kPlanCache) tiles[x] = t;
        sum += t;
        cnt += t > 0;
        mx = max(mx, t);
    }
    sum = warp_sum(sum);
    const int wcnt = __reduce_add_sync(0xffffffffu, cnt), wmax = __reduce_max_sync(0xffffffffu, mx);
    if (lane == 0) { warp_work[warp] = sum; warp_cnt[warp] = wcnt; warp_max_[warp] = wmax; }
    __syncthreads();
    const bool in = lane < kPlanWarps;
    const float work = (float)pv.H * warp_sum(in ? warp_work[lane] : 0.f);
    const int items = __reduce_add_sync(0xffffffffu, in ? warp_cnt[lane] : 0);
    const int longest = __reduce_max_sync(0xffffffffu, in ? warp_max_[lane] : 0);
    int piece = 0x7fffffff;
    if ((long long)items * pv.H < kSplitBelow && longest > kMinPiece) {
        // the last candidate is no cut
        const float share = work / kSms;
        for (int w = warp; w < kCandidates; w += kPlanWarps) {
            const int p = w == kCandidates - 1 ? 0x7fffffff : max(kMinPiece, (int)ceilf(share * 0.25f * exp2f(w * (2.585f / 30.f))));
            const float per = 1.f / (float)p;                // an estimate: no exact division needed
            float n = 0.f, most = 0.f;
            for (int x = lane; x < all; x += 32) {
                const float t = (float)item_tiles(x), k = ceilf(t * per);
                n += k;
                most = fmaxf(most, t > 0.f ? __fdividef(t, k) : 0.f);
            }
            n = warp_sum(n) * pv.H;
            most = warp_max(most);
            if (lane == 0) {
                const float rounds = ceilf(n / kSms);
                cand_cost[w] = fmaxf(rounds * (work / fmaxf(n, 1.f) + kItemCost), most + kItemCost);
                cand_piece[w] = p;
            }
        }
        __syncthreads();
        float best = cand_cost[lane];
        int at = lane;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const float c = __shfl_xor_sync(0xffffffffu, best, o);
            const int i = __shfl_xor_sync(0xffffffffu, at, o);
            if (c < best || (c == best && i > at)) { best = c; at = i; }     // of equals the longer piece
        }
        piece = cand_piece[at];
    }
    const int longest_piece = min(longest, piece);
    auto level_of = [&](int len) { return kLevels - 1 - min(kLevels - 1, (int)((long long)len * kLevels / (longest_piece + 1))); };
    for (int x = tid; x < all; x += kPlanThreads) {
        const int t = item_tiles(x);
        if (!t) continue;
        const int n = (t - 1) / piece + 1;
        atomicAdd(&level[level_of((t + n - 1) / n)], n);
    }
    __syncthreads();
    if (tid == 0) {
        int run = 0;
        for (int l = 0; l < kLevels; ++l) {
            const int v = level[l];
            ws.head->level[l] = min(run, ws.max_items);
            level[l] = run;
            run += v;
        }
        ws.head->level[kLevels] = min(run, ws.max_items);
    }
    __syncthreads();
    // the order of equal lengths may differ from run to run; no result depends on it
    for (int x = tid; x < all; x += kPlanThreads) {
        const int t = item_tiles(x);
        if (!t) continue;
        const int n = (t - 1) / piece + 1, b = x / ws.pairs, p = x - b * ws.pairs;
        const SeqState st = seqs[b];
        int at = atomicAdd(&level[level_of((t + n - 1) / n)], n);
        int part = -1;
        if (n > 1) {
            part = atomicAdd(&n_parts, n);
            (void)A2SF_IN_RANGE((long long)(part + n) * pv.H - 1, ws.parts, kDbgPagedTc);
            ws.merges[atomicAdd(&n_merges, 1)] = Merge{b, p, n, part};
        }
        for (int s = 0; s < n; ++s, ++at)
            if (A2SF_IN_RANGE(at, ws.max_items, kDbgPagedTc) && at < ws.max_items)
                ws.items[at] = Item{b, p, (int)((long long)t * s / n), (int)((long long)t * (s + 1) / n), n > 1 ? part + s : -1, st.past, st.len, 0};
    }
    __syncthreads();
    if (tid == 0) ws.head->merges = n_merges;
}

// ============================================================================================
// attn
// ============================================================================================
constexpr int kAttnThreads = 320;            // producer warp, MMA warp, 8 softmax warps
constexpr int kKStages = 3, kVStages = 2;
constexpr float kOptimisticLimit = 32768.f;  // a row sum below this keeps every probability < 2^15
constexpr float kRescaleThreshold = 8.0f;    // log2 units above the reference; beyond that limit one of 64 is 9 above
// A new reference lies so far below the row's maximum (log2 units).  fp16 holds all bits of a probability down to 2^-14 and none
// below 2^-24, while the row sum counts it: with 8 that is 2^-22 and 2^-32 of the maximum, and a tile of which all logits equal
// it still has half of the limit.  Rounded up, where logits are large: no exponent is above kBelow then.
template <typename T> constexpr float kBelow = std::is_same<T, __half>::value ? 8.f : 0.f;

struct AttnShared {
    uint64_t q_full, q_empty, k_full[kKStages], k_empty[kKStages], v_full[kVStages], v_empty[kVStages];
    uint64_t s_full[2], p_full[2], o_done[2], o_free[2];    // per stream
    uint32_t tmem_base;
    int abort_flag;
    int level[kLevels + 1];
    float xch[2][2][kBlk];                                  // [stream][column half][row]
};

template <int D> constexpr size_t attn_smem() { return (size_t)Tile<D>::kBytes * (2 + kKStages + kVStages) + sizeof(AttnShared); }
static_assert(attn_smem<128>() <= 227 * 1024, "attention shared memory");

template <typename T, int D>
__global__ void __launch_bounds__(kAttnThreads, 1)
paged_attn_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v, const __grid_constant__ AttendArgs a, const __grid_constant__ TcWs ws)
{
    constexpr int kTileBytes = Tile<D>::kBytes;
    constexpr int kFmt = std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
    constexpr int OW = D / 2;                               // output columns per thread
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t *Qs = smem, *Ks = Qs + 2 * kTileBytes, *Vs = Ks + kKStages * kTileBytes;
    AttnShared *sh = reinterpret_cast<AttnShared *>(Vs + kVStages * kTileBytes);
    const PagedView &pv = a.pv;
    const int G = pv.G, tile_tokens = kBlk / G, tile_rows = tile_tokens * G;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &sh->abort_flag;

    if (threadIdx.x == 0) {
        mbar_init(&sh->q_full, 1);
        mbar_init(&sh->q_empty, 1);
        for (int s = 0; s < kKStages; ++s) { mbar_init(&sh->k_full[s], 1); mbar_init(&sh->k_empty[s], 1); }
        for (int s = 0; s < kVStages; ++s) { mbar_init(&sh->v_full[s], 1); mbar_init(&sh->v_empty[s], 1); }
        for (int x = 0; x < 2; ++x) {
            mbar_init(&sh->s_full[x], 1);
            mbar_init(&sh->p_full[x], 2 * kBlk);
            mbar_init(&sh->o_done[x], 1);
            mbar_init(&sh->o_free[x], 2 * kBlk);
        }
        sh->abort_flag = smem_u32(smem) & 1023u ? 1 : 0;    // the swizzled tiles need this alignment
        fence_mbar_init();
        prefetch_tmap(&map_q); prefetch_tmap(&map_k); prefetch_tmap(&map_v);
    }
    if (warp == 1) {
        tmem_alloc(&sh->tmem_base, 512);
        tmem_relinquish();
    }
    // rows that no query copy fills (G does not divide 128) stay zero, so that their logits stay finite
    for (int x = threadIdx.x; x < 2 * Tile<D>::kHalves * (kBlk - tile_rows) * 8; x += kAttnThreads) {
        const int piece = x & 7, row = tile_rows + (x >> 3) % (kBlk - tile_rows), half = (x >> 3) / (kBlk - tile_rows);
        *reinterpret_cast<uint4 *>(Qs + half * Tile<D>::kHalfBytes + row * 128 + piece * 16) = make_uint4(0, 0, 0, 0);
    }
    fence_async_smem();
    dependency_wait();
    if (!ws.direct && threadIdx.x <= kLevels) sh->level[threadIdx.x] = ws.head->level[threadIdx.x];
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    dependents_may_start();
    const uint32_t tmem_base = sh->tmem_base;

    // A failed wait poisons the CTA: later waits return at once, loops keep their shape.
    auto wait = [&](uint64_t *bar, uint32_t parity) -> bool {
        if (*abort_flag) return false;
        return mbar_wait(bar, parity, abort_flag);
    };
    // Jobs: by step of length, then by head (the items of a head run together and share its K and V
    // through L2), dealt in rounds of alternating direction.
    const int n_units = ws.direct ? pv.B * ws.pairs * pv.H : sh->level[kLevels] * pv.H;
    auto dealt = [&](int round) { return round * (int)gridDim.x + (round & 1 ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x); };
    // what an item means to every role
    struct Job {
        int b, h, i0, tokens, t0, nt, ntA, ntB, past, used, part;
    };
    auto job = [&](int unit) -> Job {
        Job j;
        Item it;
        if (ws.direct) {
            // the longest pairs of all sequences and heads first, so that a round of jobs is of about one length; pairs
            // behind the chunk are empty
            const int units = pv.B * pv.H, back = unit / units, rest = unit - back * units;
            it.b = rest / pv.H;
            j.h = rest - it.b * pv.H;
            it.pair = ws.pairs - 1 - back;
            const SeqState st = seq_state(pv, it.b);
            it.past = st.past; it.len = st.len; it.part = -1;
            it.t0 = 0;
            it.t1 = it.pair * ws.pair_tokens < st.len ? pair_key_tiles(st, it.pair, ws.pair_tokens) : 0;
        } else {
            int l = 0;
            while (l < kLevels - 1 && unit >= sh->level[l + 1] * pv.H) ++l;
            const int first = sh->level[l], n_items = sh->level[l + 1] - first, rest = unit - first * pv.H;
            it = ws.items[first + rest % n_items];
            j.h = rest / n_items;
        }
        j.b = it.b;
        j.past = it.past; j.used = it.past + it.len;
        j.i0 = it.pair * ws.pair_tokens;
        j.tokens = min(ws.pair_tokens, it.len - j.i0);
        j.t0 = it.t0;
        // stream A sees no slot beyond its own last token's
        const int endA = (it.past + min(j.i0 + tile_tokens, it.len) + kBlk - 1) / kBlk;
        j.ntB = j.tokens > tile_tokens ? it.t1 - it.t0 : 0;
        j.ntA = max(0, min(it.t1, endA) - it.t0);
        j.nt = max(j.ntA, j.ntB);
        j.part = it.part < 0 ? -1 : it.part * pv.H + j.h;
        if (j.part >= 0 && !A2SF_IN_RANGE(j.part, ws.parts, kDbgPagedTc)) j.part = 0;
        return j;
    };

    if (warp == 0) {
        // ---- TMA producer: lane i copies page box i ------------------------------------------
        int kt = 0, n = 0;                                  // tiles and items so far
        for (int round = 0, unit; (unit = dealt(round)) < n_units; ++round) {
            const Job j = job(unit);
            if (j.nt == 0) continue;
            const int32_t *table = pv.table + (size_t)j.b * pv.max_pages;
            int ok = 1;
            if (lane == 0) {
                ok = n == 0 || wait(&sh->q_empty, (n - 1) & 1) ? 1 : 0;
                if (ok) {
                    const uint32_t bytes = (uint32_t)(tile_rows * 128 * Tile<D>::kHalves);
                    mbar_arrive_expect_tx(&sh->q_full, j.ntB ? 2 * bytes : bytes);
                    copy_query_tile<D>(Qs, &map_q, &sh->q_full, j.h * G, j.i0, j.b);
                    if (j.ntB) copy_query_tile<D>(Qs + kTileBytes, &map_q, &sh->q_full, j.h * G, j.i0 + tile_tokens, j.b);
                }
            }
            if (!__shfl_sync(0xffffffffu, ok, 0)) break;
            ++n;
            for (int t = 0; t < j.nt; ++t, ++kt) {
                const int tile = j.t0 + t, ks = kt % kKStages, vs = kt % kVStages;
                const PageTile p = page_tile(pv, tile, j.used);
                const int slot = tile * kBlk + lane * p.box;
                int row = 0;
                if (lane < p.boxes) row = (int)pool_row(pv, page_for_read(pv, table, slot), j.h, slot);
                const uint32_t bytes = (uint32_t)(p.boxes * p.box * 128 * Tile<D>::kHalves);
                ok = 1;
                if (lane == 0) {
                    if (kt >= kKStages) ok = wait(&sh->k_empty[ks], ((kt / kKStages) & 1) ^ 1) ? 1 : 0;
                    if (ok) mbar_arrive_expect_tx(&sh->k_full[ks], bytes);
                }
                if (!__shfl_sync(0xffffffffu, ok, 0)) break;
                copy_page_tile<D>(Ks + ks * kTileBytes, &map_k, &sh->k_full[ks], p, row);
                if (lane == 0) {
                    if (kt >= kVStages) ok = wait(&sh->v_empty[vs], ((kt / kVStages) & 1) ^ 1) ? 1 : 0;
                    if (ok) mbar_arrive_expect_tx(&sh->v_full[vs], bytes);
                }
                if (!__shfl_sync(0xffffffffu, ok, 0)) { ++kt; break; }   // K of this tile is on its way
                copy_page_tile<D>(Vs + vs * kTileBytes, &map_v, &sh->v_full[vs], p, row);
            }
        }
        if (lane == 0 && *abort_flag) {
            // copies still in flight get a bounded chance to land before the CTA exits
            int dummy = 0;
            for (int k = max(0, kt - kKStages); k < kt; ++k) mbar_wait(&sh->k_full[k % kKStages], (k / kKStages) & 1, &dummy);
            for (int k = max(0, kt - kVStages); k < kt; ++k) mbar_wait(&sh->v_full[k % kVStages], (k / kVStages) & 1, &dummy);
            if (n > 0) mbar_wait(&sh->q_full, (n - 1) & 1, &dummy);
        }
    } else if (warp == 1) {
        // ---- MMA issuer (lane 0; the warp stays together to clear values behind a sequence) -----------
        const uint32_t idesc_qk = make_idesc(kFmt, kBlk, kBlk, 0, 0);
        const uint32_t idesc_pv = make_idesc(kFmt, kBlk, D, 0, 1);        // V is MN-major
        // descriptors of the first buffers; the others lie whole tiles behind (16-byte units)
        const uint64_t step = kTileBytes >> 4;
        const uint64_t q_desc = kmajor_desc(smem_u32(Qs)), k_desc = kmajor_desc(smem_u32(Ks));
        // V as an MN-major operand: 64-wide halves 16 KB apart, 8-key groups 1024 bytes apart
        const uint64_t v_desc = make_sdesc_sw128(smem_u32(Vs), Tile<D>::kHalfBytes, 1024);
        auto issue_s = [&](int X, int kt) {
            issue_qk<D>(tmem_base + X * 2 * kBlk, q_desc + X * step, k_desc + kt % kKStages * step, idesc_qk);
            umma_commit(&sh->s_full[X]);
        };
        auto issue_pv = [&](int X, int kt, bool first) {
            const uint64_t vd = v_desc + kt % kVStages * step;
            const uint32_t sp = tmem_base + X * 2 * kBlk, o = sp + kBlk;
            // 16 keys per step: 8 columns of packed P, two 8-key groups of V.  Keys 64h .. 64h+63 have
            // their P at columns 64h .. 64h+31: a softmax thread writes over logits it has read itself.
#pragma unroll
            for (int k = 0; k < kBlk / 16; ++k)
                umma_ts(o, sp + 64 * (k >> 2) + 8 * (k & 3), vd + (uint64_t)(k * 2048 >> 4), idesc_pv, !first || k > 0);
            umma_commit(&sh->o_done[X]);
        };
        int kt = 0, n = 0, cnt[2] = {0, 0}, used_before[2] = {0, 0};      // tiles per stream; items per stream
        for (int round = 0, unit; (unit = dealt(round)) < n_units; ++round) {
            if (__any_sync(0xffffffffu, *abort_flag)) break;
            const Job j = job(unit);
            if (j.nt == 0) continue;
            const int ntX[2] = {j.ntA, j.ntB};
            wait(&sh->q_full, n++ & 1);
            wait(&sh->k_full[kt % kKStages], (kt / kKStages) & 1);
            tc_fence_after_sync();
            if (lane == 0) {
                if (j.ntA) issue_s(0, kt);
                if (j.ntB) issue_s(1, kt);
                umma_commit(&sh->k_empty[kt % kKStages]);
                if (j.nt == 1) umma_commit(&sh->q_empty);
            }
            for (int t = 0; t < j.nt; ++t, ++kt) {
                const int vs = kt % kVStages;
                wait(&sh->v_full[vs], (kt / kVStages) & 1);
                const bool more = t + 1 < j.nt;
                if (more) wait(&sh->k_full[(kt + 1) % kKStages], ((kt + 1) / kKStages) & 1);
                // slots behind the sequence may hold anything, NaN included: 0 * NaN must not reach O
                const int valid = j.used - (j.t0 + t) * kBlk;
                if (valid < kBlk) {
                    uint8_t *V = Vs + vs * kTileBytes;
                    for (int x = lane; x < Tile<D>::kHalves * (kBlk - valid) * 8; x += 32) {
                        const int piece = x & 7, row = valid + (x >> 3) % (kBlk - valid), half = (x >> 3) / (kBlk - valid);
                        *reinterpret_cast<uint4 *>(V + half * Tile<D>::kHalfBytes + row * 128 + piece * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_async_smem();
                    __syncwarp();
                }
#pragma unroll
                for (int X = 0; X < 2; ++X) {
                    if (t >= ntX[X]) continue;
                    if (t == 0 && used_before[X]) wait(&sh->o_free[X], (used_before[X] - 1) & 1);
                    wait(&sh->p_full[X], cnt[X] & 1);
                    ++cnt[X];
                    tc_fence_after_sync();
                    if (lane == 0) {
                        issue_pv(X, kt, t == 0);
                        if (t + 1 < ntX[X]) issue_s(X, kt + 1);
                    }
                }
                if (lane == 0) {
                    umma_commit(&sh->v_empty[vs]);
                    if (more) umma_commit(&sh->k_empty[(kt + 1) % kKStages]);
                    if (t + 2 == j.nt) umma_commit(&sh->q_empty);          // the last logits have been asked for
                }
                __syncwarp();
            }
            for (int X = 0; X < 2; ++X) used_before[X] += ntX[X] > 0;
        }
    } else {
        // ---- softmax + epilogue: two threads per row, the streams taken in turn ----------------------
        const int quarter = warp & 3;                      // TMEM lanes this warp may touch
        const int half = (warp - 2) >> 2;                  // logits 64*half .. 64*half+63
        const int r = quarter * 32 + lane;                 // row in the tile = TMEM lane
        const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
        const int r_tok = r / G, r_head = r - r_tok * G;   // token and head of the row in its tile,
        const int r0_tok = (r & ~3) / G, r0_head = (r & ~3) - r0_tok * G;     // and of the first of four rows
        int cnt[2] = {0, 0};
        float m_used[2], l[2];
        // no early exit here: the two warps of a quarter meet at named barriers, and after a failed wait
        // all that follows runs through without waiting
        for (int round = 0, unit; (unit = dealt(round)) < n_units; ++round) {
            const Job j = job(unit);
            if (j.nt == 0) continue;
            // The stream is a run-time number and each body stands in the code once: a CTA's first pass through
            // it waits for its instructions (1 to 2 us for every copy of a body).
            auto do_tile = [&](int X, int t, float &m_x, float &l_x, int cnt_x) {
                const uint32_t sp = tmem_base + X * 2 * kBlk + lane_base + half * 64;
                const uint32_t to = tmem_base + X * 2 * kBlk + kBlk + lane_base + half * OW;
                const int first_token = j.i0 + X * tile_tokens;
                wait(&sh->s_full[X], cnt_x & 1);
                tc_fence_after_sync();
                uint32_t v[2][32];
                tmem_ld32(sp, v[0]);
                tmem_ld32(sp + 32, v[1]);
                tmem_wait_ld();
                const int tile0 = (j.t0 + t) * kBlk;
                if (tile0 + kBlk > j.past + first_token + 1) {
                    // some row of the tile does not see all of it: a masked logit becomes -inf
                    const int vis = min(j.past + first_token + r_tok + 1, j.used) - tile0 - half * 64;
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int x = 0; x < 32; ++x)
                            if (c * 32 + x >= vis) v[c][x] = 0xff800000u;
                }
                auto write_p = [&](float neg_m) -> float {
                    const uint64_t sl2x2 = pack_f32x2(__float_as_uint(pv.sl2), __float_as_uint(pv.sl2));
                    const uint64_t nmx2 = pack_f32x2(__float_as_uint(neg_m), __float_as_uint(neg_m));
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
                        tmem_st16(sp + c * 16, p);
                    }
                    float rs[8];
#pragma unroll
                    for (int x = 0; x < 4; ++x) unpack_f32x2(rs2[x], rs[2 * x], rs[2 * x + 1]);
                    return ((rs[0] + rs[1]) + (rs[2] + rs[3])) + ((rs[4] + rs[5]) + (rs[6] + rs[7]));
                };
                float factor = 1.f, rowsum = 0.f;
                bool exact = (t == 0);
                if (!exact) {
                    rowsum = write_p(-m_x);
                    const bool bad = !(rowsum <= kOptimisticLimit);          // also NaN
                    sh->xch[X][half][r] = bad ? 1.f : 0.f;
                    named_barrier(1 + quarter, 64);                // this quarter's two warps
                    const bool pair_bad = bad || sh->xch[X][half ^ 1][r] != 0.f;
                    exact = __any_sync(0xffffffffu, pair_bad);
                    if (exact) named_barrier(1 + quarter, 64);     // flags read before the buffer is reused
                }
                if (exact) {
                    float own = -INFINITY;
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int x = 0; x < 32; ++x) own = fmaxf(own, __uint_as_float(v[c][x]));
                    sh->xch[X][half][r] = own;
                    named_barrier(1 + quarter, 64);
                    const float smax = fmaxf(own, sh->xch[X][half ^ 1][r]);
                    if (t == 0) {
                        // a piece of the keys may hold none that this row sees (then none of the following
                        // tiles does either): any finite reference gives the zeros that are wanted
                        m_x = smax == -INFINITY ? 0.f : __fmaf_ru(smax, pv.sl2, -kBelow<T>);
                        l_x = 0.f;
                    } else {
                        const float xmax = fmaf(smax, pv.sl2, -m_x);
                        const bool grow = xmax > kRescaleThreshold;
                        if (grow) {
                            const float before = m_x;
                            m_x = __fmaf_ru(smax, pv.sl2, -kBelow<T>);
                            factor = ex2_approx(before - m_x);
                        }
                        if (__any_sync(0xffffffffu, grow)) {
                            wait(&sh->o_done[X], (cnt_x - 1) & 1);          // O holds the tiles before
                            tc_fence_after_sync();
#pragma unroll 1
                            for (int c = 0; c < OW / 32; ++c) {
                                uint32_t o[32];
                                tmem_ld32(to + c * 32, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int x = 0; x < 32; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * factor);
                                tmem_st32(to + c * 32, o);
                            }
                            tmem_wait_st();
                        }
                    }
                    rowsum = write_p(-m_x);
                }
                tmem_wait_st();
                l_x = fmaf(l_x, factor, rowsum);
                tc_fence_before_sync();
                mbar_arrive(&sh->p_full[X]);
            };
#pragma unroll 1
            for (int step = 0; step < 2 * j.nt; ++step) {
                const int X = step & 1, t = step >> 1;
                if (t >= (X ? j.ntB : j.ntA)) continue;
                float m_x = X ? m_used[1] : m_used[0], l_x = X ? l[1] : l[0];
                do_tile(X, t, m_x, l_x, X ? cnt[1] : cnt[0]);
                if (X) { m_used[1] = m_x; l[1] = l_x; ++cnt[1]; }
                else   { m_used[0] = m_x; l[0] = l_x; ++cnt[0]; }
            }
            // ---- epilogue: each thread normalises (or hands on) and stores its half of the columns
            // the halves of the row sums, of both streams at once
            named_barrier(1 + quarter, 64);                    // the partner has read the last exchange
            sh->xch[0][half][r] = l[0];
            sh->xch[1][half][r] = l[1];
            named_barrier(1 + quarter, 64);
            l[0] += sh->xch[0][half ^ 1][r];
            l[1] += sh->xch[1][half ^ 1][r];
            named_barrier(1 + quarter, 64);                    // read before the next item writes
            auto finish = [&](int X, int ntX, float m_x, float lsum, int cnt_x) {
                const int tok = X * tile_tokens + r_tok, g = r_head;
                const bool live = r < tile_rows && tok < j.tokens && A2SF_IN_RANGE(j.i0 + tok, pv.c, kDbgPagedTc);
                if (ntX == 0) {
                    // a cut item whose piece lies behind everything stream A sees: an empty partial result
                    if (j.part >= 0 && X == 0 && half == 0) ws.part_ml[(size_t)j.part * ws.part_rows + r] = make_float2(-INFINITY, 0.f);
                    return;
                }
                const uint32_t to = tmem_base + X * 2 * kBlk + kBlk + lane_base + half * OW;
                const float inv = 1.f / lsum;
                const int i = j.i0 + tok;
                // addresses first: the last product is still under way.  This lane stores piece lane & 3 of rows
                // r0 .. r0 + 3, or its own row's partial columns
                T *orow[4];
                float4 *po = nullptr;
                if (j.part < 0) {
                    const int r0 = r & ~3;
                    int tk = X * tile_tokens + r0_tok, gk = r0_head;
                    T *base = static_cast<T *>(a.out) + (int64_t)j.b * a.so.b + half * OW + (lane & 3) * 8;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const bool in = r0 + k < tile_rows && tk < j.tokens && A2SF_IN_RANGE(j.i0 + tk, pv.c, kDbgPagedTc);
                        orow[k] = in ? base + (int64_t)(j.h * G + gk) * a.so.h + (int64_t)(j.i0 + tk) * a.so.t : nullptr;
                        if (++gk == G) { gk = 0; ++tk; }
                    }
                } else if (live) {
                    po = reinterpret_cast<float4 *>(ws.part_o) + ((size_t)j.part * (D / 4) + half * (OW / 4)) * ws.part_rows + X * kBlk + r;
                }
                const bool done = wait(&sh->o_done[X], (cnt_x - 1) & 1);
                tc_fence_after_sync();
                uint32_t o[OW / 32][32];
#pragma unroll
                for (int c = 0; c < OW / 32; ++c) tmem_ld32(to + c * 32, o[c]);
                tmem_wait_ld();
                tc_fence_before_sync();
                mbar_arrive(&sh->o_free[X]);                   // the accumulator is in registers
#pragma unroll
                for (int c = 0; c < OW / 32; ++c) {
                    if (j.part < 0) {
                        uint4 w[4];
#pragma unroll
                        for (int q4 = 0; q4 < 4; ++q4) {
                            uint32_t x[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                x[e] = pack2<T>(__uint_as_float(o[c][q4 * 8 + 2 * e]) * inv, __uint_as_float(o[c][q4 * 8 + 2 * e + 1]) * inv);
                            w[q4] = make_uint4(x[0], x[1], x[2], x[3]);
                        }
                        transpose4(w);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (orow[k] && done) *reinterpret_cast<uint4 *>(orow[k] + c * 32) = w[k];
                    } else if (po && done) {
#pragma unroll
                        for (int q8 = 0; q8 < 8; ++q8) {
                            *po = make_float4(__uint_as_float(o[c][q8 * 4]), __uint_as_float(o[c][q8 * 4 + 1]), __uint_as_float(o[c][q8 * 4 + 2]),
                                              __uint_as_float(o[c][q8 * 4 + 3]));
                            po += ws.part_rows;
                        }
                    }
                }
                if (half == 0 && live && done) {
                    if (j.part < 0) {
                        const float z = m_x + log2f(lsum);
                        ws.lse2[((size_t)j.b * pv.H + j.h) * pv.c * G + (size_t)i * G + g] = z;
                        if (a.lse) a.lse[(((size_t)j.b * pv.H + j.h) * G + g) * pv.c + i] = z * 0.6931471805599453f;
                    } else {
                        ws.part_ml[(size_t)j.part * ws.part_rows + X * kBlk + r] = make_float2(lsum > 0.f ? m_x : -INFINITY, lsum);
                    }
                }
            };
#pragma unroll 1
            for (int X = 0; X < 2; ++X)
                finish(X, X ? j.ntB : j.ntA, X ? m_used[1] : m_used[0], X ? l[1] : l[0], X ? cnt[1] : cnt[0]);
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

// ============================================================================================
// merge: a block per 32 rows of a cut item; lane = row, a warp takes every eighth group of four columns
// ============================================================================================
constexpr int kMergeThreads = 256;

template <typename T, int D>
__global__ void __launch_bounds__(kMergeThreads)
paged_merge_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ TcWs ws)
{
    constexpr int NG = D / 4 / 8;                            // column groups of a warp
    constexpr int LD = D + 8;                                // halfwords of a staged row
    __shared__ __align__(16) T stage[32][LD];
    const PagedView &pv = a.pv;
    const int G = pv.G, tile_tokens = kBlk / G, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    dependency_wait();
    dependents_may_start();
    const int row_blocks = ws.part_rows / 32;
    const long long jobs = (long long)ws.head->merges * pv.H * row_blocks;
    for (long long x = blockIdx.x; x < jobs; x += gridDim.x) {
        const int pr0 = (int)(x % row_blocks) * 32, pr = pr0 + lane;
        const long long y = x / row_blocks;
        const int h = (int)(y % pv.H);
        const Merge mg = ws.merges[y / pv.H];
        const SeqState st = seq_state(pv, mg.b);
        auto token = [&](int row) {                          // of the chunk, or -1 for a row that is none
            const int X = row / kBlk, r = row - X * kBlk, tok = X * tile_tokens + r / G;
            const int i = mg.pair * ws.pair_tokens + tok;
            return r < tile_tokens * G && tok < ws.pair_tokens && i < st.len ? i : -1;
        };
        const size_t base = ((size_t)mg.part * pv.H + h) * ws.part_rows, step = (size_t)pv.H * ws.part_rows;
        const int i = token(pr);
        // pieces that hold nothing the row sees have weight 0; what lies there is not used
        float mx = -INFINITY, l = 0.f;
        for (int s = 0; s < mg.n; ++s) {
            const float2 ml = i >= 0 ? ws.part_ml[base + s * step + pr] : make_float2(0.f, 0.f);
            mx = fmaxf(mx, ml.y > 0.f ? ml.x : -INFINITY);
        }
        float4 o[NG];
#pragma unroll
        for (int e = 0; e < NG; ++e) o[e] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
        for (int s = 0; s < mg.n; ++s) {
            const float2 ml = i >= 0 ? ws.part_ml[base + s * step + pr] : make_float2(0.f, 0.f);
            const float f = ml.y > 0.f ? exp2f(ml.x - mx) : 0.f;
            l = fmaf(f, ml.y, l);
            const float4 *src = reinterpret_cast<const float4 *>(ws.part_o) + (base + s * step) * (D / 4) + pr;
#pragma unroll
            for (int e = 0; e < NG; ++e) {
                const float4 v = f > 0.f ? src[(size_t)(warp + 8 * e) * ws.part_rows] : make_float4(0.f, 0.f, 0.f, 0.f);
                o[e].x = fmaf(f, v.x, o[e].x); o[e].y = fmaf(f, v.y, o[e].y);
                o[e].z = fmaf(f, v.z, o[e].z); o[e].w = fmaf(f, v.w, o[e].w);
            }
        }
        const float inv = 1.f / l;
        __syncthreads();                                     // the stage has been read
#pragma unroll
        for (int e = 0; e < NG; ++e)
            *reinterpret_cast<uint2 *>(&stage[lane][(warp + 8 * e) * 4]) = make_uint2(pack2<T>(o[e].x * inv, o[e].y * inv), pack2<T>(o[e].z * inv, o[e].w * inv));
        if (warp == 0 && i >= 0) {
            const int g = (pr % kBlk) % G;
            const float z = mx + log2f(l);
            ws.lse2[((size_t)mg.b * pv.H + h) * pv.c * G + (size_t)i * G + g] = z;
            if (a.lse) a.lse[(((size_t)mg.b * pv.H + h) * G + g) * pv.c + i] = z * 0.6931471805599453f;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < 32 * (D / 8); e += kMergeThreads) {
            const int row = e / (D / 8), ch = e % (D / 8), ir = token(pr0 + row), g = ((pr0 + row) % kBlk) % G;
            if (ir >= 0)
                *reinterpret_cast<uint4 *>(static_cast<T *>(a.out) + (int64_t)mg.b * a.so.b + (int64_t)(h * G + g) * a.so.h +
                                           (int64_t)ir * a.so.t + ch * 8) = *reinterpret_cast<const uint4 *>(&stage[row][ch * 8]);
        }
    }
}

// ============================================================================================
// score
// ============================================================================================
constexpr int kScoreThreads = 320;           // producer warp, MMA warp, 8 epilogue warps
constexpr int kScoreStages = 2;
// Ring of row-constant vectors.  Slot x % ring is rewritten for tile x after the products of tile x-2 have
// retired; those needed the accumulator of tile x-4, i.e. every thread had finished tile x-5.
constexpr int kScoreRing = 8;

struct ScoreShared {
    uint64_t k_full, k_empty, q_full[kScoreStages], q_empty[kScoreStages], acc_full[2], acc_empty[2], c_ready[kScoreRing];
    uint32_t tmem_base;
    int abort_flag;
    alignas(16) float cbuf[kScoreRing][kBlk];
    float part[kBlk];
    long long prefix[A2SF_PAGED_MAX_SEQUENCES + 1];
};
template <int D> constexpr size_t score_smem() { return 1024 + (size_t)Tile<D>::kBytes * (1 + kScoreStages) + sizeof(ScoreShared); }

// Sum of exp2(s * sl2 - c) over this thread's 64 rows; Masked: only rows lo .. hi-1 of them.
template <bool Masked>
__device__ __forceinline__ float strip_sum(const uint32_t (&r)[2][32], const float *cb, float sl2, int lo, int hi)
{
    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int x = 0; x < 32; x += 4) {
            const float4 c4 = *reinterpret_cast<const float4 *>(cb + c * 32 + x);
            const float cc[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float pw = ex2_approx(fmaf(__uint_as_float(r[c][x + e]), sl2, -cc[e]));
                if (Masked) pw = c * 32 + x + e >= lo && c * 32 + x + e < hi ? pw : 0.f;
                part[e] += pw;
            }
        }
    }
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// A sequence's key tiles: the row tiles that see tile kt are the last rows_of(kt) of N.
struct SeqRows {
    int past, len, tiles, N, tile_tokens, first0;           // first0: first row tile with a weight
    __device__ __forceinline__ int first(int kt) const { return max(first0, (kt * kBlk - past) / tile_tokens); }
    __device__ __forceinline__ int rows_of(int kt) const { return N - first(kt); }
    // tiles 0 .. flat()-1 are seen by the same rows
    __device__ __forceinline__ int flat() const { return min(tiles, (past + first0 * tile_tokens) / kBlk + 1); }
};
__device__ __forceinline__ SeqRows seq_rows(const PagedView &pv, float nl2a, int b)
{
    const SeqState st = seq_state(pv, b);
    SeqRows s;
    s.tile_tokens = kBlk / pv.G;
    s.past = st.past; s.len = st.len;
    s.tiles = st.len > 0 ? (st.past + st.len + kBlk - 1) / kBlk : 0;
    s.N = (st.len + s.tile_tokens - 1) / s.tile_tokens;
    s.first0 = first_weighted_token(st.len, nl2a) / s.tile_tokens;
    return s;
}
// Pairs of one head, by a warp.
__device__ __forceinline__ int seq_pairs(const SeqRows &s)
{
    const int lane = threadIdx.x & 31, flat = s.flat();
    int sum = 0;
    for (int kt = flat + lane; kt < s.tiles; kt += 32) sum += s.rows_of(kt);
    return __reduce_add_sync(0xffffffffu, sum) + (s.tiles ? flat * s.rows_of(0) : 0);
}

struct ScorePos {             // a place in the list: key tile kt of (b, h), its row tile q, where the tile begins
    int b, h, kt, q;
    long long begins;
};
// The place of pair w, by a warp; prefix: pairs of one head, summed over the sequences before.
__device__ __forceinline__ ScorePos score_pos(const PagedView &pv, float nl2a, const long long *prefix, long long w)
{
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = pv.B - 1;                              // last b with H * prefix[b] <= w
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (pv.H * prefix[mid] <= w) lo = mid;
        else hi = mid - 1;
    }
    const SeqRows s = seq_rows(pv, nl2a, lo);
    const long long rest = w - pv.H * prefix[lo], per_head = prefix[lo + 1] - prefix[lo];
    ScorePos p;
    p.b = lo;
    p.h = (int)(rest / per_head);
    int r = (int)(rest - p.h * per_head);
    const int flat = s.flat(), n0 = s.rows_of(0);
    if (r < flat * n0) {
        p.kt = r / n0;
        p.q = r - p.kt * n0;
    } else {
        r -= flat * n0;
        int kt0 = flat;
        for (;; kt0 += 32) {                                // the tile whose running sum goes beyond r
            const int n = kt0 + lane < s.tiles ? s.rows_of(kt0 + lane) : 0;
            int incl = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += y;
            }
            const unsigned beyond = __ballot_sync(0xffffffffu, incl > r);
            if (beyond || kt0 + 32 >= s.tiles) {
                const int at = beyond ? __ffs(beyond) - 1 : 31;
                p.kt = kt0 + at;
                p.q = r - __shfl_sync(0xffffffffu, incl - n, at);
                break;
            }
            r -= __shfl_sync(0xffffffffu, incl, 31);
        }
    }
    p.begins = w - p.q;
    return p;
}
// prefix[0 .. B] of the sequences' pairs, by all warps of a block of `warps`
__device__ __forceinline__ void score_prefix(long long *prefix, const PagedView &pv, float nl2a, int warps)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int b = warp; b < pv.B; b += warps) {
        const int n = seq_pairs(seq_rows(pv, nl2a, b));
        if (lane == 0) prefix[b + 1] = n;
    }
    if (threadIdx.x == 0) prefix[0] = 0;
    __syncthreads();
    if (warp == 0) {
        long long run = 0;
        for (int b0 = 0; b0 < pv.B; b0 += 32) {
            long long incl = b0 + lane < pv.B ? prefix[b0 + lane + 1] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += y;
            }
            if (b0 + lane < pv.B) prefix[b0 + lane + 1] = run + incl;
            run += __shfl_sync(0xffffffffu, incl, 31);
        }
    }
    __syncthreads();
}

template <int D>
__global__ void __launch_bounds__(kScoreThreads, 2)
paged_score_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                      const __grid_constant__ AttendArgs a, const __grid_constant__ TcWs ws, int ab_fmt)
{
    constexpr int kTileBytes = Tile<D>::kBytes;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *Ks = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *Qs = Ks + kTileBytes;
    ScoreShared *sh = reinterpret_cast<ScoreShared *>(Qs + kScoreStages * kTileBytes);
    const PagedView &pv = a.pv;
    const int G = pv.G, tile_tokens = kBlk / G, tile_rows = tile_tokens * G;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &sh->abort_flag;

    if (threadIdx.x == 0) {
        mbar_init(&sh->k_full, 1);
        mbar_init(&sh->k_empty, 1);
        for (int s = 0; s < kScoreStages; ++s) { mbar_init(&sh->q_full[s], 1); mbar_init(&sh->q_empty[s], 1); }
        for (int x = 0; x < 2; ++x) { mbar_init(&sh->acc_full[x], 1); mbar_init(&sh->acc_empty[x], 256); }
        for (int x = 0; x < kScoreRing; ++x) mbar_init(&sh->c_ready[x], 1);
        sh->abort_flag = 0;
        fence_mbar_init();
        prefetch_tmap(&map_q);
        prefetch_tmap(&map_k);
    }
    if (warp == 1) {
        tmem_alloc(&sh->tmem_base, 256);
        tmem_relinquish();
    }
    score_prefix(sh->prefix, pv, a.nl2a, kScoreThreads / 32);     // from the lengths: no kernel of the call writes them
    // rows that no query copy fills stay zero, so that their logits stay finite
    for (int x = threadIdx.x; x < kScoreStages * Tile<D>::kHalves * (kBlk - tile_rows) * 8; x += kScoreThreads) {
        const int piece = x & 7, row = tile_rows + (x >> 3) % (kBlk - tile_rows), half = (x >> 3) / (kBlk - tile_rows);
        *reinterpret_cast<uint4 *>(Qs + half * Tile<D>::kHalfBytes + row * 128 + piece * 16) = make_uint4(0, 0, 0, 0);
    }
    fence_async_smem();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = sh->tmem_base;
    const long long total = pv.H * sh->prefix[pv.B], share = (total + gridDim.x - 1) / gridDim.x;
    long long w0 = blockIdx.x * share;
    const long long w1 = w0 + share < total ? w0 + share : total;
    ScorePos at = {};
    SeqRows seq = {};
    if (w0 < w1) {
        at = score_pos(pv, a.nl2a, sh->prefix, w0);
        seq = seq_rows(pv, a.nl2a, at.b);
    }
    // the pair behind `at`'s key tile
    auto next_tile = [&](long long w) {
        at.q = 0;
        if (w < w1 && ++at.kt == seq.tiles) {
            at.kt = 0;
            if (++at.h == pv.H) {
                at.h = 0;
                do seq = seq_rows(pv, a.nl2a, ++at.b); while (seq.tiles == 0);      // there is one: w < w1
            }
        }
    };
    if (ws.whole_scores && at.q > 0) {                     // that tile is another CTA's
        w0 += seq.rows_of(at.kt) - at.q;
        next_tile(w0);
    }

    struct Job {
        int b, h, j0, past, len, used, q0, nq;             // query tiles q0 .. q0 + nq - 1
        int part;                                          // -1: all of the key tile's; else where its sums go
    };
    // the part of this CTA's share that lies in the current key tile; then on to the next tile
    auto next_job = [&](long long &w) -> Job {
        Job j;
        j.b = at.b; j.h = at.h; j.j0 = at.kt * kBlk;
        j.past = seq.past; j.len = seq.len; j.used = seq.past + seq.len;
        const int n = seq.rows_of(at.kt);
        j.nq = ws.whole_scores ? n : (int)min((long long)(n - at.q), w1 - w);
        j.q0 = seq.first(at.kt) + at.q;
        // a tile begun by another CTA is this one's first, a tile that the next one goes on with its last
        j.part = at.q > 0 ? 2 * (int)blockIdx.x : j.nq < n ? 2 * (int)blockIdx.x + 1 : -1;
        w += j.nq;
        next_tile(w);
        return j;
    };
    auto wait = [&](uint64_t *bar, uint32_t parity) -> bool {
        if (*abort_flag) return false;
        return mbar_wait(bar, parity, abort_flag);
    };

    if (warp == 0) {
        // Only the row constants come from the kernels before: the first K and Q tiles are requested, and the
        // first products made, without waiting for them.
        int qt = 0, n = 0;
        bool waited = false;
        for (long long w = w0; w < w1; ++n) {
            const Job j = next_job(w);
            const PageTile p = page_tile(pv, j.j0 / kBlk, j.used);
            const int slot = j.j0 + lane * p.box;
            int row = 0, ok = 1;
            if (lane < p.boxes) row = (int)pool_row(pv, page_for_read(pv, pv.table + (size_t)j.b * pv.max_pages, slot), j.h, slot);
            if (lane == 0) {
                ok = n == 0 || wait(&sh->k_empty, (n - 1) & 1) ? 1 : 0;
                if (ok) mbar_arrive_expect_tx(&sh->k_full, (uint32_t)(p.boxes * p.box * 128 * Tile<D>::kHalves));
            }
            if (!__shfl_sync(0xffffffffu, ok, 0)) break;
            copy_page_tile<D>(Ks, &map_k, &sh->k_full, p, row);
            const float *lse2 = ws.lse2 + ((size_t)j.b * pv.H + j.h) * pv.c * G;
            for (int t = 0; t < j.nq; ++t, ++qt) {
                const int s = qt % kScoreStages, i0 = (j.q0 + t) * tile_tokens;
                ok = 1;
                if (lane == 0) {
                    if (qt >= kScoreStages) ok = wait(&sh->q_empty[s], ((qt / kScoreStages) & 1) ^ 1) ? 1 : 0;
                    if (ok) {
                        mbar_arrive_expect_tx(&sh->q_full[s], (uint32_t)(tile_rows * 128 * Tile<D>::kHalves));
                        copy_query_tile<D>(Qs + s * kTileBytes, &map_q, &sh->q_full[s], j.h * G, i0, j.b);
                    }
                }
                if (!waited) {
                    dependency_wait();
                    dependents_may_start();                 // the CTA's part: behind a wait, as everywhere
                }
                waited = true;
                float c4[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = lane * 4 + e, i = i0 + r / G;
                    c4[e] = r < tile_rows && i < j.len ? lse2[(size_t)i0 * G + r] + age_exponent(j.len - 1 - i, a.nl2a) : INFINITY;
                }
                if (!__shfl_sync(0xffffffffu, ok, 0)) break;
                *reinterpret_cast<float4 *>(&sh->cbuf[qt % kScoreRing][lane * 4]) = make_float4(c4[0], c4[1], c4[2], c4[3]);
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh->c_ready[qt % kScoreRing]);
            }
        }
        if (!waited) {
            dependency_wait();
            dependents_may_start();
        }
        if (lane == 0 && *abort_flag) {
            int dummy = 0;
            for (int k = max(0, qt - kScoreStages); k < qt; ++k) mbar_wait(&sh->q_full[k % kScoreStages], (k / kScoreStages) & 1, &dummy);
            if (n > 0) mbar_wait(&sh->k_full, (n - 1) & 1, &dummy);
        }
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = make_idesc(ab_fmt, kBlk, kBlk, 0, 0);
            const uint64_t k_desc = kmajor_desc(smem_u32(Ks));
            const uint64_t q_desc = kmajor_desc(smem_u32(Qs));
            int qt = 0, n = 0;
            for (long long w = w0; w < w1 && !*abort_flag; ++n) {
                const Job j = next_job(w);
                wait(&sh->k_full, n & 1);
                for (int t = 0; t < j.nq; ++t, ++qt) {
                    const int s = qt % kScoreStages, acc = qt & 1;
                    wait(&sh->q_full[s], (qt / kScoreStages) & 1);
                    // from the third product on the epilogue is waited for, which waits for the attention: a time
                    // that no limit of a wait may hold
                    if (qt == 2) dependency_wait();
                    wait(&sh->acc_empty[acc], ((qt >> 1) & 1) ^ 1);
                    tc_fence_after_sync();
                    issue_qk<D>(tmem_base + acc * kBlk, k_desc, q_desc + s * (uint64_t)(kTileBytes >> 4), idesc);
                    umma_commit(&sh->q_empty[s]);
                    umma_commit(&sh->acc_full[acc]);
                }
                umma_commit(&sh->k_empty);
            }
        }
    } else {
        const int quarter = warp & 3, hsel = (warp - 2) >> 2;
        const int key = quarter * 32 + lane;
        int qt = 0;
        for (long long w = w0; w < w1;) {
            const Job j = next_job(w);
            const int slot = j.j0 + key;
            float *dst = nullptr, old = 0.f;
            if (j.part < 0 && hsel == 0 && slot < j.used) {
                const int page = page_for_write(pv, pv.table + (size_t)j.b * pv.max_pages, slot);
                if (page >= 0) {
                    dst = pv.scores + pool_row(pv, page, j.h, slot);
                    old = *dst;
                }
            }
            if (qt == 0) dependency_wait();                 // as the producer does: not a wait with a limit
            float sum = 0.f;
            for (int t = 0; t < j.nq; ++t, ++qt) {
                const int acc = qt & 1, i0 = (j.q0 + t) * tile_tokens;
                wait(&sh->c_ready[qt % kScoreRing], (qt / kScoreRing) & 1);
                wait(&sh->acc_full[acc], (qt >> 1) & 1);
                tc_fence_after_sync();
                const float *cb = sh->cbuf[qt % kScoreRing] + hsel * 64;
                uint32_t r[2][32];
                const uint32_t addr = tmem_base + acc * kBlk + hsel * 64 + ((uint32_t)(quarter * 32) << 16);
                tmem_ld32(addr, r[0]);
                tmem_ld32(addr + 32, r[1]);
                tmem_wait_ld();
                tc_fence_before_sync();
                mbar_arrive(&sh->acc_empty[acc]);
                // tiles with rows that do not see the slot, or with rows past the chunk (whose queries may
                // hold anything), take the test; the others run the bare multiply-add / exponential / add
                if (j.j0 + kBlk > j.past + i0 + 1 || i0 + tile_tokens > j.len)
                    sum += strip_sum<true>(r, cb, pv.sl2, max(0, slot - j.past - i0) * G - hsel * 64,
                                           min(tile_rows, (j.len - i0) * G) - hsel * 64);
                else
                    sum += strip_sum<false>(r, cb, pv.sl2, 0, 0);
            }
            if (hsel == 1) sh->part[key] = sum;
            named_barrier(1, 256);
            if (dst && !*abort_flag) *dst = fmaf(old, ex2_approx(-age_exponent(j.len, a.nl2a)), sum + sh->part[key]);
            if (j.part >= 0 && hsel == 0 && A2SF_IN_RANGE(j.part, 2 * kScoreCtas, kDbgPagedTc)) ws.score_parts[(size_t)j.part * kBlk + key] = sum + sh->part[key];
            named_barrier(1, 256);                          // read before the next item writes
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, 256);
    }
    if (threadIdx.x == 0 && sh->abort_flag) *pv.status = A2SF_ERR_TIMEOUT;
}

// Block k: the key tile that the cut before CTA k's share goes through, if it is the tile's first cut.
__global__ void __launch_bounds__(kBlk)
paged_score_join_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ TcWs ws)
{
    __shared__ long long prefix[A2SF_PAGED_MAX_SEQUENCES + 1];
    const PagedView &pv = a.pv;
    score_prefix(prefix, pv, a.nl2a, kBlk / 32);
    const long long total = pv.H * prefix[pv.B], share = (total + kScoreCtas - 1) / kScoreCtas;
    const int k = blockIdx.x + 1;
    const long long w = k * share;
    ScorePos at = {};
    SeqRows seq = {};
    bool mine = w < total;
    if (mine) {
        at = score_pos(pv, a.nl2a, prefix, w);
        seq = seq_rows(pv, a.nl2a, at.b);
        mine = at.begins < w && at.begins >= w - share;
    }
    const int slot = at.kt * kBlk + threadIdx.x;
    float *dst = nullptr, old = 0.f;
    if (mine && slot < seq.past + seq.len) {
        const int page = page_for_write(pv, pv.table + (size_t)at.b * pv.max_pages, slot);
        if (page >= 0) {
            dst = pv.scores + pool_row(pv, page, at.h, slot);
            old = *dst;
        }
    }
    dependency_wait();
    if (!dst) return;
    const int last = (int)((at.begins + seq.rows_of(at.kt) - 1) / share);
    float sum = ws.score_parts[(size_t)(2 * (k - 1) + 1) * kBlk + threadIdx.x];
    for (int c = k; c <= last; ++c) sum += ws.score_parts[(size_t)(2 * c) * kBlk + threadIdx.x];
    *dst = fmaf(old, ex2_approx(-age_exponent(seq.len, a.nl2a)), sum);
}

size_t pad(size_t x) { return (x + 255) / 256 * 256; }

TcWs carve(const PagedView &pv, void *mem, size_t *bytes)
{
    TcWs w;
    const int tile_tokens = kBlk / pv.G;
    // a chunk of one row tile needs no second stream
    w.pair_tokens = 2 * tile_tokens;
    w.pairs = (pv.c + w.pair_tokens - 1) / w.pair_tokens;
    w.part_rows = pv.c <= tile_tokens ? kBlk : 2 * kBlk;
    const size_t U = (size_t)pv.B * pv.H, items = (size_t)pv.B * w.pairs;
    const size_t cap_tiles = (((size_t)pv.max_pages << pv.ps_shift) + kBlk - 1) / kBlk;
    w.max_items = (int)(items + kMaxParts);
    w.direct = cap_tiles <= kDirectTiles && items * pv.H < 0x7fffffff;
    w.whole_scores = (pv.c + tile_tokens - 1) / tile_tokens <= kWholeRows;
    size_t parts = w.direct ? 0 : items * pv.H * ((cap_tiles + kMinPiece - 1) / kMinPiece);
    if (parts > kMaxParts) parts = kMaxParts;
    w.parts = (int)parts;
    char *base = static_cast<char *>(mem);
    size_t off = 0;
    w.lse2 = reinterpret_cast<float *>(base + off); off += pad(U * pv.c * pv.G * 4);
    w.head = reinterpret_cast<PlanHead *>(base + off); off += 256;
    w.items = reinterpret_cast<Item *>(base + off); off += pad(w.max_items * sizeof(Item));
    w.merges = reinterpret_cast<Merge *>(base + off); off += pad(items * sizeof(Merge));
    w.part_ml = reinterpret_cast<float2 *>(base + off); off += pad(parts * w.part_rows * 8);
    w.part_o = reinterpret_cast<float *>(base + off); off += pad(parts * w.part_rows * pv.d * 4);
    w.score_parts = reinterpret_cast<float *>(base + off); off += pad((size_t)2 * kScoreCtas * kBlk * 4);
    if (bytes) *bytes = off;
    return w;
}

template <typename T, int D>
cudaError_t launch(int dtype, const AttendArgs &a, cudaStream_t s)
{
    cudaError_t e = allow_dynamic_smem<paged_attn_tc_kernel<T, D>>(attn_smem<D>());
    if (e == cudaSuccess) e = allow_dynamic_smem<paged_score_tc_kernel<D>>(score_smem<D>());
    if (e != cudaSuccess) return e;
    CUtensorMap mq, mk, mv;
    const int box = a.pv.ps;
    if (!make_query_map(&mq, dtype, a.q, a.pv, a.sq) || !make_pool_map(&mk, dtype, a.pv.k, a.pv, box) ||
        !make_pool_map(&mv, dtype, a.pv.v, a.pv, box))
        return cudaErrorInvalidValue;
    const TcWs ws = carve(a.pv, a.ws, nullptr);
    if ((long long)ws.max_items * a.pv.H > 0x7fffffffll) return cudaErrorInvalidValue;
    if (!ws.direct) {
        if ((e = launch_chained(paged_plan_kernel, 1, kPlanThreads, 0, s, a.pv, ws)) != cudaSuccess) return e;
        count_launch();
    }
    e = launch_chained(paged_attn_tc_kernel<T, D>, kSms, kAttnThreads, attn_smem<D>(), s, mq, mk, mv, a, ws);
    if (e != cudaSuccess) return e;
    count_launch();
    if (!ws.direct) {
        if ((e = launch_chained(paged_merge_kernel<T, D>, 4 * kSms, kMergeThreads, 0, s, a, ws)) != cudaSuccess) return e;
        count_launch();
    }
    if (!a.scores) return cudaSuccess;
    e = launch_chained(paged_score_tc_kernel<D>, kScoreCtas, kScoreThreads, score_smem<D>(), s, mq, mk, a, ws, dtype == A2SF_BF16 ? 1 : 0);
    if (e != cudaSuccess) return e;
    count_launch();
    if (ws.whole_scores) return cudaSuccess;
    if ((e = launch_chained(paged_score_join_kernel, kScoreCtas - 1, kBlk, 0, s, a, ws)) != cudaSuccess) return e;
    count_launch();
    return cudaSuccess;
}

}  // namespace

size_t attend_tc_ws_bytes(const PagedView &pv)
{
    size_t bytes = 0;
    carve(pv, nullptr, &bytes);
    return bytes;
}

cudaError_t launch_attend_tc(int dtype, const AttendArgs &a, cudaStream_t s)
{
    const bool wide = a.pv.d == 128;
    if (dtype == A2SF_BF16) return wide ? launch<__nv_bfloat16, 128>(dtype, a, s) : launch<__nv_bfloat16, 64>(dtype, a, s);
    return wide ? launch<__half, 128>(dtype, a, s) : launch<__half, 64>(dtype, a, s);
}

}  // namespace a2sf
