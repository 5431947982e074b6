// Back to the budget: which slots of a head stay, and the rows that have to move for it.
//
// One CTA per (sequence, K/V head).  Of n slots, n - M leave: the smallest under (score, position, slot) among
// those outside the recent window.  A radix search narrows the score at which the cut falls, 8 bits at a
// time, and then the position -- many scores are equal when alpha = 0 or a chunk was just appended -- until at
// most kShort slots are left to decide about; those are ranked directly.  Usually two digits do; bits that all
// candidates share are passed over (a cut among 950 equal scores: 35 us digit by digit, 28 so).  The survivors
// become a bit mask, and a scan over it in slot order lists the moves: integer work, exact, the same on
// every run.  In place only the survivors above M move, into the holes below M: at most min(M, n - M) rows.
//
// Bound by memory -- 8 bytes per slot for the decision, two rows read and written per move -- where there are many
// heads: then a CTA moves its own rows, and one CTA's search hides behind the others' copies.  Where there are
// few, long moves are left to a kernel that spreads them over the whole device.  Every CTA reads past and start, so
// where past_out or start_out is one of them they change in a kernel behind.
#include <type_traits>

#include "paged.cuh"

namespace a2sf {

A2SF_DEBUG_TRANSLATION_UNIT(paged_evict)

namespace {

constexpr int kCached = 16384;       // slots whose score key and position fit in shared memory
constexpr int kMaskWords = 1024;     // survivors' mask: 32768 slots; beyond, it is worked out again where it is needed
constexpr int kShort = 64;           // slots that are ranked directly
constexpr int kFewDrops = 8;         // as many slots leave one minimum after the other
constexpr int kInline = 64;          // moves that the searching CTA makes itself in any case
constexpr int kDirect = 256;         // ... and all that a call can have, where nothing else asks for a second kernel
constexpr int kWide = 512;           // threads of a searching CTA where heads are few
constexpr int kRows = 4;             // rows of a lane group in flight

struct EvictArgs {
    PagedView pv;
    int M, R;
    const int32_t *dst_table;        // [B][dst_max_pages] or nullptr (in place)
    int dst_max_pages;
    int32_t *past_out, *start_out;
    int32_t *from, *to;              // [U][M] slot lists (to: in place only)
    int32_t *moves;                  // [U]
    int32_t *ends;                   // [B][2] new past, new start
    int blocks;                      // of the move kernel, per unit; 0: every CTA moves its own rows
    bool direct;                     // there is no move kernel: the lengths change here
};

// Order-preserving key of a score, -0 like +0, every NaN behind infinity; kNoKey stands for a slot that is no
// candidate (inside the recent window, or behind the last one).
constexpr unsigned kNoKey = 0xffffffffu;
__device__ __forceinline__ unsigned score_key(float s)
{
    const unsigned bits = __float_as_uint(s + 0.f);
    const unsigned key = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
    return s != s ? 0xfffffffeu : key;
}

template <int NT> struct SelShared {
    static constexpr int kSelWarps = NT / 32;
    int hist[256];
    int warp_tot[2][kSelWarps + 1];
    unsigned prefix, all_or, all_and;
    int rank, equal, total, count;
    unsigned list_key[kShort], list_pos[kShort];
    int list_slot[kShort];
    unsigned thr_key, thr_pos;
    int thr_slot;
    unsigned long long low_key[2][kSelWarps];
    int low_slot[2][kSelWarps], leaving[kFewDrops];
    unsigned mask[kMaskWords];
};

// Exclusive scan of one int per warp (lane 0 holds it) over the CTA's warps, for `which`.
template <int NT> __device__ __forceinline__ int warps_excl_scan(SelShared<NT> &sh, int which, int v, int &total)
{
    constexpr int kSelWarps = NT / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0) sh.warp_tot[which][warp] = v;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kSelWarps; ++w) {
        const int t = sh.warp_tot[which][w];
        before += w < warp ? t : 0;
        total += t;
    }
    return before;
}

// Rows k0, k0 + step, .. of a unit's list; a group of ROW_BYTES / 16 lanes copies one row of K and of V.
template <int ROW_BYTES>
__device__ __forceinline__ void move_rows(const EvictArgs &a, int u, int b, int h, int moves, int group, int groups)
{
    constexpr int LPR = ROW_BYTES / 16;
    const int part = threadIdx.x % LPR;
    const bool fresh = a.dst_table != nullptr;
    const int32_t *from_row = a.pv.table + (size_t)b * a.pv.max_pages;
    const int32_t *to_row = fresh ? a.dst_table + (size_t)b * a.dst_max_pages : from_row;
    // kRows rows in flight: a move is a chain of three loads (list, page, row)
    for (int k0 = group; k0 < moves; k0 += groups * kRows) {
        int64_t s[kRows], t[kRows];
        uint4 kv[kRows], vv[kRows];
        float sc[kRows];
        int32_t ps[kRows];
#pragma unroll
        for (int x = 0; x < kRows; ++x) {
            const int k = k0 + x * groups;
            t[x] = -1;
            if (k >= moves || !A2SF_IN_RANGE(k, a.M, kDbgPagedEvict)) continue;
            const int src = a.from[(size_t)u * a.M + k], dst = fresh ? k : a.to[(size_t)u * a.M + k];
            const int to_page = page_for_write(a.pv, to_row, dst);
            s[x] = pool_row(a.pv, page_for_read(a.pv, from_row, src), h, src);
            if (to_page >= 0) t[x] = pool_row(a.pv, to_page, h, dst);
        }
#pragma unroll
        for (int x = 0; x < kRows; ++x) {
            if (t[x] < 0) continue;
            kv[x] = ld_stream16_rw(a.pv.k + s[x] * ROW_BYTES + part * 16);
            vv[x] = ld_stream16_rw(a.pv.v + s[x] * ROW_BYTES + part * 16);
            if (part == 0) { sc[x] = a.pv.scores[s[x]]; ps[x] = a.pv.positions[s[x]]; }
        }
#pragma unroll
        for (int x = 0; x < kRows; ++x) {
            if (t[x] < 0) continue;
            __stcs(reinterpret_cast<uint4 *>(a.pv.k + t[x] * ROW_BYTES + part * 16), kv[x]);
            __stcs(reinterpret_cast<uint4 *>(a.pv.v + t[x] * ROW_BYTES + part * 16), vv[x]);
            if (part == 0) { a.pv.scores[t[x]] = sc[x]; a.pv.positions[t[x]] = ps[x]; }
        }
    }
}

template <int ROW_BYTES, int kSelThreads>
__global__ void __launch_bounds__(kSelThreads, kSelThreads == 256 ? 3 : 1)
paged_select_kernel(const __grid_constant__ EvictArgs a, int cached)
{
    constexpr int kSelWarps = kSelThreads / 32;
    extern __shared__ __align__(16) unsigned cache[];   // [cached] keys, [cached] positions
    __shared__ SelShared<kSelThreads> sh;
    const int u = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = u / a.pv.H, h = u - b * a.pv.H;
    dependency_wait();
    dependents_may_start();
    const SeqState st = seq_state(a.pv, b);
    const int n = st.past + st.len, M = a.M;
    const int start = a.pv.start ? a.pv.start[b] : st.past;
    const long long newest = (long long)start + st.len - a.R;       // positions from here on are recent
    const int32_t *table = a.pv.table + (size_t)b * a.pv.max_pages;
    if (h == 0 && tid == 0) {
        (a.direct ? a.past_out[b] : a.ends[2 * b]) = min(n, M);
        (a.direct ? a.start_out[b] : a.ends[2 * b + 1]) = start + st.len;
    }
    const bool fresh = a.dst_table != nullptr;
    const int drop = n - M;
    int32_t *from = a.from + (size_t)u * M, *to = a.to + (size_t)u * M;
    int moves = fresh ? min(n, M) : 0;
    if (drop > 0) {
        unsigned *keys = cache;
        int32_t *poss = reinterpret_cast<int32_t *>(cache + cached);
        // Slots leave from among those outside the window.  Positions given twice can make the window
        // hold more than the budget; then all others leave and the window is ranked itself.
        bool from_recent = false;
        // four slots j .. j+3 (j a multiple of 4: they share a page)
        auto fetch = [&](int j, uint4 &k, int4 &p) {
            const int64_t row = pool_row(a.pv, page_for_read(a.pv, table, j), h, j);
            const float4 sc = *reinterpret_cast<const float4 *>(a.pv.scores + row);
            p = *reinterpret_cast<const int4 *>(a.pv.positions + row);
            auto key = [&](float s, int pos, int x) { return x < n && ((long long)pos >= newest) == from_recent ? score_key(s) : kNoKey; };
            k = make_uint4(key(sc.x, p.x, j), key(sc.y, p.y, j + 1), key(sc.z, p.z, j + 2), key(sc.w, p.w, j + 3));
        };
        auto fill = [&] {
#pragma unroll 2
            for (int j = 4 * tid; j < n && j < cached; j += 4 * kSelThreads) {
                uint4 k;
                int4 p;
                fetch(j, k, p);
                *reinterpret_cast<uint4 *>(keys + j) = k;
                *reinterpret_cast<int4 *>(poss + j) = p;
            }
        };
        auto keys4 = [&](int j, unsigned (&k)[4]) {
            uint4 v;
            int4 p;
            if (j < cached) v = *reinterpret_cast<const uint4 *>(keys + j);
            else fetch(j, v, p);
            k[0] = v.x; k[1] = v.y; k[2] = v.z; k[3] = v.w;
        };
        auto key_at = [&](int j) -> unsigned {
            if (j < cached) return keys[j];
            unsigned k[4];
            keys4(j & ~3, k);
            return j & 2 ? (j & 1 ? k[3] : k[2]) : (j & 1 ? k[1] : k[0]);
        };
        auto pos_at = [&](int j) -> unsigned {           // signed positions in unsigned order
            const int32_t p = j < cached ? poss[j] : a.pv.positions[pool_row(a.pv, page_for_read(a.pv, table, j), h, j)];
            return (unsigned)p ^ 0x80000000u;
        };
        fill();
        // A generation step lets a few slots leave: the minimum under (score, position, slot), as often as needed.
        bool found = drop <= kFewDrops && n <= cached;
        if (found) {
            __syncthreads();                             // keys and positions are in place
            unsigned long long gone = 0, low;            // the last one that left, this thread's lowest behind it
            int gone_slot = -1, low_slot;
            auto lowest = [&] {
                low = ~0ull;
                low_slot = 0x7fffffff;
                for (int j = 4 * tid; j < n; j += 4 * kSelThreads) {
                    const uint4 k = *reinterpret_cast<const uint4 *>(keys + j);
                    const int4 q = *reinterpret_cast<const int4 *>(poss + j);
                    auto take = [&](unsigned key, int pos, int slot) {
                        const unsigned long long x = (unsigned long long)key << 32 | ((unsigned)pos ^ 0x80000000u);
                        if (key != kNoKey && (x > gone || (x == gone && slot > gone_slot)) && x < low) { low = x; low_slot = slot; }
                    };
                    take(k.x, q.x, j); take(k.y, q.y, j + 1); take(k.z, q.z, j + 2); take(k.w, q.w, j + 3);
                }
            };
            lowest();
            for (int r = 0; r < drop && found; ++r) {
                unsigned long long x = low;
                int slot = low_slot;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    const unsigned long long y = __shfl_xor_sync(0xffffffffu, x, o);
                    const int z = __shfl_xor_sync(0xffffffffu, slot, o);
                    if (y < x || (y == x && z < slot)) { x = y; slot = z; }
                }
                if (lane == 0) { sh.low_key[r & 1][warp] = x; sh.low_slot[r & 1][warp] = slot; }
                __syncthreads();
                x = sh.low_key[r & 1][0];
                slot = sh.low_slot[r & 1][0];
#pragma unroll
                for (int w = 1; w < kSelWarps; ++w) {
                    const unsigned long long y = sh.low_key[r & 1][w];
                    const int z = sh.low_slot[r & 1][w];
                    if (y < x || (y == x && z < slot)) { x = y; slot = z; }
                }
                found = x != ~0ull;                      // else too few candidates: the general search sorts that out
                gone = x;
                gone_slot = slot;
                if (tid == 0) sh.leaving[r] = slot;
                if (slot == low_slot && r + 1 < drop) lowest();
            }
            if (tid == 0) { sh.thr_key = (unsigned)(gone >> 32); sh.thr_pos = (unsigned)gone; sh.thr_slot = gone_slot; }
            __syncthreads();
        }
        const bool listed = found && !fresh;
        if (listed) {
            // in place, holes and survivors from M on follow from the few that leave
            int rank_of = 0, others = 0;
            bool leaves = false;
            if (tid < drop) {
                const int hole = sh.leaving[tid], up = M + tid;
                for (int r = 0; r < drop; ++r) {
                    rank_of += sh.leaving[r] < hole;
                    others += sh.leaving[r] >= M && sh.leaving[r] < up;
                    leaves |= sh.leaving[r] == up;
                }
                if (hole < M && A2SF_IN_RANGE(rank_of, M, kDbgPagedEvict)) to[rank_of] = hole;
                if (!leaves && A2SF_IN_RANGE(tid - others, M, kDbgPagedEvict)) from[tid - others] = up;
            }
            for (int r = 0; r < drop; ++r) moves += sh.leaving[r] < M;
        }
        if (!found) {
            // The threshold's score is found from the top, eight bits at a time, then its position and its slot (part 0, 1, 2).  A
            // candidate is in question while it agrees with all that is known; `open` are the bits of the part that are not.
            unsigned thr[3] = {0u, 0u, 0u}, open = 0xffffffffu;
            int part = 0, shift = 24;
            auto value = [&](unsigned k, int j) { return part == 0 ? k : part == 1 ? pos_at(j) : (unsigned)j; };
            auto agrees = [&](unsigned k, int j) {
                if (k == kNoKey || ((k ^ thr[0]) & (part == 0 ? ~open : 0xffffffffu)) != 0u) return false;
                if (part == 0) return true;
                return ((pos_at(j) ^ thr[1]) & (part == 1 ? ~open : 0xffffffffu)) == 0u && (part < 2 || (((unsigned)j ^ thr[2]) & ~open) == 0u);
            };
            int rank = drop, total = n;                      // 1-based rank of the last one to leave
            for (;;) {
                if (tid < 256) sh.hist[tid] = 0;
                if (tid == 0) { sh.count = 0; sh.all_or = 0u; sh.all_and = 0xffffffffu; }
                __syncthreads();
                for (int j = 4 * tid; j < n; j += 4 * kSelThreads) {
                    unsigned k[4];
                    keys4(j, k);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (agrees(k[e], j + e)) atomicAdd(&sh.hist[(value(k[e], j + e) >> shift) & 255u], 1);
                }
                __syncthreads();
                if (warp == 0) {                             // 8 bins a lane, then the lane that holds the rank
                    int c[8], sum = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) { c[e] = sh.hist[lane * 8 + e]; sum += c[e]; }
                    int incl = sum;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const int x = __shfl_up_sync(0xffffffffu, incl, o);
                        if (lane >= o) incl += x;
                    }
                    int before = incl - sum;
                    if (before < rank && rank <= incl) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            if (before < rank && rank <= before + c[e]) {
                                sh.prefix = (unsigned)(lane * 8 + e) << shift;
                                sh.rank = rank - before;
                                sh.equal = c[e];
                            }
                            before += c[e];
                        }
                    }
                    if (lane == 31) sh.total = incl;
                }
                __syncthreads();
                if (part == 0 && shift == 24 && !from_recent && sh.total < drop) {
                    from_recent = true;
                    rank = drop - sh.total;
                    fill();
                    __syncthreads();
                    continue;
                }
                thr[part] |= sh.prefix;
                open = (1u << shift) - 1u;
                rank = sh.rank;
                const int equal = sh.equal;
                if (equal <= kShort || (part == 2 && open == 0u)) break;     // all bits of the slot tell all of them apart
                // Eight bits that told little (a quarter or more still agrees: equal scores, most of all) say that the next eight
                // may not either: then a look at which bits differ at all, one pass without atomics, finds the ones that do.
                bool look = 4 * equal >= total;
                total = equal;
                shift = shift > 8 ? shift - 8 : 0;
                for (;;) {
                    if (open == 0u && part < 2) { ++part; open = 0xffffffffu; look = true; }
                    if (!look) break;
                    unsigned any = 0u, all = 0xffffffffu;
                    for (int j = 4 * tid; j < n; j += 4 * kSelThreads) {
                        unsigned k[4];
                        keys4(j, k);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (agrees(k[e], j + e)) { const unsigned v = value(k[e], j + e); any |= v; all &= v; }
                    }
                    any = __reduce_or_sync(0xffffffffu, any);
                    all = __reduce_and_sync(0xffffffffu, all);
                    if (lane == 0) { atomicOr(&sh.all_or, any); atomicAnd(&sh.all_and, all); }
                    __syncthreads();
                    any = sh.all_or;
                    const unsigned differ = (any ^ sh.all_and) & open;
                    const int top = 32 - __clz((int)differ); // bits from here on are the same
                    open = top == 32 ? 0xffffffffu : (1u << top) - 1u;
                    thr[part] = any & ~open;
                    shift = top > 8 ? top - 8 : 0;
                    look = false;
                    __syncthreads();
                    if (open == 0u && tid == 0) { sh.all_or = 0u; sh.all_and = 0xffffffffu; }
                    if (open == 0u) __syncthreads();
                }
            }
            // the slots that agree so far, ranked by (score, position, slot)
            const int m = min(sh.equal, kShort);
            for (int j = 4 * tid; j < n; j += 4 * kSelThreads) {
                unsigned k[4];
                keys4(j, k);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (!agrees(k[e], j + e)) continue;
                    const int x = atomicAdd(&sh.count, 1);
                    if (A2SF_IN_RANGE(x, kShort, kDbgPagedEvict) && x < kShort) { sh.list_key[x] = k[e]; sh.list_pos[x] = pos_at(j + e); sh.list_slot[x] = j + e; }
                }
            }
            __syncthreads();
            if (tid < m) {
                const unsigned k = sh.list_key[tid], p = sh.list_pos[tid];
                const int s = sh.list_slot[tid];
                int less = 0;
                for (int x = 0; x < m; ++x) {
                    const unsigned k2 = sh.list_key[x], p2 = sh.list_pos[x];
                    less += k2 < k || (k2 == k && (p2 < p || (p2 == p && sh.list_slot[x] < s)));
                }
                if (less == rank - 1) { sh.thr_key = k; sh.thr_pos = p; sh.thr_slot = s; }
            }
            __syncthreads();
        }
        if (!listed) {
            const unsigned tk = sh.thr_key, tp = sh.thr_pos;
            const int ts = sh.thr_slot;
            auto stays = [&](int j) {
                const unsigned k = key_at(j);
                if (k == kNoKey) return !from_recent;
                if (k != tk) return k > tk;
                const unsigned p = pos_at(j);
                return p != tp ? p > tp : j > ts;
            };
            // every warp takes a contiguous range of slots, 32 at a time: mask and counts, scan over the warps, list
            const int per = ((n + kSelWarps - 1) / kSelWarps + 31) / 32 * 32;
            const int w0 = min(n, warp * per), w1 = min(n, w0 + per);
            auto low = [&](int j0) { return j0 + 32 <= M ? 0xffffffffu : j0 >= M ? 0u : (1u << (M - j0)) - 1u; };
            int stay_lo = 0, stay_hi = 0;                    // survivors below / from slot M on
            for (int j0 = w0; j0 < w1; j0 += 32) {
                const unsigned s = __ballot_sync(0xffffffffu, j0 + lane < w1 && stays(j0 + lane));
                if (lane == 0 && j0 / 32 < kMaskWords) sh.mask[j0 / 32] = s;
                stay_lo += __popc(s & low(j0));
                stay_hi += __popc(s & ~low(j0));
            }
            int total_lo, total_hi;
            const int lo0 = warps_excl_scan(sh, 0, stay_lo, total_lo), hi0 = warps_excl_scan(sh, 1, stay_hi, total_hi);
            auto mask_of = [&](int j0) -> unsigned {
                return j0 / 32 < kMaskWords ? sh.mask[j0 / 32] : __ballot_sync(0xffffffffu, j0 + lane < w1 && stays(j0 + lane));
            };
            const unsigned lt = (1u << lane) - 1u;
            if (fresh) {
                int at = lo0 + hi0;
                for (int j0 = w0; j0 < w1; j0 += 32) {
                    const unsigned s = mask_of(j0);
                    const int k = at + __popc(s & lt);
                    if ((s >> lane & 1) && A2SF_IN_RANGE(k, M, kDbgPagedEvict) && k < M) from[k] = j0 + lane;
                    at += __popc(s);
                }
            } else {
                int hole = min(w0, M) - lo0, src = hi0;      // holes and survivors before this warp's range
                for (int j0 = w0; j0 < w1; j0 += 32) {
                    const unsigned s = mask_of(j0);
                    const unsigned in = j0 + 32 <= w1 ? 0xffffffffu : (1u << (w1 - j0)) - 1u;
                    const unsigned lo = low(j0), holes = in & lo & ~s, ups = s & ~lo;
                    const int kh = hole + __popc(holes & lt), ks = src + __popc(ups & lt);
                    if ((holes >> lane & 1) && A2SF_IN_RANGE(kh, M, kDbgPagedEvict) && kh < M) to[kh] = j0 + lane;
                    if ((ups >> lane & 1) && A2SF_IN_RANGE(ks, M, kDbgPagedEvict) && ks < M) from[ks] = j0 + lane;
                    hole += __popc(holes);
                    src += __popc(ups);
                }
                moves = total_hi;
            }
        }
    } else if (fresh) {
        for (int j = tid; j < n; j += kSelThreads) from[j] = j;
    }
    const bool here = a.blocks == 0 || moves <= kInline;
    if (tid == 0) a.moves[u] = here ? 0 : moves;
    if (!here) return;
    __syncthreads();                                     // the lists, written by this CTA
    constexpr int LPR = ROW_BYTES / 16;
    move_rows<ROW_BYTES>(a, u, b, h, moves, tid / LPR, kSelThreads / LPR);
}

constexpr int kMoveThreads = 256;

// Long moves of few heads, and the new lengths.
template <int ROW_BYTES>
__global__ void __launch_bounds__(kMoveThreads)
paged_move_kernel(const __grid_constant__ EvictArgs a)
{
    dependency_wait();
    for (int b = blockIdx.x * kMoveThreads + threadIdx.x; b < a.pv.B; b += gridDim.x * kMoveThreads) {
        a.past_out[b] = a.ends[2 * b];
        a.start_out[b] = a.ends[2 * b + 1];
    }
    if (a.blocks == 0) return;
    constexpr int LPR = ROW_BYTES / 16, RPB = kMoveThreads / LPR;
    const int u = blockIdx.x / a.blocks, y = blockIdx.x - u * a.blocks, b = u / a.pv.H, h = u - b * a.pv.H;
    move_rows<ROW_BYTES>(a, u, b, h, a.moves[u], y * RPB + threadIdx.x / LPR, a.blocks * RPB);
}

size_t pad(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

size_t evict_ws_bytes(size_t units, int budget)
{
    return 2 * pad(units * (size_t)budget * 4) + 2 * pad(units * 8);
}

cudaError_t launch_evict(int elem_bytes, const PagedView &pv, int budget, int recent, const int32_t *dst_table,
                         int dst_max_pages, int32_t *past_out, int32_t *start_out, void *ws, cudaStream_t s)
{
    const size_t units = (size_t)pv.B * pv.H;
    EvictArgs a;
    a.pv = pv; a.M = budget; a.R = recent;
    a.dst_table = dst_table; a.dst_max_pages = dst_max_pages;
    a.past_out = past_out; a.start_out = start_out;
    char *w = static_cast<char *>(ws);
    a.from = reinterpret_cast<int32_t *>(w); w += pad(units * (size_t)budget * 4);
    a.to = reinterpret_cast<int32_t *>(w); w += pad(units * (size_t)budget * 4);
    a.moves = reinterpret_cast<int32_t *>(w); w += pad(units * 8);
    a.ends = reinterpret_cast<int32_t *>(w);
    const int cap = pv.max_pages << pv.ps_shift;
    const int cached = cap < kCached ? cap : kCached;
    const size_t smem = (size_t)cached * 8;
    const int row_bytes = pv.d * elem_bytes, rpb = kMoveThreads / (row_bytes / 16);
    // from two CTAs per SM on the heads fill the device with their own copies
    long long blocks = 0;
    if (units < 2 * (size_t)device_sm_count()) {
        blocks = ((budget < cap ? budget : cap) + rpb * kRows - 1) / (rpb * kRows);
        const long long want = (16ll * device_sm_count() + (long long)units - 1) / (long long)units;
        if (blocks > want) blocks = want;
    }
    // New lengths that do not lie where the old ones are read need no second kernel for their own sake; and so many moves
    // at most are no more than it costs (1 us: 3 heads from 304 slots to 40, 12.1 us with it, 10.9 without).
    const int bound = dst_table ? (budget < cap ? budget : cap) : (cap - budget < budget ? cap - budget : budget);
    auto apart = [&](const int32_t *out, const int32_t *in) { return !in || out + pv.B <= in || in + pv.B <= out; };
    a.direct = (blocks == 0 || bound <= kDirect) && apart(past_out, pv.past) && apart(past_out, pv.start) && apart(past_out, pv.lens) &&
               apart(start_out, pv.past) && apart(start_out, pv.start) && apart(start_out, pv.lens);
    if (a.direct) blocks = 0;
    a.blocks = (int)blocks;
    const unsigned grid = blocks ? (unsigned)(units * blocks) : 1u;
    auto run = [&](auto select, int threads, auto move) -> cudaError_t {
        cudaError_t e = launch_chained(select, (unsigned)units, threads, smem, s, a, cached);
        if (e != cudaSuccess) return e;
        count_launch();
        if (a.direct) return cudaSuccess;
        e = launch_chained(move, grid, kMoveThreads, 0, s, a);
        if (e == cudaSuccess) count_launch();
        return e;
    };
    // static shared memory counts towards the 48 KB that need no permission: it is asked for the most, whatever this call takes
    constexpr size_t most = (size_t)kCached * 8;
    // Twice the threads where every head has an SM to itself (21 heads, 17 of 3,237 slots leave: 28 us with 256 threads, 21 with
    // 512, 20 with 1024, which lose elsewhere; 69 heads, 3 of 4,330: 14.9 and 15.1).
    const bool wide = units <= (size_t)device_sm_count();
    auto pick = [&](auto rows) -> cudaError_t {
        constexpr int RB = decltype(rows)::value;
        cudaError_t e = wide ? allow_dynamic_smem<paged_select_kernel<RB, kWide>>(most) : allow_dynamic_smem<paged_select_kernel<RB, 256>>(most);
        if (e != cudaSuccess) return e;
        return wide ? run(paged_select_kernel<RB, kWide>, kWide, paged_move_kernel<RB>) : run(paged_select_kernel<RB, 256>, 256, paged_move_kernel<RB>);
    };
    switch (row_bytes) {
    case 128: return pick(std::integral_constant<int, 128>{});
    case 256: return pick(std::integral_constant<int, 256>{});
    default: return pick(std::integral_constant<int, 512>{});
    }
}

}  // namespace a2sf
