// Back to the budget: which slots of a head stay, and the rows that have to move for it.
//
//   select  one CTA per (sequence, K/V head).  Of n slots, n - M leave: those with the smallest
//           (score, position) among the slots outside the recent window.  A radix select over the 32
//           ordered score bits (8 at a time) finds the score at which the cut falls, a second one over
//           the positions decides among slots of exactly that score -- there are many when alpha = 0
//           or a chunk was just appended -- and a scan in slot order lists the moves.  Integer work:
//           exact, and the same on every run.
//   move    grid-wide copies of the listed rows (K, V, score, position).
// In place only the survivors above M move, into the holes below M: at most min(M, n - M) rows.
// Bound by memory: 8 bytes per slot for the decision, two rows read and written per move.
#include "paged.cuh"

namespace a2sf {

A2SF_DEBUG_TRANSLATION_UNIT(paged_evict)

namespace {

constexpr int kSelThreads = 512;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kCached = 16384;       // slots whose (score key, position) fit in shared memory

struct EvictArgs {
    PagedView pv;
    int M, R;
    const int32_t *dst_table;        // [B][dst_max_pages] or nullptr (in place)
    int dst_max_pages;
    int32_t *past_out, *start_out;
    int32_t *from, *to;              // [U][M] slot lists (to: in place only)
    int32_t *moves;                  // [U]
    int32_t *ends;                   // [B][2] new past, new start
    int blocks;                      // of the move kernel, per unit
};

// Order-preserving key of a score; every NaN sorts last, -0 like +0.
__device__ __forceinline__ unsigned score_key(float s)
{
    if (s != s) return 0xffffffffu;
    const unsigned bits = __float_as_uint(s + 0.f);
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

struct SelShared {
    int hist[256];
    int warp_tot[3][kSelWarps + 1];
    unsigned prefix;
    int rank, equal, ncand;
};

// Exclusive scan of one int per warp (lane 0 holds it) over the CTA's warps, for `which`.
__device__ __forceinline__ int warps_excl_scan(SelShared &sh, int which, int v, int &total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0) sh.warp_tot[which][warp] = v;
    __syncthreads();
    if (warp == which) {
        const int t = lane < kSelWarps ? sh.warp_tot[which][lane] : 0;
        int ti = t;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, ti, o);
            if (lane >= o) ti += x;
        }
        if (lane < kSelWarps) sh.warp_tot[which][lane] = ti - t;
        if (lane == 31) sh.warp_tot[which][kSelWarps] = ti;
    }
    __syncthreads();
    total = sh.warp_tot[which][kSelWarps];
    return sh.warp_tot[which][warp];
}

__global__ void __launch_bounds__(kSelThreads, 4)
paged_select_kernel(const __grid_constant__ EvictArgs a, int cached)
{
    extern __shared__ __align__(8) uint2 cache[];       // [cached] (key, position)
    __shared__ SelShared sh;
    const int u = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = u / a.pv.H, h = u - b * a.pv.H;
    dependents_may_start();
    const SeqState st = seq_state(a.pv, b);
    const int n = st.past + st.len, M = a.M;
    const int start = a.pv.start ? a.pv.start[b] : st.past;
    const long long newest = (long long)start + st.len - a.R;       // positions from here on are recent
    const int32_t *table = a.pv.table + (size_t)b * a.pv.max_pages;
    if (h == 0 && tid == 0) {
        a.ends[2 * b] = min(n, M);
        a.ends[2 * b + 1] = start + st.len;
    }
    const bool fresh = a.dst_table != nullptr;
    const int drop = n - M;
    int32_t *from = a.from + (size_t)u * M, *to = a.to + (size_t)u * M;
    if (drop <= 0) {
        if (fresh)
            for (int j = tid; j < n; j += kSelThreads) from[j] = j;
        if (tid == 0) a.moves[u] = fresh ? n : 0;
        return;
    }
    auto fetch = [&](int j) -> uint2 {
        const int64_t row = pool_row(a.pv, page_for_read(a.pv, table, j), h, j);
        return make_uint2(score_key(a.pv.scores[row]), (unsigned)a.pv.positions[row]);
    };
#pragma unroll 4
    for (int j = tid; j < min(n, cached); j += kSelThreads) cache[j] = fetch(j);
    auto item = [&](int j) -> uint2 { return j < cached ? cache[j] : fetch(j); };
    auto recent = [&](const uint2 &x) { return (long long)(int)x.y >= newest; };
    if (tid == 0) sh.ncand = 0;
    __syncthreads();
    int mine = 0;
    for (int j = tid; j < n; j += kSelThreads) mine += recent(item(j)) ? 0 : 1;
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (lane == 0) atomicAdd(&sh.ncand, mine);
    __syncthreads();
    // Slots leave from among those outside the window.  Positions given twice can make the window
    // hold more than the budget; then all others leave and the window is ranked itself.
    const bool from_recent = sh.ncand < drop;
    auto candidate = [&](const uint2 &x) { return recent(x) == from_recent; };
    int rank = from_recent ? drop - sh.ncand : drop;    // 1-based rank of the last one to leave
    // digits 0-3: the score; 4-7: the position, among slots of the threshold score
    unsigned thr_key = 0, thr_pos = 0;
    bool pos_needed = true;
    for (int digit = 0; digit < 8 && pos_needed; ++digit) {
        const int shift = 24 - 8 * (digit & 3);
        const unsigned above = (digit & 3) == 0 ? 0u : 0xffffffffu << (shift + 8);
        if (tid < 256) sh.hist[tid] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += kSelThreads) {
            const uint2 x = item(j);
            if (!candidate(x)) continue;
            const unsigned v = digit < 4 ? x.x : x.y ^ 0x80000000u;      // positions are signed
            const unsigned thr = digit < 4 ? thr_key : thr_pos;
            if (digit >= 4 && x.x != thr_key) continue;
            if ((v & above) == (thr & above)) atomicAdd(&sh.hist[(v >> shift) & 255u], 1);
        }
        __syncthreads();
        if (warp == 0) {                                 // 8 bins a lane, then the lane that holds the rank
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
                        break;
                    }
                    before += c[e];
                }
            }
        }
        __syncthreads();
        if (digit < 4) thr_key |= sh.prefix;
        else           thr_pos |= sh.prefix;
        rank = sh.rank;
        if (digit == 3) pos_needed = sh.equal != rank;   // all slots of that score leave: no second key
    }
    // leaves: candidates below (thr_key, thr_pos), and the first `rank` of those equal to it
    auto below = [&](const uint2 &x) {
        return candidate(x) && (x.x < thr_key || (pos_needed && x.x == thr_key && (x.y ^ 0x80000000u) < thr_pos));
    };
    auto equal = [&](const uint2 &x) {
        return candidate(x) && x.x == thr_key && (!pos_needed || (x.y ^ 0x80000000u) == thr_pos);
    };
    auto drops = [&](const uint2 &x) { return below(x) || (from_recent && !recent(x)); };
    // every warp takes a contiguous range of slots, 32 at a time: count, scan over the warps, list
    const int per = ((n + kSelWarps - 1) / kSelWarps + 31) / 32 * 32;
    const int w0 = min(n, warp * per), w1 = min(n, w0 + per);
    int eq_cnt = 0, total;
    for (int j0 = w0; j0 < w1; j0 += 32) {
        const int j = j0 + lane;
        eq_cnt += __popc(__ballot_sync(0xffffffffu, j < w1 && equal(item(j))));
    }
    const int eq0 = warps_excl_scan(sh, 0, eq_cnt, total);
    int eq = eq0, stay_lo = 0, stay_hi = 0;              // survivors below / from slot M on
    const unsigned lt = (1u << lane) - 1u;
    auto stays = [&](int j, int &eq_run) {
        bool in = j < w1, is_eq = false, s = false;
        if (in) {
            const uint2 x = item(j);
            is_eq = equal(x);
            s = !drops(x);
        }
        const unsigned eqs = __ballot_sync(0xffffffffu, is_eq);
        if (is_eq) s = eq_run + __popc(eqs & lt) >= rank;
        eq_run += __popc(eqs);
        return __ballot_sync(0xffffffffu, s);
    };
    for (int j0 = w0; j0 < w1; j0 += 32) {
        const unsigned s = stays(j0 + lane, eq);
        const unsigned lo = j0 + 32 <= M ? 0xffffffffu : j0 >= M ? 0u : (1u << (M - j0)) - 1u;
        stay_lo += __popc(s & lo);
        stay_hi += __popc(s & ~lo);
    }
    int total_hi;
    const int lo0 = warps_excl_scan(sh, 1, stay_lo, total);
    const int hi0 = warps_excl_scan(sh, 2, stay_hi, total_hi);
    eq = eq0;
    if (fresh) {
        int at = lo0 + hi0;
        for (int j0 = w0; j0 < w1; j0 += 32) {
            const unsigned s = stays(j0 + lane, eq);
            const int k = at + __popc(s & lt);
            if ((s >> lane & 1) && k < M) from[k] = j0 + lane;
            at += __popc(s);
        }
        if (tid == 0) a.moves[u] = M;
    } else {
        int hole = min(w0, M) - lo0, src = hi0;          // holes and survivors before this warp's range
        for (int j0 = w0; j0 < w1; j0 += 32) {
            const unsigned s = stays(j0 + lane, eq);
            const unsigned in = j0 + 32 <= w1 ? 0xffffffffu : (1u << (w1 - j0)) - 1u;
            const unsigned lo = j0 + 32 <= M ? 0xffffffffu : j0 >= M ? 0u : (1u << (M - j0)) - 1u;
            const unsigned holes = in & lo & ~s, ups = s & ~lo;
            const int kh = hole + __popc(holes & lt), ks = src + __popc(ups & lt);
            if ((holes >> lane & 1) && kh < M) to[kh] = j0 + lane;
            if ((ups >> lane & 1) && ks < M) from[ks] = j0 + lane;
            hole += __popc(holes);
            src += __popc(ups);
        }
        if (tid == 0) a.moves[u] = total_hi;
    }
}

constexpr int kMoveThreads = 256;
constexpr int kRows = 4;             // rows of a lane group in flight

// A group of ROW_BYTES / 16 lanes copies one row of K and of V.
template <int ROW_BYTES>
__global__ void __launch_bounds__(kMoveThreads)
paged_move_kernel(const __grid_constant__ EvictArgs a)
{
    constexpr int LPR = ROW_BYTES / 16, RPB = kMoveThreads / LPR;
    const int u = blockIdx.x / a.blocks, by = blockIdx.x - u * a.blocks, b = u / a.pv.H, h = u - b * a.pv.H;
    dependency_wait();
    if (h == 0 && by == 0 && threadIdx.x == 0) {
        a.past_out[b] = a.ends[2 * b];
        a.start_out[b] = a.ends[2 * b + 1];
    }
    const int moves = a.moves[u], part = threadIdx.x % LPR;
    const bool fresh = a.dst_table != nullptr;
    const int32_t *from_row = a.pv.table + (size_t)b * a.pv.max_pages;
    const int32_t *to_row = fresh ? a.dst_table + (size_t)b * a.dst_max_pages : from_row;
    // kRows rows of a lane group in flight: a move is a chain of three loads (list, page, row)
    for (int k0 = by * RPB * kRows + threadIdx.x / LPR; k0 < moves; k0 += a.blocks * RPB * kRows) {
        int64_t s[kRows], t[kRows];
        uint4 kv[kRows], vv[kRows];
        float sc[kRows];
        int32_t ps[kRows];
#pragma unroll
        for (int x = 0; x < kRows; ++x) {
            const int k = k0 + x * RPB;
            t[x] = -1;
            if (k >= moves) continue;
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
            *reinterpret_cast<uint4 *>(a.pv.k + t[x] * ROW_BYTES + part * 16) = kv[x];
            *reinterpret_cast<uint4 *>(a.pv.v + t[x] * ROW_BYTES + part * 16) = vv[x];
            if (part == 0) { a.pv.scores[t[x]] = sc[x]; a.pv.positions[t[x]] = ps[x]; }
        }
    }
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
    a.blocks = 1;
    char *w = static_cast<char *>(ws);
    a.from = reinterpret_cast<int32_t *>(w); w += pad(units * (size_t)budget * 4);
    a.to = reinterpret_cast<int32_t *>(w); w += pad(units * (size_t)budget * 4);
    a.moves = reinterpret_cast<int32_t *>(w); w += pad(units * 8);
    a.ends = reinterpret_cast<int32_t *>(w);
    const int cap = pv.max_pages << pv.ps_shift;
    const int cached = cap < kCached ? cap : kCached;
    cudaError_t e = allow_dynamic_smem<paged_select_kernel>((size_t)cached * 8);
    if (e != cudaSuccess) return e;
    paged_select_kernel<<<(unsigned)units, kSelThreads, (size_t)cached * 8, s>>>(a, cached);
    count_launch();
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    const int row_bytes = pv.d * elem_bytes, rpb = kMoveThreads / (row_bytes / 16);
    const int most = budget < cap ? budget : cap;
    long long blocks = (most + rpb * kRows - 1) / (rpb * kRows);
    const long long want = (16ll * device_sm_count() + (long long)units - 1) / (long long)units;
    if (blocks > want) blocks = want;
    a.blocks = (int)blocks;
    const unsigned grid = (unsigned)(units * blocks);
    switch (row_bytes) {
    case 128: e = launch_follower(paged_move_kernel<128>, grid, kMoveThreads, 0, s, a); break;
    case 256: e = launch_follower(paged_move_kernel<256>, grid, kMoveThreads, 0, s, a); break;
    default: e = launch_follower(paged_move_kernel<512>, grid, kMoveThreads, 0, s, a); break;
    }
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace a2sf
