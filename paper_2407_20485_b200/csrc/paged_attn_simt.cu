// Attention of a chunk over a paged cache in 32-bit storage, on the CUDA cores: the tensor cores' input types
// cannot give fp32 logits and probabilities.
//
// The G query heads of a K/V head and the tokens of the chunk are folded into rows r = i*G + g of
// one matrix per (sequence, K/V head), so K and V are read once for the whole group.
//   attn   flash attention: 16 x 16 threads own 16*RT rows and walk over 64-slot tiles; a thread holds
//          RT x 4 logits and RT x d/16 outputs in registers, running maximum and sum per row.
//   score  S_j <- alpha^len S_j + sum_r alpha^age(r) exp(s_rj - lse_r): 16 x 16 threads own 16*KT slots and
//          walk over the rows that see them, so a slot's sum is made in one place, in a fixed order.
// The next tile is on its way (16-byte asynchronous copies into a second buffer) while one is worked on.
// Bound by fp32 multiply-adds where there is work for all SMs: 8 shared-memory loads of 16 bytes feed 64 of
// them at RT = KT = 4.  A small call is bound by the latency of its few tiles instead: it takes RT = 1 and
// KT = 1, four times as many CTAs with a quarter of the work each (2 prompts of 129 tokens, 4 heads, d = 64:
// 39 us at 4, 20.5 us at 1).
#include "paged.cuh"

namespace a2sf {

A2SF_DEBUG_TRANSLATION_UNIT(paged_attn_simt)

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;        // slots (attn) or rows (score) of a walked tile

template <int D> struct Lay {
    static constexpr int LD = D + 4;                 // 16 lanes reading 16 rows meet 32 different banks
    static constexpr int LP = kTile + 4;
    static constexpr int kTileFloats = kTile * LD;
    static constexpr size_t attn(int rows) { return (size_t)(rows * LD + 4 * kTileFloats + rows * LP) * sizeof(float); }
    static constexpr size_t score(int slots) { return (size_t)(slots * LD + 2 * kTileFloats + 16 * slots + 2 * kTile) * sizeof(float); }
};

struct Unit {
    int b, h, past, len, rows;   // rows = len * G
    const int32_t *table;
};

__device__ __forceinline__ Unit make_unit(const PagedView &pv, int u)
{
    Unit x;
    x.b = u / pv.H;
    x.h = u - x.b * pv.H;
    const SeqState st = seq_state(pv, x.b);
    x.past = st.past; x.len = st.len; x.rows = st.len * pv.G;
    x.table = pv.table + (size_t)x.b * pv.max_pages;
    return x;
}

// 16 bytes global -> shared, asynchronously; zeros where `live` is false (nothing is read then)
__device__ __forceinline__ void copy16(float *dst, const float *src, bool live)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src),
                 "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// rows r0 .. r0+n-1 of the unit's folded query matrix; rows past the end become zero
template <int D>
__device__ __forceinline__ void copy_queries(float *dst, const AttendArgs &a, const Unit &u, int r0, int n)
{
    constexpr int CH = D / 4;
    for (int x = threadIdx.x; x < n * CH; x += kThreads) {
        const int row = x / CH, ch = x % CH, r = r0 + row;
        const bool live = r < u.rows && A2SF_IN_RANGE(r, a.pv.c * a.pv.G, kDbgPagedSimt);
        const int i = live ? r / a.pv.G : 0, g = live ? r - i * a.pv.G : 0;
        const float *p = static_cast<const float *>(a.q) + u.b * a.sq.b + (int64_t)(u.h * a.pv.G + g) * a.sq.h + (int64_t)i * a.sq.t;
        copy16(dst + row * Lay<D>::LD + ch * 4, p + ch * 4, live);
    }
}

// slots j0 .. j0+n-1 of the unit's keys or values; slots from `limit` on become zero and are not read
template <int D>
__device__ __forceinline__ void copy_slots(float *dst, const PagedView &pv, const Unit &u, const char *pool, int j0, int limit, int n)
{
    constexpr int CH = D / 4;
    for (int x = threadIdx.x; x < n * CH; x += kThreads) {
        const int row = x / CH, ch = x % CH, j = j0 + row;
        const bool live = j < limit;
        const int64_t at = live ? pool_row(pv, page_for_read(pv, u.table, j), u.h, j) * D : 0;
        copy16(dst + row * Lay<D>::LD + ch * 4, reinterpret_cast<const float *>(pool) + at + ch * 4, live);
    }
}

// s[i][j] = a_row(ty*R+i) . b_row(tx+16j)
template <int D, int R, int C>
__device__ __forceinline__ void products(float (&s)[R][C], const float *A, const float *B, int ty, int tx)
{
    constexpr int LD = Lay<D>::LD;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < C; ++j) s[i][j] = 0.f;
#pragma unroll 4
    for (int k = 0; k < D; k += 4) {
        float4 x[R], y[C];
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = *reinterpret_cast<const float4 *>(A + (ty * R + i) * LD + k);
#pragma unroll
        for (int j = 0; j < C; ++j) y[j] = *reinterpret_cast<const float4 *>(B + (tx + 16 * j) * LD + k);
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < C; ++j) {
                s[i][j] = fmaf(x[i].x, y[j].x, s[i][j]);
                s[i][j] = fmaf(x[i].y, y[j].y, s[i][j]);
                s[i][j] = fmaf(x[i].z, y[j].z, s[i][j]);
                s[i][j] = fmaf(x[i].w, y[j].w, s[i][j]);
            }
    }
}

template <int D, int RT>
__global__ void __launch_bounds__(kThreads)
paged_attn_simt_kernel(const __grid_constant__ AttendArgs a, int row_tiles)
{
    constexpr int LD = Lay<D>::LD, LP = Lay<D>::LP, NO = D / 64, kR = 16 * RT;
    extern __shared__ __align__(16) float sm[];
    float *Q = sm, *K = Q + kR * LD, *V = K + 2 * Lay<D>::kTileFloats, *P = V + 2 * Lay<D>::kTileFloats;
    const int G = a.pv.G;
    dependency_wait();
    dependents_may_start();
    const Unit u = make_unit(a.pv, blockIdx.x / row_tiles);
    // the tiles that see most slots first
    const int r0 = (row_tiles - 1 - blockIdx.x % row_tiles) * kR;
    if (r0 >= u.rows) return;
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    const int last_row = min(r0 + kR, u.rows) - 1;
    const int limit = u.past + last_row / G + 1;         // slots that the last row sees
    copy_queries<D>(Q, a, u, r0, kR);
    copy_slots<D>(K, a.pv, u, a.pv.k, 0, limit, kTile);
    copies_commit();
    copy_slots<D>(V, a.pv, u, a.pv.v, 0, limit, kTile);
    copies_commit();

    int vis[RT];                                          // slots that each of this thread's rows sees
    float m[RT], l[RT], o[RT][NO][4];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        vis[i] = u.past + min(r0 + ty * RT + i, last_row) / G + 1;
        m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
        for (int j = 0; j < NO; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][j][e] = 0.f;
    }
    int buf = 0;
    for (int j0 = 0; j0 < limit; j0 += kTile, buf ^= 1) {
        copies_wait<1>();                                 // keys (and queries) are here; values may be on their way
        __syncthreads();                                  // ... everybody's, and the tile before has been read
        float *next_k = K + (buf ^ 1) * Lay<D>::kTileFloats, *next_v = V + (buf ^ 1) * Lay<D>::kTileFloats;
        if (j0 + kTile < limit) copy_slots<D>(next_k, a.pv, u, a.pv.k, j0 + kTile, limit, kTile);
        copies_commit();
        float s[RT][4];
        products<D, RT, 4>(s, Q, K + buf * Lay<D>::kTileFloats, ty, tx);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            float mx = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[i][j] = j0 + tx + 16 * j < vis[i] ? s[i][j] * a.pv.sl2 : -INFINITY;
                mx = fmaxf(mx, s[i][j]);
            }
#pragma unroll
            for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
            // a tile may hold nothing for this row (the first holds one slot at least, so m is finite from there on)
            const float mn = fmaxf(m[i], mx);
            const float factor = exp2f(m[i] - mn);
            m[i] = mn;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = exp2f(s[i][j] - mn);
                sum += p;
                P[(ty * RT + i) * LP + tx + 16 * j] = p;
            }
#pragma unroll
            for (int w = 8; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
            l[i] = fmaf(l[i], factor, sum);
#pragma unroll
            for (int j = 0; j < NO; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][j][e] *= factor;
        }
        copies_wait<1>();                                 // values are here; the next keys may be on their way
        __syncthreads();
        if (j0 + kTile < limit) copy_slots<D>(next_v, a.pv, u, a.pv.v, j0 + kTile, limit, kTile);
        copies_commit();
        const float *Vt = V + buf * Lay<D>::kTileFloats;
#pragma unroll 2
        for (int k = 0; k < kTile; k += 4) {
            float p4[RT][4];
#pragma unroll
            for (int i = 0; i < RT; ++i) *reinterpret_cast<float4 *>(p4[i]) = *reinterpret_cast<const float4 *>(P + (ty * RT + i) * LP + k);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                for (int j = 0; j < NO; ++j) {
                    const float4 v = *reinterpret_cast<const float4 *>(Vt + (k + kk) * LD + j * 64 + tx * 4);
#pragma unroll
                    for (int i = 0; i < RT; ++i) {
                        o[i][j][0] = fmaf(p4[i][kk], v.x, o[i][j][0]);
                        o[i][j][1] = fmaf(p4[i][kk], v.y, o[i][j][1]);
                        o[i][j][2] = fmaf(p4[i][kk], v.z, o[i][j][2]);
                        o[i][j][3] = fmaf(p4[i][kk], v.w, o[i][j][3]);
                    }
                }
        }
    }
    float *lse2 = static_cast<float *>(a.ws);
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int r = r0 + ty * RT + i;
        if (r > last_row || !A2SF_IN_RANGE(r, a.pv.c * G, kDbgPagedSimt)) continue;
        const int tok = r / G, g = r - tok * G;
        const float inv = 1.f / l[i];
        float *dst = static_cast<float *>(a.out) + u.b * a.so.b + (int64_t)(u.h * G + g) * a.so.h + (int64_t)tok * a.so.t;
#pragma unroll
        for (int j = 0; j < NO; ++j)
            *reinterpret_cast<float4 *>(dst + j * 64 + tx * 4) = make_float4(o[i][j][0] * inv, o[i][j][1] * inv, o[i][j][2] * inv, o[i][j][3] * inv);
        if (tx == 0) {
            const float z = m[i] + log2f(l[i]);
            lse2[(size_t)(u.b * a.pv.H + u.h) * a.pv.c * G + r] = z;
            if (a.lse) a.lse[((size_t)u.b * a.pv.H * G + u.h * G + g) * a.pv.c + tok] = z * 0.6931471805599453f;
        }
    }
}

template <int D, int KT>
__global__ void __launch_bounds__(kThreads)
paged_score_simt_kernel(const __grid_constant__ AttendArgs a, int slot_tiles)
{
    constexpr int LD = Lay<D>::LD, kS = 16 * KT;
    extern __shared__ __align__(16) float sm[];
    float *K = sm, *Q = K + kS * LD, *part = Q + 2 * Lay<D>::kTileFloats, *cr = part + 16 * kS;
    const int G = a.pv.G;
    const Unit u = make_unit(a.pv, blockIdx.x / slot_tiles);
    const int j0 = (blockIdx.x % slot_tiles) * kS, used = u.past + u.len;
    const bool idle = u.len == 0 || j0 >= used;
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    // rows before the first weighted token, or before the token that first sees the tile, add nothing
    const int first = max(max(first_weighted_token(u.len, a.nl2a), j0 - u.past), 0) * G / kTile * kTile;
    float old = 0.f, *dst = nullptr;
    if (!idle) {
        copy_slots<D>(K, a.pv, u, a.pv.k, j0, used, kS);
        copy_queries<D>(Q, a, u, first, kTile);
        if (tid < kS && j0 + tid < used) {
            const int page = page_for_write(a.pv, u.table, j0 + tid);
            if (page >= 0) {
                dst = a.pv.scores + pool_row(a.pv, page, u.h, j0 + tid);
                old = *dst;
            }
        }
    }
    copies_commit();
    dependency_wait();                                    // everything before does not depend on the attention
    if (idle) { copies_wait<0>(); return; }
    const float *lse2 = static_cast<const float *>(a.ws) + (size_t)(u.b * a.pv.H + u.h) * a.pv.c * G;
    auto constant = [&](int r) { return r < u.rows ? lse2[r] + age_exponent(u.len - 1 - r / G, a.nl2a) : INFINITY; };
    if (tid < kTile) cr[tid] = constant(first + tid);
    float sum[KT];
#pragma unroll
    for (int j = 0; j < KT; ++j) sum[j] = 0.f;
    int buf = 0;
    for (int r0 = first; r0 < u.rows; r0 += kTile, buf ^= 1) {
        copies_wait<0>();
        __syncthreads();                                  // this tile is here, the one before has been read
        const bool more = r0 + kTile < u.rows;
        if (more) copy_queries<D>(Q + (buf ^ 1) * Lay<D>::kTileFloats, a, u, r0 + kTile, kTile);
        copies_commit();
        const float next_c = more && tid < kTile ? constant(r0 + kTile + tid) : 0.f;
        float s[4][KT];
        products<D, 4, KT>(s, Q + buf * Lay<D>::kTileFloats, K, ty, tx);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int vis = u.past + (r0 + ty * 4 + i) / G + 1;
            const float c = cr[buf * kTile + ty * 4 + i];
#pragma unroll
            for (int j = 0; j < KT; ++j)
                sum[j] += j0 + tx + 16 * j < vis ? exp2f(fmaf(s[i][j], a.pv.sl2, -c)) : 0.f;
        }
        if (more && tid < kTile) cr[(buf ^ 1) * kTile + tid] = next_c;
    }
#pragma unroll
    for (int j = 0; j < KT; ++j) part[ty * kS + tx + 16 * j] = sum[j];
    __syncthreads();
    if (dst) {
        float total = 0.f;
#pragma unroll
        for (int y = 0; y < 16; ++y) total += part[y * kS + tid];        // fixed order
        *dst = fmaf(old, exp2f(-age_exponent(u.len, a.nl2a)), total);
    }
}

template <int D, int T>
cudaError_t launch(const AttendArgs &a, cudaStream_t s)
{
    constexpr size_t attn = Lay<D>::attn(16 * T), score = Lay<D>::score(16 * T);
    cudaError_t e = allow_dynamic_smem<paged_attn_simt_kernel<D, T>>(attn);
    if (e == cudaSuccess) e = allow_dynamic_smem<paged_score_simt_kernel<D, T>>(score);
    if (e != cudaSuccess) return e;
    const long long units = (long long)a.pv.B * a.pv.H;
    const long long row_tiles = ((long long)a.pv.c * a.pv.G + 16 * T - 1) / (16 * T);
    const long long slot_tiles = (((long long)a.pv.max_pages << a.pv.ps_shift) + 16 * T - 1) / (16 * T);
    if (units * row_tiles > 0x7fffffffll || units * slot_tiles > 0x7fffffffll) return cudaErrorInvalidValue;
    if ((e = launch_chained(paged_attn_simt_kernel<D, T>, (unsigned)(units * row_tiles), kThreads, attn, s, a, (int)row_tiles)) != cudaSuccess) return e;
    count_launch();
    if (!a.scores) return cudaSuccess;
    e = launch_chained(paged_score_simt_kernel<D, T>, (unsigned)(units * slot_tiles), kThreads, score, s, a, (int)slot_tiles);
    if (e == cudaSuccess) count_launch();
    return e;
}

}  // namespace

size_t attend_simt_ws_bytes(const PagedView &pv)
{
    return (size_t)pv.B * pv.H * pv.G * pv.c * sizeof(float);          // log-sum-exp of every row
}

cudaError_t launch_attend_simt(const AttendArgs &a, cudaStream_t s)
{
    // tiles of 64 rows as soon as there is one for every second SM
    const long long tiles = (long long)a.pv.B * a.pv.H * (((long long)a.pv.c * a.pv.G + 63) / 64);
    const bool large = 2 * tiles >= device_sm_count();
    if (a.pv.d == 128) return large ? launch<128, 4>(a, s) : launch<128, 1>(a, s);
    return large ? launch<64, 4>(a, s) : launch<64, 1>(a, s);
}

}  // namespace a2sf
