// Attention of a chunk over a paged cache on the CUDA cores: 32-bit storage, where the logits and
// probabilities have to keep fp32 accuracy that the tensor cores' input types cannot give.
//
// The G query heads of a K/V head and the tokens of the chunk are folded into rows r = i*G + g of
// one matrix per (sequence, K/V head), so K and V are read once for the whole group.
//   pass 1  flash attention: a CTA owns 64 rows and walks over the key tiles that they see; a thread
//           holds 4 x 4 logits and 4 x d/16 outputs in registers, running maximum and sum per row.
//   pass 2  S_j <- alpha^len S_j + sum_r alpha^age(r) exp(s_rj - lse_r): a CTA owns 64 slots and walks
//           over the rows that see them, so a slot's sum is made in one place, in a fixed order.
// Bound by fp32 multiply-adds: 8 shared-memory loads of 16 bytes feed 64 of them in pass 1's QK^T.
#include "paged.cuh"

namespace a2sf {

A2SF_DEBUG_TRANSLATION_UNIT(paged_attn_simt)

namespace {

constexpr int kThreads = 256;
constexpr int kR = 64;           // rows per tile
constexpr int kK = 64;           // key slots per tile

template <int D> struct Smem {
    static constexpr int LD = D + 4;                 // 16 lanes reading 16 rows meet 32 different banks
    static constexpr int LP = kK + 4;
    static constexpr size_t kAttn = (size_t)(kR * LD + kK * LD + kR * LP) * sizeof(float);
    static constexpr size_t kScore = (size_t)(kR * LD + kK * LD + 16 * kK + kR) * sizeof(float);
};

struct Unit {
    int b, h, past, len, rows;   // rows = len * G
    const int32_t *table;
};

// rows r0 .. r0+63 of the unit's folded query matrix, as fp32; rows past the end are zero
template <typename T, int D>
__device__ __forceinline__ void load_queries(float *dst, const AttendArgs &a, const Unit &u, int r0)
{
    constexpr int VEC = Elem<T>::kVec, CH = D / VEC;
    for (int x = threadIdx.x; x < kR * CH; x += kThreads) {
        const int row = x / CH, ch = x % CH, r = r0 + row;
        float f[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = 0.f;
        if (r < u.rows) {
            const int i = r / a.pv.G, g = r - i * a.pv.G;
            const T *p = static_cast<const T *>(a.q) + u.b * a.sq.b + (int64_t)(u.h * a.pv.G + g) * a.sq.h + (int64_t)i * a.sq.t;
            Elem<T>::unpack(*reinterpret_cast<const uint4 *>(p + ch * VEC), f);
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) dst[row * Smem<D>::LD + ch * VEC + e] = f[e];
    }
}

// slots j0 .. j0+63 of the unit's keys or values, as fp32; slots from `limit` on are zero and not read
template <typename T, int D>
__device__ __forceinline__ void load_slots(float *dst, const PagedView &pv, const Unit &u, const char *pool, int j0, int limit)
{
    constexpr int VEC = Elem<T>::kVec, CH = D / VEC;
    for (int x = threadIdx.x; x < kK * CH; x += kThreads) {
        const int row = x / CH, ch = x % CH, j = j0 + row;
        float f[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = 0.f;
        if (j < limit) {
            const int64_t at = pool_row(pv, page_for_read(pv, u.table, j), u.h, j) * D;
            Elem<T>::unpack(*reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(pool) + at + ch * VEC), f);
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) dst[row * Smem<D>::LD + ch * VEC + e] = f[e];
    }
}

// s[i][j] = q_row(ty*4+i) . k_row(tx+16j)
template <int D>
__device__ __forceinline__ void logits(float (&s)[4][4], const float *Q, const float *K, int ty, int tx)
{
    constexpr int LD = Smem<D>::LD;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
    for (int k = 0; k < D; k += 4) {
        float4 q4[4], k4[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q4[i] = *reinterpret_cast<const float4 *>(Q + (ty * 4 + i) * LD + k);
#pragma unroll
        for (int j = 0; j < 4; ++j) k4[j] = *reinterpret_cast<const float4 *>(K + (tx + 16 * j) * LD + k);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[i][j] = fmaf(q4[i].x, k4[j].x, s[i][j]);
                s[i][j] = fmaf(q4[i].y, k4[j].y, s[i][j]);
                s[i][j] = fmaf(q4[i].z, k4[j].z, s[i][j]);
                s[i][j] = fmaf(q4[i].w, k4[j].w, s[i][j]);
            }
    }
}

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

template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
paged_attn_simt_kernel(const __grid_constant__ AttendArgs a, int row_tiles)
{
    constexpr int LD = Smem<D>::LD, LP = Smem<D>::LP, NO = D / 64;
    extern __shared__ __align__(16) float sm[];
    float *Q = sm, *KV = Q + kR * LD, *P = KV + kK * LD;
    const int G = a.pv.G;
    const Unit u = make_unit(a.pv, blockIdx.x / row_tiles);
    // the tiles that see most slots first
    const int r0 = (row_tiles - 1 - blockIdx.x % row_tiles) * kR;
    if (r0 >= u.rows) return;
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    const int last_row = min(r0 + kR, u.rows) - 1;
    const int limit = u.past + last_row / G + 1;         // slots that the last row sees
    load_queries<T, D>(Q, a, u, r0);

    int vis[4];                                           // slots that each of this thread's rows sees
    float m[4], l[4], o[4][NO][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        vis[i] = u.past + min(r0 + ty * 4 + i, last_row) / G + 1;
        m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
        for (int j = 0; j < NO; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][j][e] = 0.f;
    }
    for (int j0 = 0; j0 < limit; j0 += kK) {
        __syncthreads();
        load_slots<T, D>(KV, a.pv, u, a.pv.k, j0, limit);
        __syncthreads();
        float s[4][4];
        logits<D>(s, Q, KV, ty, tx);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float mx = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[i][j] = j0 + tx + 16 * j < vis[i] ? s[i][j] * a.pv.sl2 : -INFINITY;
                mx = fmaxf(mx, s[i][j]);
            }
#pragma unroll
            for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
            // a tile may hold nothing for this row (its mask leaves the first slot at least, so m is
            // finite from the first tile on)
            const float mn = fmaxf(m[i], mx);
            const float factor = exp2f(m[i] - mn);
            m[i] = mn;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = exp2f(s[i][j] - mn);
                sum += p;
                P[(ty * 4 + i) * LP + tx + 16 * j] = p;
            }
#pragma unroll
            for (int w = 8; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
            l[i] = fmaf(l[i], factor, sum);
#pragma unroll
            for (int j = 0; j < NO; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][j][e] *= factor;
        }
        __syncthreads();
        load_slots<T, D>(KV, a.pv, u, a.pv.v, j0, limit);
        __syncthreads();
#pragma unroll 2
        for (int k = 0; k < kK; k += 4) {
            float p4[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<float4 *>(p4[i]) = *reinterpret_cast<const float4 *>(P + (ty * 4 + i) * LP + k);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                for (int j = 0; j < NO; ++j) {
                    const float4 v = *reinterpret_cast<const float4 *>(KV + (k + kk) * LD + j * 64 + tx * 4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
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
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + ty * 4 + i;
        if (r > last_row) continue;
        const int tok = r / G, g = r - tok * G;
        const float inv = 1.f / l[i];
        T *dst = static_cast<T *>(a.out) + u.b * a.so.b + (int64_t)(u.h * G + g) * a.so.h + (int64_t)tok * a.so.t;
#pragma unroll
        for (int j = 0; j < NO; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) dst[j * 64 + tx * 4 + e] = Elem<T>::from_float(o[i][j][e] * inv);
        if (tx == 0) {
            const float z = m[i] + log2f(l[i]);
            lse2[(size_t)(u.b * a.pv.H + u.h) * a.pv.c * G + r] = z;
            if (a.lse) a.lse[((size_t)u.b * a.pv.H * G + u.h * G + g) * a.pv.c + tok] = z * 0.6931471805599453f;
        }
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
paged_score_simt_kernel(const __grid_constant__ AttendArgs a, int slot_tiles)
{
    constexpr int LD = Smem<D>::LD;
    extern __shared__ __align__(16) float sm[];
    float *Q = sm, *K = Q + kR * LD, *part = K + kK * LD, *cr = part + 16 * kK;
    const int G = a.pv.G;
    const Unit u = make_unit(a.pv, blockIdx.x / slot_tiles);
    const int j0 = (blockIdx.x % slot_tiles) * kK, used = u.past + u.len;
    if (u.len == 0 || j0 >= used) return;
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    const float *lse2 = static_cast<const float *>(a.ws) + (size_t)(u.b * a.pv.H + u.h) * a.pv.c * G;
    load_slots<T, D>(K, a.pv, u, a.pv.k, j0, used);
    // rows before the first weighted token, or before the token that first sees the tile, add nothing
    const int first = max(first_weighted_token(u.len, a.nl2a), j0 - u.past);
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (int r0 = max(0, first) * G / kR * kR; r0 < u.rows; r0 += kR) {
        __syncthreads();
        load_queries<T, D>(Q, a, u, r0);
        if (tid < kR) {
            const int r = r0 + tid;
            cr[tid] = r < u.rows ? lse2[r] + age_exponent(u.len - 1 - r / G, a.nl2a) : INFINITY;
        }
        __syncthreads();
        float s[4][4];
        logits<D>(s, Q, K, ty, tx);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int vis = u.past + (r0 + ty * 4 + i) / G + 1;
            const float c = cr[ty * 4 + i];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                sum[j] += j0 + tx + 16 * j < vis ? exp2f(fmaf(s[i][j], a.pv.sl2, -c)) : 0.f;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) part[ty * kK + tx + 16 * j] = sum[j];
    __syncthreads();
    const int j = j0 + tid;
    if (tid < kK && j < used) {
        float total = 0.f;
#pragma unroll
        for (int y = 0; y < 16; ++y) total += part[y * kK + tid];        // fixed order
        const int page = page_for_write(a.pv, u.table, j);
        if (page >= 0) {
            float *dst = a.pv.scores + pool_row(a.pv, page, u.h, j);
            *dst = fmaf(*dst, exp2f(-age_exponent(u.len, a.nl2a)), total);
        }
    }
}

template <typename T, int D>
cudaError_t launch(const AttendArgs &a, cudaStream_t s)
{
    cudaError_t e = allow_dynamic_smem<paged_attn_simt_kernel<T, D>>(Smem<D>::kAttn);
    if (e == cudaSuccess) e = allow_dynamic_smem<paged_score_simt_kernel<T, D>>(Smem<D>::kScore);
    if (e != cudaSuccess) return e;
    const long long units = (long long)a.pv.B * a.pv.H;
    const long long row_tiles = ((long long)a.pv.c * a.pv.G + kR - 1) / kR;
    const long long slot_tiles = (((long long)a.pv.max_pages << a.pv.ps_shift) + kK - 1) / kK;
    if (units * row_tiles > 0x7fffffffll || units * slot_tiles > 0x7fffffffll) return cudaErrorInvalidValue;
    paged_attn_simt_kernel<T, D><<<(unsigned)(units * row_tiles), kThreads, Smem<D>::kAttn, s>>>(a, (int)row_tiles);
    count_launch();
    if ((e = cudaGetLastError()) != cudaSuccess || !a.scores) return e;
    paged_score_simt_kernel<T, D><<<(unsigned)(units * slot_tiles), kThreads, Smem<D>::kScore, s>>>(a, (int)slot_tiles);
    count_launch();
    return cudaGetLastError();
}

}  // namespace

size_t attend_simt_ws_bytes(const PagedView &pv)
{
    return (size_t)pv.B * pv.H * pv.G * pv.c * sizeof(float);          // log-sum-exp of every row
}

cudaError_t launch_attend_simt(int dtype, const AttendArgs &a, cudaStream_t s)
{
    const bool wide = a.pv.d == 128;
    switch (dtype) {
    case A2SF_F32: return wide ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
    case A2SF_BF16: return wide ? launch<__nv_bfloat16, 128>(a, s) : launch<__nv_bfloat16, 64>(a, s);
    default: return wide ? launch<__half, 128>(a, s) : launch<__half, 64>(a, s);
    }
}

}  // namespace a2sf
