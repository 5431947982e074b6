// Attention of a chunk over a paged cache: 32-bit storage, and calls of 16-bit storage that are too small for the tiles of
// tcgen05 (128 rows, a CTA per SM, a plan).
//
// The G query heads of a K/V head and the tokens of the chunk are folded into rows r = i*G + g of
// one matrix per (sequence, K/V head), so K and V are read once for the whole group.
//   attn   rows in tiles of 16 x R warps, keys in tiles of 64; running maximum and sum per row.  R = 4: a warp has
//          16 rows and all keys of a tile.  R = 1: the four warps share 16 rows and take 16 keys of a tile each.
//          Where that makes too few CTAs the keys are cut into pieces as well.
//   merge  joins the pieces.
//   score  S_j <- alpha^len S_j + sum_r alpha^age(r) exp(s_rj - lse_r): the same with slots as rows and queries
//          as keys, so a slot's sum is made in one place, in a fixed order.
//
// 32 bits: products on mma.sync m16n8k8 with operands of 11 bits: x = hi + lo, hi rounded and lo cut to 11 bits, and
// a b = hi hi + hi lo + lo hi.  What is left out is below 2^-21 |a b|, less than the fp32 sum of 64 products
// may be off; sums are fp32.  That is 171 multiply-adds a clock and SM against 128 on the CUDA cores, of which
// shared-memory loads left 39 % (64 heads, 2048 tokens, d = 128: 3609 us on CUDA cores, 1813 so, 58 % of the 171).  An instruction's
// k index means what both operands agree on, so a lane reads four neighbouring elements of a row at once and uses them in
// two steps; the accumulators of Q K^T are the operand of P V as they are.
// 16 bits: products on mma.sync m16n8k16, operands by ldmatrix; P is the sum of two terms of the storage type, off by the square
// of half a step (36 heads, 302 tokens, d = 64: 18.0 us with one term, 18.6 with two).
//
// Windowed (Win): a row tile walks over the near slots of its rows (see Near); attn and merge alone.
//
// The next tile's keys are on their way (16-byte asynchronous copies) while the tile before is finished, values while
// logits are made (16 bits: a whole tile ahead, with two buffers); a warp looks up the pages of its rows all at once (one after the other: 262 us where it takes 164).
// Bound by the instructions around the products -- four to split an operand -- and, in small calls, by the latency of a
// few tiles twice over (2 x 4 heads, 129 tokens, d = 64: 11.2 us in 32 bits; 12 heads, 64 tokens: 5.7 in 16, two kernels).
#include <algorithm>

#include "paged.cuh"

namespace a2sf {

A2SF_DEBUG_TRANSLATION_UNIT(paged_attn_mma)

namespace {

constexpr int kThreads = 128;
constexpr int kTile = 64;        // keys (attn) or rows (score) of a walked tile
constexpr int kSms = 148;
// The reference (what is subtracted before the exponential, log2 units) lies so far below the maximum: fp16 then holds all bits of a
// probability down to 2^-29 of the largest, and some down to 2^-39; what is below packs to 0 while the row sum counts it.
template <typename T> constexpr int kBelow = std::is_same<T, __half>::value ? 15 : 0;

// Row distances in shared memory, in elements.  32 bits: 8 lanes reading 64 bytes of 2 rows (Q, K), or 16 bytes of every second
// of 8 rows (V), meet 32 different banks; 16 bits: 8 rows of an 8 x 8 matrix do.
template <typename T, int D> struct Lay {
    static constexpr int LD = sizeof(T) == 4 ? D + 16 : D + 8;               // Q, K
    static constexpr int LV = sizeof(T) == 4 ? D + 4 : D + 8;
    static constexpr int kBufs = sizeof(T) == 4 ? 1 : 2;                     // of K and of V: two where a CTA then still takes a third of an SM
    static constexpr size_t attn(int rows) { return (size_t)(rows * LD + kBufs * kTile * (LD + LV)) * sizeof(T); }
    static constexpr size_t score(int slots) { return (size_t)(slots * LD + 2 * kTile * LD) * sizeof(T) + (4 * kTile + 4 * 16) * sizeof(float); }
    static_assert((size_t)kTile * (LD + LV) * sizeof(T) >= (size_t)(128 + 64 * D) * sizeof(float), "the joined results take the place of K and V");
};

struct MmaWs {
    float *lse2;                 // [B*H][c*G] log-sum-exp, log2 units
    float2 *ml;                  // [pieces][B*H][c*G] reference (log2 units), sum
    float *o;                    // [pieces][B*H][c*G][d]
    int pieces;
};

struct Unit {
    int b, h, past, len, rows;   // rows = len * G; past in near slots
    const int32_t *table;
    Near near;
};

__device__ __forceinline__ Unit make_unit(const PagedView &pv, int u)
{
    Unit x;
    x.b = u / pv.H;
    x.h = u - x.b * pv.H;
    const SeqState st = seq_state(pv, x.b);
    x.past = st.past; x.len = st.len; x.rows = st.len * pv.G;
    x.table = pv.table + (size_t)x.b * pv.max_pages;
    x.near = near_slots<false>(pv, st.past, 0);
    return x;
}

// 16 bytes global -> shared, asynchronously; zeros where `live` is false (nothing is read then)
__device__ __forceinline__ void copy16(void *dst, const void *src, bool live)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src),
                 "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Rows r0 .. r0+N-1 of the unit's folded query matrix; rows past the end become zero.  A warp's lanes work out the
// addresses of the rows that it copies, all at once.
template <typename T, int D, int N>
__device__ __forceinline__ void copy_queries(T *dst, const AttendArgs &a, const Unit &u, int r0)
{
    constexpr int VEC = 16 / sizeof(T), CH = D / VEC, kAt = 32 / CH, kPer = N / (kThreads / 32);      // rows of a warp's copy, rows of a warp
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, ch = lane % CH, sub = lane / CH;
    const int mine = r0 + warp * kPer + lane;
    const bool live = lane < kPer && mine < u.rows && A2SF_IN_RANGE(mine, a.pv.c * a.pv.G, kDbgPagedMma);
    const int i = live ? mine / a.pv.G : 0, g = live ? mine - i * a.pv.G : 0;
    const long long at = live ? u.b * a.sq.b + (int64_t)(u.h * a.pv.G + g) * a.sq.h + (int64_t)i * a.sq.t : -1;
#pragma unroll
    for (int x = 0; x < kPer; x += kAt) {
        const long long from = __shfl_sync(0xffffffffu, at, x + sub);
        copy16(dst + (warp * kPer + x + sub) * Lay<T, D>::LD + ch * VEC, static_cast<const T *>(a.q) + (from < 0 ? 0 : from) + ch * VEC, from >= 0);
    }
}

// slots j0 .. j0+N-1 of the unit's keys or values; slots from `limit` on, and those that no row sees, become zero and are not
// read.  A warp's lanes look up the rows that it copies, all at once.
template <typename T, int D, int N, bool Win = false>
__device__ __forceinline__ void copy_slots(T *dst, int ld, const PagedView &pv, const Unit &u, const char *pool, int j0, int limit)
{
    constexpr int VEC = 16 / sizeof(T), CH = D / VEC, kAt = 32 / CH, kPer = N / (kThreads / 32);      // rows of a warp's copy, rows of a warp
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, ch = lane % CH, sub = lane / CH;
    const int mine = j0 + warp * kPer + lane;
    const bool live = lane < kPer && mine < limit && !(Win && mine < u.near.dead && mine >= pv.sinks);
    const int real = real_slot<Win>(pv, u.near, mine), row = live ? (int)pool_row(pv, page_for_read(pv, u.table, real), u.h, real) : -1;
#pragma unroll
    for (int x = 0; x < kPer; x += kAt) {
        const int from = __shfl_sync(0xffffffffu, row, x + sub);
        copy16(dst + (warp * kPer + x + sub) * ld + ch * VEC, reinterpret_cast<const T *>(pool) + (int64_t)max(from, 0) * D + ch * VEC, from >= 0);
    }
}

// x = hi + lo up to 2^-23 |x|, both of 11 significant bits
__device__ __forceinline__ void split(float x, uint32_t &hi, uint32_t &lo)
{
    hi = (__float_as_uint(x) + 0x1000u) & 0xffffe000u;
    lo = __float_as_uint(x - __uint_as_float(hi)) & 0xffffe000u;
}
__device__ __forceinline__ void mma8(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The warp's part of the products.
//   products  s[n][e] = a_row . b_row for 16 rows of A and 8 N rows of B.  Lane (g, c) = (lane / 4, lane % 4) gets rows g (e < 2)
//             and g + 8 of A against rows 8n + 2c + e % 2 of B.
//   values    o += p V for 16 rows of p, laid out like s, and 8 N keys.
//   store     row x (0: g, 1: g + 8) of o, times f.
template <typename T, int D> struct Ops;

template <int D> struct Ops<float, D> {
    template <int N> static __device__ __forceinline__ void products(float (&s)[N][4], const float *A, const float *B)
    {
        constexpr int LD = Lay<float, D>::LD;
        const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
        // An instruction's result is there after about four others have been issued, so several accumulators are in turn: of four
        // n-tiles, or of two and the two small products apart (2^-11 of the first one).
        constexpr int GN = N < 4 ? N : 4, kSmall = N < 4 ? 2 : 1;
        float small[kSmall][N][4];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[n][e] = 0.f;
#pragma unroll
                for (int x = 0; x < kSmall; ++x) small[x][n][e] = 0.f;
            }
#pragma unroll 2
        for (int k = 0; k < D; k += 16) {
            const float4 x0 = *reinterpret_cast<const float4 *>(A + g * LD + k + 4 * c), x1 = *reinterpret_cast<const float4 *>(A + (g + 8) * LD + k + 4 * c);
            uint32_t hi[2][4], lo[2][4];
            split(x0.x, hi[0][0], lo[0][0]); split(x1.x, hi[0][1], lo[0][1]);
            split(x0.y, hi[0][2], lo[0][2]); split(x1.y, hi[0][3], lo[0][3]);
            split(x0.z, hi[1][0], lo[1][0]); split(x1.z, hi[1][1], lo[1][1]);
            split(x0.w, hi[1][2], lo[1][2]); split(x1.w, hi[1][3], lo[1][3]);
#pragma unroll
            for (int n0 = 0; n0 < N; n0 += GN) {
                uint32_t h[GN][4], l[GN][4];
#pragma unroll
                for (int n = 0; n < GN; ++n) {
                    const float4 y = *reinterpret_cast<const float4 *>(B + ((n0 + n) * 8 + g) * LD + k + 4 * c);
                    split(y.x, h[n][0], l[n][0]); split(y.y, h[n][1], l[n][1]); split(y.z, h[n][2], l[n][2]); split(y.w, h[n][3], l[n][3]);
                }
#pragma unroll
                for (int x = 0; x < 2; ++x) {
#pragma unroll
                    for (int n = 0; n < GN; ++n) mma8(small[0][n0 + n], hi[x], l[n][2 * x], l[n][2 * x + 1]);
#pragma unroll
                    for (int n = 0; n < GN; ++n) mma8(s[n0 + n], hi[x], h[n][2 * x], h[n][2 * x + 1]);
#pragma unroll
                    for (int n = 0; n < GN; ++n) mma8(small[kSmall - 1][n0 + n], lo[x], h[n][2 * x], h[n][2 * x + 1]);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] += kSmall == 2 ? small[0][n][e] + small[kSmall - 1][n][e] : small[0][n][e];
    }

    template <int N> static __device__ __forceinline__ void values(float (&o)[D / 8][4], const float (&s)[N][4], const float *V)
    {
        constexpr int LV = Lay<float, D>::LV;
        // output column 32q + 4g' + i is column g' of the instruction's n-tile 4q + i; k index c is key 2c, c + 4 key 2c + 1
        const int g = (threadIdx.x & 31) >> 2, c = threadIdx.x & 3;
        const float *v0 = V + 2 * c * LV + 4 * g;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            uint32_t hi[4], lo[4];
            split(s[n][0], hi[0], lo[0]); split(s[n][2], hi[1], lo[1]);
            split(s[n][1], hi[2], lo[2]); split(s[n][3], hi[3], lo[3]);
#pragma unroll
            for (int q = 0; q < D / 32; q += 2) {
                uint32_t h0[8], l0[8], h1[8], l1[8];
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const float4 y0 = *reinterpret_cast<const float4 *>(v0 + n * 8 * LV + 32 * (q + p)), y1 = *reinterpret_cast<const float4 *>(v0 + (n * 8 + 1) * LV + 32 * (q + p));
                    split(y0.x, h0[4 * p], l0[4 * p]); split(y0.y, h0[4 * p + 1], l0[4 * p + 1]); split(y0.z, h0[4 * p + 2], l0[4 * p + 2]); split(y0.w, h0[4 * p + 3], l0[4 * p + 3]);
                    split(y1.x, h1[4 * p], l1[4 * p]); split(y1.y, h1[4 * p + 1], l1[4 * p + 1]); split(y1.z, h1[4 * p + 2], l1[4 * p + 2]); split(y1.w, h1[4 * p + 3], l1[4 * p + 3]);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) mma8(o[4 * q + i], hi, l0[i], l1[i]);
#pragma unroll
                for (int i = 0; i < 8; ++i) mma8(o[4 * q + i], lo, h0[i], h1[i]);
#pragma unroll
                for (int i = 0; i < 8; ++i) mma8(o[4 * q + i], hi, h0[i], h1[i]);
            }
        }
    }

    template <typename U> static __device__ __forceinline__ void store(U *dst, const float (&o)[D / 8][4], int x, float f)
    {
        const int c = threadIdx.x & 3;
#pragma unroll
        for (int q = 0; q < D / 32; ++q)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *reinterpret_cast<float4 *>(dst + 32 * q + 8 * c + 4 * e) =
                    make_float4(o[4 * q][2 * x + e] * f, o[4 * q + 1][2 * x + e] * f, o[4 * q + 2][2 * x + e] * f, o[4 * q + 3][2 * x + e] * f);
    }
};

// 16-bit storage: the operands as they are; probabilities as two terms of the storage type.
__device__ __forceinline__ void load4(uint32_t (&r)[4], const void *p)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"((uint32_t)__cvta_generic_to_shared(p)) : "memory");
}
__device__ __forceinline__ void load4_trans(uint32_t (&r)[4], const void *p)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"((uint32_t)__cvta_generic_to_shared(p)) : "memory");
}
__device__ __forceinline__ void mma16(__half, float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16(__nv_bfloat16, float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack(__half, float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t pack(__nv_bfloat16, float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// what packing left of a pair
__device__ __forceinline__ uint32_t pack_rest(__half t, float lo, float hi, uint32_t packed)
{
    const float2 y = __half22float2(*reinterpret_cast<const __half2 *>(&packed));
    return pack(t, lo - y.x, hi - y.y);
}
__device__ __forceinline__ uint32_t pack_rest(__nv_bfloat16 t, float lo, float hi, uint32_t packed)
{
    return pack(t, lo - __uint_as_float(packed << 16), hi - __uint_as_float(packed & 0xffff0000u));      // a bf16 is the upper half of an fp32
}

template <typename T, int D> struct Ops {
    template <int N> static __device__ __forceinline__ void products(float (&s)[N][4], const T *A, const T *B)
    {
        constexpr int LD = Lay<T, D>::LD;
        const int lane = threadIdx.x & 31;
        const T *pa = A + (lane & 15) * LD + (lane >> 4) * 8, *pb = B + ((lane & 7) + (lane >> 4) * 8) * LD + (lane >> 3 & 1) * 8;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
#pragma unroll
        for (int k = 0; k < D; k += 16) {
            uint32_t x[4];
            load4(x, pa + k);
#pragma unroll
            for (int n = 0; n < N; n += 2) {
                uint32_t y[4];
                load4(y, pb + n * 8 * LD + k);
                mma16(T(), s[n], x, y[0], y[1]);
                mma16(T(), s[n + 1], x, y[2], y[3]);
            }
        }
    }
    template <int N> static __device__ __forceinline__ void values(float (&o)[D / 8][4], const float (&s)[N][4], const T *V)
    {
        constexpr int LV = Lay<T, D>::LV;
        const int lane = threadIdx.x & 31;
        const T *pv = V + (lane & 15) * LV + (lane >> 4) * 8;
#pragma unroll
        for (int n = 0; n < N; n += 2) {
            uint32_t p[4], rest[4];                          // a probability is the sum of two terms of the storage type
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float a = s[n + (x >> 1)][2 * (x & 1)], b = s[n + (x >> 1)][2 * (x & 1) + 1];
                p[x] = pack(T(), a, b);
                rest[x] = pack_rest(T(), a, b, p[x]);
            }
#pragma unroll
            for (int d = 0; d < D / 8; d += 2) {
                uint32_t y[4];
                load4_trans(y, pv + n * 8 * LV + d * 8);
                mma16(T(), o[d], rest, y[0], y[1]);
                mma16(T(), o[d + 1], rest, y[2], y[3]);
                mma16(T(), o[d], p, y[0], y[1]);
                mma16(T(), o[d + 1], p, y[2], y[3]);
            }
        }
    }
    static __device__ __forceinline__ void put2(float *dst, float a, float b) { *reinterpret_cast<float2 *>(dst) = make_float2(a, b); }
    static __device__ __forceinline__ void put2(T *dst, float a, float b) { *reinterpret_cast<uint32_t *>(dst) = pack(T(), a, b); }
    template <typename U> static __device__ __forceinline__ void store(U *dst, const float (&o)[D / 8][4], int x, float f)
    {
        const int c = threadIdx.x & 3;
#pragma unroll
        for (int n = 0; n < D / 8; ++n) put2(dst + n * 8 + 2 * c, o[n][2 * x] * f, o[n][2 * x + 1] * f);
    }
};

__device__ __forceinline__ float quad_max(float x)
{
    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
    return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
}
__device__ __forceinline__ float quad_sum(float x)
{
    x += __shfl_xor_sync(0xffffffffu, x, 1);
    return x + __shfl_xor_sync(0xffffffffu, x, 2);
}

template <typename T> __device__ __forceinline__ T *out_row(const AttendArgs &a, const Unit &u, int r)
{
    const int tok = r / a.pv.G, g = r - tok * a.pv.G;
    return static_cast<T *>(a.out) + u.b * a.so.b + (int64_t)(u.h * a.pv.G + g) * a.so.h + (int64_t)tok * a.so.t;
}
__device__ __forceinline__ void store_lse(const AttendArgs &a, const MmaWs &ws, const Unit &u, int r, float z)
{
    const int tok = r / a.pv.G, g = r - tok * a.pv.G;
    const size_t unit = (size_t)u.b * a.pv.H + u.h;
    if (ws.lse2) ws.lse2[unit * a.pv.c * a.pv.G + r] = z;
    if (a.lse) a.lse[(unit * a.pv.G + g) * a.pv.c + tok] = z * 0.6931471805599453f;
}

template <typename T, int D, int R, bool Win>
__global__ void __launch_bounds__(kThreads)
paged_attn_mma_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ MmaWs ws, int row_tiles)
{
    constexpr int LD = Lay<T, D>::LD, LV = Lay<T, D>::LV, kBufs = Lay<T, D>::kBufs, kRows = 16 * R, N = R == 4 ? 8 : 2;
    extern __shared__ __align__(16) uint8_t sm[];
    T *Q = reinterpret_cast<T *>(sm), *K = Q + kRows * LD, *V = K + kBufs * kTile * LD;
    const int G = a.pv.G;
    dependency_wait();
    dependents_may_start();
    const int piece = blockIdx.x % ws.pieces, work = blockIdx.x / ws.pieces;
    // the tiles that see most slots first, of all units
    const int units = a.pv.B * a.pv.H, tile = work / units;
    Unit u = make_unit(a.pv, work - tile * units);
    const int r0 = (row_tiles - 1 - tile) * kRows;
    if (r0 >= u.rows) return;
    if (Win) {
        u.near = near_slots<Win>(a.pv, u.past, r0 / G);
        u.past = u.near.past;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int last_row = min(r0 + kRows, u.rows) - 1;
    const int limit = u.past + last_row / G + 1;         // slots that the last row sees
    const int tiles = (limit + kTile - 1) / kTile;
    const int t0 = (int)((long long)tiles * piece / ws.pieces), t1 = (int)((long long)tiles * (piece + 1) / ws.pieces);
    copy_queries<T, D, kRows>(Q, a, u, r0);
    if (t0 < t1) copy_slots<T, D, kTile, Win>(K, LD, a.pv, u, a.pv.k, t0 * kTile, limit);
    copies_commit();
    if (t0 < t1) copy_slots<T, D, kTile, Win>(V, LV, a.pv, u, a.pv.v, t0 * kTile, limit);
    copies_commit();

    const int wr = R == 4 ? 16 * warp : 0, wk = R == 4 ? 0 : 16 * warp;      // the warp's rows and keys of a tile
    int vis[2];                                          // slots that the lane's rows see
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[D / 8][4];
#pragma unroll
    for (int x = 0; x < 2; ++x) vis[x] = u.past + min(r0 + wr + g + 8 * x, last_row) / G + 1;
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][e] = 0.f;

    for (int t = t0; t < t1; ++t) {
        const int j0 = t * kTile;
        copies_wait<1>();                                 // keys (and queries) are here; values may be on their way
        __syncthreads();
        const int buf = kBufs == 2 ? (t - t0) & 1 : 0, next = kBufs == 2 ? buf ^ 1 : 0;
        auto next_keys = [&] {
            if (t + 1 < t1) copy_slots<T, D, kTile, Win>(K + next * kTile * LD, LD, a.pv, u, a.pv.k, j0 + kTile, limit);
            copies_commit();
        };
        auto next_values = [&] {
            if (t + 1 < t1) copy_slots<T, D, kTile, Win>(V + next * kTile * LV, LV, a.pv, u, a.pv.v, j0 + kTile, limit);
            copies_commit();
        };
        if (kBufs == 2) next_keys();
        float s[N][4];
        Ops<T, D>::template products<N>(s, Q + wr * LD, K + (buf * kTile + wk) * LD);
        if (kBufs == 1) { __syncthreads(); next_keys(); }  // the keys have been read
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            float mx = -INFINITY;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float &v = s[n][2 * x + e];
                    const int j = j0 + wk + n * 8 + 2 * c + e;
                    v = j < vis[x] && (!Win || j >= vis[x] - a.pv.window || j < a.pv.sinks) ? v * a.pv.sl2 : -INFINITY;
                    mx = fmaxf(mx, v);
                }
            const float mn = fmaxf(m[x], reference<kBelow<T>>(quad_max(mx)));
            const float ref = mn == -INFINITY ? 0.f : mn; // nothing seen so far: any finite reference gives zeros
            const float factor = exp2f(m[x] - ref);
            m[x] = mn;
            float sum = 0.f;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float &v = s[n][2 * x + e];
                    v = exp2f(v - ref);
                    sum += v;
                }
            l[x] = fmaf(l[x], factor, sum);               // of this lane's keys
#pragma unroll
            for (int n = 0; n < D / 8; ++n) { o[n][2 * x] *= factor; o[n][2 * x + 1] *= factor; }
        }
        copies_wait<1>();                                 // values are here; the next keys may be on their way
        __syncthreads();
        if (kBufs == 2) next_values();
        Ops<T, D>::template values<N>(o, s, V + (buf * kTile + wk) * LV);
        if (kBufs == 1) { __syncthreads(); next_values(); }      // the values have been read
    }
    copies_wait<0>();
    const size_t rows_all = (size_t)a.pv.B * a.pv.H * a.pv.c * G, row_base = ((size_t)u.b * a.pv.H + u.h) * a.pv.c * G;
#pragma unroll
    for (int x = 0; x < 2; ++x) l[x] = quad_sum(l[x]);
    if constexpr (R == 4) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int r = r0 + wr + g + 8 * x;
            if (r > last_row || !A2SF_IN_RANGE(r, a.pv.c * G, kDbgPagedMma)) continue;
            const bool whole = ws.pieces == 1;
            if (whole) Ops<T, D>::store(out_row<T>(a, u, r), o, x, 1.f / l[x]);
            else       Ops<T, D>::store(ws.o + ((size_t)piece * rows_all + row_base + r) * D, o, x, 1.f);
            if (c == 0) {
                if (whole) store_lse(a, ws, u, r, m[x] + log2f(l[x]));
                else       ws.ml[(size_t)piece * rows_all + row_base + r] = make_float2(m[x], l[x]);
            }
        }
    } else {
        // the four warps' results, joined in shared memory (the keys' and values' place)
        float2 *ml = reinterpret_cast<float2 *>(K);       // [4][16]
        float *part = reinterpret_cast<float *>(ml + 64);  // [4][16][D]
        __syncthreads();
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if (c == 0) ml[warp * 16 + g + 8 * x] = make_float2(m[x], l[x]);
            Ops<T, D>::store(part + (warp * 16 + g + 8 * x) * D, o, x, 1.f);
        }
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * (D / 4); e += kThreads) {
            const int row = e / (D / 4), d4 = e - row * (D / 4), r = r0 + row;
            if (r > last_row || !A2SF_IN_RANGE(r, a.pv.c * G, kDbgPagedMma)) continue;
            float mx = -INFINITY, sum = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) mx = fmaxf(mx, ml[w * 16 + row].x);
            const float ref = mx == -INFINITY ? 0.f : mx;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float2 y = ml[w * 16 + row];
                const float f = exp2f(y.x - ref);
                const float4 p = *reinterpret_cast<const float4 *>(part + (w * 16 + row) * D + d4 * 4);
                sum = fmaf(f, y.y, sum);
                v.x = fmaf(f, p.x, v.x); v.y = fmaf(f, p.y, v.y); v.z = fmaf(f, p.z, v.z); v.w = fmaf(f, p.w, v.w);
            }
            const bool whole = ws.pieces == 1;
            if (whole) {
                T *dst = out_row<T>(a, u, r) + d4 * 4;
                const float f = 1.f / sum;
                if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(dst) = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
                else                          *reinterpret_cast<uint2 *>(dst) = make_uint2(pack(T(), v.x * f, v.y * f), pack(T(), v.z * f, v.w * f));
            } else {
                *reinterpret_cast<float4 *>(ws.o + ((size_t)piece * rows_all + row_base + r) * D + d4 * 4) = v;
            }
            if (d4 == 0) {
                if (whole) store_lse(a, ws, u, r, mx + log2f(sum));
                else       ws.ml[(size_t)piece * rows_all + row_base + r] = make_float2(mx, sum);
            }
        }
    }
}

// A warp per row.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
paged_merge_mma_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ MmaWs ws)
{
    dependency_wait();
    dependents_may_start();
    const int rows = a.pv.c * a.pv.G, lane = threadIdx.x & 31;
    const long long rows_all = (long long)a.pv.B * a.pv.H * rows;
    for (long long x = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); x < rows_all; x += (long long)gridDim.x * (kThreads / 32)) {
        const int unit = (int)(x / rows), r = (int)(x - (long long)unit * rows);
        const Unit u = make_unit(a.pv, unit);
        if (r >= u.rows) continue;
        float mx = -INFINITY, sum = 0.f, v[D / 32];
        for (int p = 0; p < ws.pieces; ++p) mx = fmaxf(mx, ws.ml[p * rows_all + x].x);
#pragma unroll
        for (int e = 0; e < D / 32; ++e) v[e] = 0.f;
        for (int p = 0; p < ws.pieces; ++p) {
            const float2 y = ws.ml[p * rows_all + x];
            const float f = exp2f(y.x - mx);                  // 0 where the piece holds nothing that the row sees
            sum = fmaf(f, y.y, sum);
#pragma unroll
            for (int e = 0; e < D / 32; ++e) v[e] = fmaf(f, ws.o[(p * rows_all + x) * D + e * 32 + lane], v[e]);
        }
        const float inv = 1.f / sum;
        T *dst = out_row<T>(a, u, r);
#pragma unroll
        for (int e = 0; e < D / 32; ++e) dst[e * 32 + lane] = Elem<T>::from_float(v[e] * inv);
        if (lane == 0) store_lse(a, ws, u, r, mx + log2f(sum));
    }
}

// R = 4: 64 slots, 16 a warp, against all rows of a tile.  R = 1: 16 slots, every warp against 16 rows of a tile.
template <typename T, int D, int R>
__global__ void __launch_bounds__(kThreads)
paged_score_mma_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ MmaWs ws)
{
    constexpr int LD = Lay<T, D>::LD, kSlots = 16 * R, N = R == 4 ? 8 : 2;
    extern __shared__ __align__(16) uint8_t sm[];
    T *K = reinterpret_cast<T *>(sm), *Q = K + kSlots * LD;
    float *cr = reinterpret_cast<float *>(Q + 2 * kTile * LD);
    int *seen = reinterpret_cast<int *>(cr + 2 * kTile);
    float *part = cr + 4 * kTile;                         // [4][16]
    const int G = a.pv.G;
    const int units = a.pv.B * a.pv.H, tile = blockIdx.x / units;
    const Unit u = make_unit(a.pv, blockIdx.x - tile * units);
    const int j0 = tile * kSlots, used = u.past + u.len;  // those that most rows see first
    const bool idle = u.len == 0 || j0 >= used;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    // rows before the first weighted token, or before the token that first sees the tile, add nothing
    const int first = idle ? 0 : max(max(first_weighted_token(u.len, a.nl2a), j0 - u.past), 0) * G / kTile * kTile;
    // a thread brings one slot up to date: R = 4: the lane c = 0 of rows g and g + 8 has two
    float old[2] = {0.f, 0.f}, *dst[2] = {nullptr, nullptr};
    const int ws0 = R == 4 ? 16 * warp : 0, wr = R == 4 ? 0 : 16 * warp;     // the warp's slots and rows of a tile
    if (!idle) {
        copy_slots<T, D, kSlots>(K, LD, a.pv, u, a.pv.k, j0, used);
        copy_queries<T, D, kTile>(Q, a, u, first);
        if (c == 0 && (R == 4 || warp == 0)) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int j = j0 + ws0 + g + 8 * x;
                const int page = j < used ? page_for_write(a.pv, u.table, j) : -1;
                if (page < 0) continue;
                dst[x] = a.pv.scores + pool_row(a.pv, page, u.h, j);
                old[x] = *dst[x];
            }
        }
    }
    copies_commit();
    dependency_wait();                                    // everything before does not depend on the attention
    if (idle) { copies_wait<0>(); return; }
    const float *lse2 = ws.lse2 + ((size_t)u.b * a.pv.H + u.h) * a.pv.c * G;
    auto constant = [&](int r, float &k, int &see) {      // of row r, and the slots that it sees
        const int i = r / G;
        k = r < u.rows ? lse2[r] + age_exponent(u.len - 1 - i, a.nl2a) : INFINITY;
        see = r < u.rows ? u.past + i + 1 : 0;
    };
    if (tid < kTile) constant(first + tid, cr[tid], seen[tid]);
    float sum[2] = {0.f, 0.f};
    int buf = 0;
    for (int r0 = first; r0 < u.rows; r0 += kTile, buf ^= 1) {
        copies_wait<0>();
        __syncthreads();                                  // this tile is here, the one before has been read
        const bool more = r0 + kTile < u.rows;
        if (more) copy_queries<T, D, kTile>(Q + (buf ^ 1) * kTile * LD, a, u, r0 + kTile);
        copies_commit();
        float next_c = 0.f;
        int next_seen = 0;
        if (more && tid < kTile) constant(r0 + kTile + tid, next_c, next_seen);
        float s[N][4];
        Ops<T, D>::template products<N>(s, K + ws0 * LD, Q + (buf * kTile + wr) * LD);
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int at = buf * kTile + wr + n * 8 + 2 * c + e;
                const float k = cr[at];
                const int see = seen[at];
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    sum[x] += j0 + ws0 + g + 8 * x < see ? exp2f(fmaf(s[n][2 * x + e], a.pv.sl2, -k)) : 0.f;
            }
        if (more && tid < kTile) { cr[(buf ^ 1) * kTile + tid] = next_c; seen[(buf ^ 1) * kTile + tid] = next_seen; }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) sum[x] = quad_sum(sum[x]);
    if constexpr (R == 1) {
        if (c == 0) { part[warp * 16 + g] = sum[0]; part[warp * 16 + g + 8] = sum[1]; }
        __syncthreads();
#pragma unroll
        for (int x = 0; x < 2; ++x) sum[x] = (part[g + 8 * x] + part[16 + g + 8 * x]) + (part[32 + g + 8 * x] + part[48 + g + 8 * x]);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
        if (dst[x]) *dst[x] = fmaf(old[x], exp2f(-age_exponent(u.len, a.nl2a)), sum[x]);
}

size_t pad(size_t x) { return (x + 255) / 256 * 256; }

// Tiles of 64 rows, each of K's and V's rows read a quarter as often, where they and the pieces that the keys can be cut into
// (two tiles of keys at least, four in 16 bits) are four for every SM; else tiles of 16 rows.  Times in us with tiles of 16 and of 64 rows:
// 64 heads, 2048 tokens, d = 128: 2330 and 1813; 4 heads, 200 x 4 rows behind 20,000 keys: 762 and 498 (no more than two
// pieces an SM: 533); 140 heads, 122 rows: 59 and 80; 16 heads, 129 rows, d = 64: 11.2 and 20.  Scores the same with slots for
// rows, where nothing is cut: 140 heads, 698 slots: 66 and 60; 9 heads, 1204 slots: 152 and 209.
struct Shape {
    bool large;
    long long row_tiles, slot_tiles;
    int pieces;
    bool large_score;
};
Shape shape_of(int dtype, const PagedView &pv, bool windowed)
{
    Shape s;
    const long long units = (long long)pv.B * pv.H, rows = (long long)pv.c * pv.G, cap = near_capacity(pv, windowed, std::min(pv.c, 64));      // of a row tile
    const long long most = std::max(1ll, (cap + kTile - 1) / kTile / (dtype == A2SF_F32 ? 2 : 4)), tiles = units * ((rows + 63) / 64);
    s.large = tiles * most >= 4 * kSms;
    s.row_tiles = s.large ? (rows + 63) / 64 : (rows + 15) / 16;
    s.large_score = units * ((cap + 63) / 64) >= 4 * kSms;
    s.slot_tiles = s.large_score ? (cap + 63) / 64 : (cap + 15) / 16;
    s.pieces = (int)std::min(most, std::max(1ll, 4ll * kSms / (units * s.row_tiles)));
    return s;
}

MmaWs carve(int dtype, const PagedView &pv, bool windowed, void *mem, size_t *bytes)
{
    MmaWs w;
    const size_t rows = (size_t)pv.B * pv.H * pv.G * pv.c;
    w.pieces = shape_of(dtype, pv, windowed).pieces;
    char *base = static_cast<char *>(mem);
    size_t off = 0;
    const size_t parts = w.pieces > 1 ? rows * w.pieces : 0;
    w.lse2 = windowed ? nullptr : reinterpret_cast<float *>(base + off); off += windowed ? 0 : pad(rows * 4);     // for the scores
    w.ml = reinterpret_cast<float2 *>(base + off); off += pad(parts * 8);
    w.o = reinterpret_cast<float *>(base + off); off += pad(parts * pv.d * 4);
    if (bytes) *bytes = off;
    return w;
}

template <typename T, int D, int R, bool Win>
cudaError_t launch_attn(const AttendArgs &a, const MmaWs &ws, long long row_tiles, cudaStream_t s)
{
    const long long grid = (long long)a.pv.B * a.pv.H * row_tiles * ws.pieces;
    if (grid > 0x7fffffffll) return cudaErrorInvalidValue;
    constexpr size_t smem = Lay<T, D>::attn(16 * R);
    cudaError_t e = allow_dynamic_smem<paged_attn_mma_kernel<T, D, R, Win>>(smem);
    if (e == cudaSuccess) e = launch_chained(paged_attn_mma_kernel<T, D, R, Win>, (unsigned)grid, kThreads, smem, s, a, ws, (int)row_tiles);
    if (e == cudaSuccess) count_launch();
    return e;
}
template <typename T, int D, int R>
cudaError_t launch_score(const AttendArgs &a, const MmaWs &ws, long long slot_tiles, cudaStream_t s)
{
    const long long grid = (long long)a.pv.B * a.pv.H * slot_tiles;
    if (grid > 0x7fffffffll) return cudaErrorInvalidValue;
    constexpr size_t smem = Lay<T, D>::score(16 * R);
    cudaError_t e = allow_dynamic_smem<paged_score_mma_kernel<T, D, R>>(smem);
    if (e == cudaSuccess) e = launch_chained(paged_score_mma_kernel<T, D, R>, (unsigned)grid, kThreads, smem, s, a, ws);
    if (e == cudaSuccess) count_launch();
    return e;
}

template <typename T, int D, bool Win>
cudaError_t launch(int dtype, const AttendArgs &a, cudaStream_t s)
{
    const Shape sh = shape_of(dtype, a.pv, Win);
    const MmaWs ws = carve(dtype, a.pv, Win, a.ws, nullptr);
    cudaError_t e = sh.large ? launch_attn<T, D, 4, Win>(a, ws, sh.row_tiles, s) : launch_attn<T, D, 1, Win>(a, ws, sh.row_tiles, s);
    if (e != cudaSuccess) return e;
    if (ws.pieces > 1) {
        const long long rows = (long long)a.pv.B * a.pv.H * a.pv.c * a.pv.G, grid = (rows + 3) / 4;
        e = launch_chained(paged_merge_mma_kernel<T, D>, (unsigned)(grid < 8 * kSms ? grid : 8 * kSms), kThreads, 0, s, a, ws);
        if (e != cudaSuccess) return e;
        count_launch();
    }
    if (Win || !a.scores) return cudaSuccess;
    return sh.large_score ? launch_score<T, D, 4>(a, ws, sh.slot_tiles, s) : launch_score<T, D, 1>(a, ws, sh.slot_tiles, s);
}

template <bool Win>
cudaError_t launch(int dtype, const AttendArgs &a, cudaStream_t s)
{
    const bool wide = a.pv.d == 128;
    switch (dtype) {
    case A2SF_F32: return wide ? launch<float, 128, Win>(dtype, a, s) : launch<float, 64, Win>(dtype, a, s);
    case A2SF_BF16: return wide ? launch<__nv_bfloat16, 128, Win>(dtype, a, s) : launch<__nv_bfloat16, 64, Win>(dtype, a, s);
    default: return wide ? launch<__half, 128, Win>(dtype, a, s) : launch<__half, 64, Win>(dtype, a, s);
    }
}

}  // namespace

size_t attend_mma_ws_bytes(int dtype, const PagedView &pv, bool windowed)
{
    size_t bytes = 0;
    carve(dtype, pv, windowed, nullptr, &bytes);
    return bytes;
}

cudaError_t launch_attend_mma(int dtype, const AttendArgs &a, cudaStream_t s)
{
    return a.windowed ? launch<true>(dtype, a, s) : launch<false>(dtype, a, s);
}

}  // namespace a2sf
