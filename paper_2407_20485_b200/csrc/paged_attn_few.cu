// Attention of a few rows (len * G <= 16: generation, drafted tokens) over a paged cache.
//
// Every K and V row is read once and used for at most 16 rows: the cache's bytes bound this, and there
// may be one long sequence or a thousand ragged ones.  So the work is cut without regard to either: the
// 64-slot tiles of all (sequence, K/V head) units form one list, every CTA takes an equal, contiguous
// share, and a share that begins or ends inside a unit leaves partial results that the finish kernel joins.
// The list is built on the device from past and lens (the host knows neither).
//
//   main    warp 0 copies tiles (K and V, TMA boxes of up to a page, 128-byte swizzle) into a ring;
//           consumer warps take 16 slots (32 for d = 64, 8 in 32-bit storage) of each tile and keep their own running
//           maximum, sum and output.  16-bit storage: S[16 slots x 8 rows] = K Q^T and O^T[d x 8] += V^T P^T
//           on mma.sync m16n8k16, K and V^T straight from ldmatrix (.trans for V); P changes from
//           accumulator to operand layout with movmatrix.  The rows fill 8 of the instruction's columns, so
//           the tensor rate is of no account and tcgen05 (128 rows at least) would compute on padding.
//           32-bit storage: the same on the CUDA cores, a lane working on a quarter of a key.  Logits go to the workspace (4 bytes per slot and
//           row next to 4 d or 8 d bytes of K and V) so that scores need no second pass over K.
//   finish  joins the partial outputs; S <- alpha^len S + sum_r alpha^age exp2(x_r - lse_r).
//   whole   instead of both where no sequence can have more than a few tiles: a CTA takes whole units, keeps
//           logits and partial results in shared memory and ends each unit itself.
// Windowed (Win): the same over the near slots of a sequence (see Near), which is all that it sees; no logits are kept, and the
// finish kernel joins outputs alone.  Few units take a form of their own:
//   cluster a cluster of CTAs per unit, joined through their shared memory.
// P goes into P V as two terms of the storage type (off by the square of half a step; one term would be off by half a
// step of every product, which shows where products cancel), as in the steps of the slot cache.  The memory time hides it: one
// token over 32 x 40 caches of up to 4096 slots 241 us with one term, 242 with two; four tokens, G = 4, over 2 x 8 x 32,700
// slots 61.4 and 62.0.  The row sum and the scores use the unrounded values.
#include <type_traits>

#include "paged.cuh"
#include "tc_sm100.cuh"

namespace a2sf {

A2SF_DEBUG_TRANSLATION_UNIT(paged_attn_few)

namespace {

using namespace tc;

// Slots of a tile: 16 KB of K and of V for 16-bit rows of either size.
template <typename T, int D> constexpr int tile_slots = D * sizeof(T) == 128 ? 128 : 64;
// Consumer warps of a CTA.  32-bit storage spends 8 times the instructions on a slot and runs one CTA per SM
// (d = 128), so twice as many warps share a tile there to hide each other's latencies.
template <typename T> constexpr int warps_of = sizeof(T) == 4 ? 8 : 4;
constexpr int kFinishThreads = 256;
constexpr int kSms = 148;
// A column's reference is what is subtracted before the exponential (log2 units).  It is set kBelow under the maximum and stays
// until a logit lies more than kSlack above it.  bf16 and fp32 have the range for any: sums of 2^14 and of values up to
// 2^113 / slots stay finite.  fp16 has not: what falls under 2^-24 packs to 0 while the row sum still counts it, and from 2^-14
// down there are fewer bits.  So its probabilities use the range up to 2^15, and that begins 2^-37 and 2^-27 under the maximum.
template <typename T> constexpr int kBelow = std::is_same<T, __half>::value ? 13 : 0;
template <typename T> constexpr float kSlack = std::is_same<T, __half>::value ? 15.f : 14.f;

__host__ __device__ constexpr int rows_padded(int rows) { return rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : rows <= 8 ? 8 : 16; }

template <typename T, int D> struct Ring {
    static constexpr int kTile = tile_slots<T, D>;
    static constexpr int kRowBytes = D * (int)sizeof(T);
    static constexpr int kChunks = kRowBytes / 128;                // 128-byte columns of a tile
    static constexpr int kTileBytes = kTile * kRowBytes;           // K or V
    static constexpr int kStages = kRowBytes == 512 ? 2 : 3;
    static constexpr size_t kBytes = (size_t)kStages * 2 * kTileBytes + 1024;
};

struct FewWs {
    float *logits;        // [U][slots][NP], log2 units
    float2 *ml;           // [segments][warps][NP] reference (log2 units), sum
    float *o;             // [segments][warps][NP][D]
    int32_t *prefix;      // [B + 1] tiles of a head, summed over the sequences before
    int slots;            // padded slots of a unit
    int segs;             // segments that there is room for, times warps
};

template <typename T> struct Mma16;
template <> struct Mma16<__half> {
    __device__ static void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    __device__ static uint32_t pack(float lo, float hi)
    {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    __device__ static void subtract(float (&x)[2], uint32_t packed)
    {
        const float2 y = __half22float2(*reinterpret_cast<const __half2 *>(&packed));
        x[0] -= y.x; x[1] -= y.y;
    }
};
template <> struct Mma16<__nv_bfloat16> {
    __device__ static void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    __device__ static uint32_t pack(float lo, float hi)
    {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    __device__ static void subtract(float (&x)[2], uint32_t packed)      // a bf16 is the upper half of an fp32
    {
        x[0] -= __uint_as_float(packed << 16);
        x[1] -= __uint_as_float(packed & 0xffff0000u);
    }
};

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Byte offset of 16-byte piece `piece` of row `row` in a tile of 128-byte columns (TMA's 128-byte swizzle).
template <int Tile> __device__ __forceinline__ uint32_t tile_offset(int row, int piece)
{
    return (uint32_t)((piece >> 3) * (Tile * 128) + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
}

__device__ __forceinline__ const void *query_row(const AttendArgs &a, int b, int h, int r, size_t elem)
{
    const int i = r / a.pv.G, g = r - i * a.pv.G;
    return static_cast<const char *>(a.q) + (b * a.sq.b + (int64_t)(h * a.pv.G + g) * a.sq.h + (int64_t)i * a.sq.t) * elem;
}

// ---- a consumer warp on 16-bit storage: NC = 4, 8 or 16 rows ----------------------------------------
// A probability is the sum of two terms of the storage type: hi, and lo, what rounding to hi left.  Up to four rows (kBeside) use
// half of the instruction's columns: the other half gets the same rows, lo is what they bring into P V, and end() adds the
// two.  It is a kernel of its own: with both forms in one, one token over 32 x 40 caches takes 247 us and not 242.
template <typename T, int D, int NC, bool Win> struct Body16 {
    static constexpr bool kBeside = NC == 4;
    static constexpr int CG = kBeside ? 1 : NC / 8, KS = D / 16, kTile = tile_slots<T, D>, kSub = kTile / warps_of<T> / 16;
    uint32_t q[CG][KS][2];
    float o[CG][KS][4], m[CG][2], l[CG][2];
    int vis[CG][2], dead;

    __device__ void begin(const AttendArgs &a, const Where &x, const SeqState &st, const Near &near, float *)
    {
        dead = near.dead;
        const int lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3, rows = st.len * a.pv.G;
#pragma unroll
        for (int g = 0; g < CG; ++g) {
            const int row = (g * 8 + r) % NC;
            const uint32_t *src = row < rows ? static_cast<const uint32_t *>(query_row(a, x.b, x.h, row, sizeof(T))) : nullptr;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                q[g][k][0] = src ? src[k * 8 + c] : 0u;
                q[g][k][1] = src ? src[k * 8 + c + 4] : 0u;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[g][k][e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int col = (g * 8 + 2 * c + e) % NC;
                vis[g][e] = col < rows ? st.past + col / a.pv.G + 1 : 0;
                m[g][e] = -INFINITY;
                l[g][e] = 0.f;
            }
        }
    }

    // kSub x 16 slots from j0 on (rows `row0` .. of the tile); `used` slots of the sequence hold tokens
    __device__ void tile(const AttendArgs &a, uint8_t *K, uint8_t *V, int row0, int j0, int used, float *logits, int NP, float *)
    {
        const int lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
        float x[kSub][CG][4];
        const uint32_t kb = smem_u32(K), vb = smem_u32(V);
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
#pragma unroll
            for (int g = 0; g < CG; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[u][g][e] = 0.f;
            const int row = row0 + u * 16 + (lane & 15), piece = lane >> 4;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                uint32_t f[4];
                ldmatrix4(f, kb + tile_offset<kTile>(row, 2 * k + piece));
#pragma unroll
                for (int g = 0; g < CG; ++g) Mma16<T>::mma(x[u][g], f, q[g][k][0], q[g][k][1]);
            }
        }
        // what lies behind the sequence may be anything: its keys are masked, its values made zero
        if (j0 + kSub * 16 > used || (Win && j0 < dead && j0 + kSub * 16 > a.pv.sinks)) {
            for (int e = lane; e < kSub * 16 * (D / 8); e += 32) {
                const int rr = e / (D / 8);
                if (j0 + rr >= used || (Win && j0 + rr < dead && j0 + rr >= a.pv.sinks)) *reinterpret_cast<uint4 *>(V + tile_offset<kTile>(row0 + rr, e % (D / 8))) = make_uint4(0, 0, 0, 0);
            }
            fence_async_smem();            // these writes come before the copy that next fills the stage
            __syncwarp();
        }
        // The reference of a column moves only when a logit exceeds it by more than kSlack: probabilities up to 2^kSlack
        // are as exact, and no maximum is looked for in between.
        bool beyond = false;
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int g = 0; g < CG; ++g) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = j0 + u * 16 + r + (e >> 1) * 8;
                    const bool seen = j < vis[g][e & 1] && (!Win || j >= vis[g][e & 1] - a.pv.window || j < a.pv.sinks);
                    x[u][g][e] = seen ? x[u][g][e] * a.pv.sl2 : -INFINITY;
                    beyond |= x[u][g][e] - m[g][e & 1] > kSlack<T>;       // also where m is still -inf; the difference is exact
                }
                if (logits) {
                    const int col = g * 8 + 2 * c;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float *dst = logits + (size_t)(j0 + u * 16 + r + half * 8) * NP + col;
                        if (col + 1 < NP) *reinterpret_cast<float2 *>(dst) = make_float2(x[u][g][2 * half], x[u][g][2 * half + 1]);
                        else if (col < NP) *dst = x[u][g][2 * half];
                    }
                }
            }
        if (__any_sync(0xffffffffu, beyond)) {
#pragma unroll
            for (int g = 0; g < CG; ++g) {
                float f[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float mx = fmaxf(x[0][g][e], x[0][g][e + 2]);
#pragma unroll
                    for (int u = 1; u < kSub; ++u) mx = fmaxf(mx, fmaxf(x[u][g][e], x[u][g][e + 2]));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                    const float mn = fmaxf(m[g][e], reference<kBelow<T>>(mx));
                    f[e] = mn == -INFINITY ? 1.f : ex2(m[g][e] - mn);
                    m[g][e] = mn;
                    l[g][e] *= f[e];
                }
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[g][k][e] *= f[e & 1];
            }
        }
        uint32_t p[kSub][CG][2], rest[kSub][CG][2];
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int g = 0; g < CG; ++g) {
                float w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    // nothing seen so far: any finite reference gives the zeros that are wanted
                    w[e] = ex2(x[u][g][e] - (m[g][e & 1] == -INFINITY ? 0.f : m[g][e & 1]));
                    l[g][e & 1] += w[e];
                }
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t hi = Mma16<T>::pack(w[2 * half], w[2 * half + 1]);
                    float left[2] = {w[2 * half], w[2 * half + 1]};
                    Mma16<T>::subtract(left, hi);
                    const uint32_t lo = Mma16<T>::pack(left[0], left[1]);
                    if (!kBeside) rest[u][g][half] = movmatrix_trans(lo);
                    p[u][g][half] = movmatrix_trans(kBeside && c >= 2 ? lo : hi);
                }
            }
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
            const int row = row0 + u * 16 + (lane >> 4) * 8 + (lane & 7), piece = (lane >> 3) & 1;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                uint32_t v[4];
                ldmatrix4_trans(v, vb + tile_offset<kTile>(row, 2 * k + piece));
#pragma unroll
                for (int g = 0; g < CG; ++g)
                    if (!kBeside) Mma16<T>::mma(o[g][k], v, rest[u][g][0], rest[u][g][1]);
#pragma unroll
                for (int g = 0; g < CG; ++g) Mma16<T>::mma(o[g][k], v, p[u][g][0], p[u][g][1]);
            }
        }
    }

    __device__ void end(float2 *ml, float *op, int NP)
    {
        const int lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
        if (kBeside) {
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[0][k][e] += __shfl_xor_sync(0xffffffffu, o[0][k][e], 2);
        }
#pragma unroll
        for (int g = 0; g < CG; ++g)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float sum = l[g][e];
                sum += __shfl_xor_sync(0xffffffffu, sum, 4);
                sum += __shfl_xor_sync(0xffffffffu, sum, 8);
                sum += __shfl_xor_sync(0xffffffffu, sum, 16);
                const int col = g * 8 + 2 * c + e;
                if (col >= NP) continue;
                if (r == 0) ml[col] = make_float2(m[g][e], sum);
                if (m[g][e] == -INFINITY) continue;         // the row saw nothing here: no output is read either
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    op[(size_t)col * D + k * 16 + r] = o[g][k][e];
                    op[(size_t)col * D + k * 16 + 8 + r] = o[g][k][2 + e];
                }
            }
    }
};

// ---- a consumer warp on 32-bit storage: NC rows, all in use or zero ----------------------------------
template <int D, int NC, bool Win> struct Body32 {
    static constexpr int DV = D / 32;                       // output elements per lane
    static constexpr int QP = D / 4, QS = QP + 4;           // a quarter of a query, and its distance in shared memory
    float o[NC][DV], m[NC], l[NC];
    int rows, G, past, dead;
    unsigned long long tokens;                              // token of row r in bits 4r .. 4r+3

    __device__ int seen_by(int r) const { return r < rows ? (int)(tokens >> (4 * r) & 15) + 1 : -(1 << 30); }

    // scratch: [NC][4][QS] queries, shared by the consumer warps, then [8][NC] probabilities of each warp
    __device__ void begin(const AttendArgs &a, const Where &x, const SeqState &st, const Near &near, float *scratch)
    {
        constexpr int kThreads = 32 * warps_of<float>;
        const int tid = threadIdx.x - 32;
        rows = st.len * a.pv.G; G = a.pv.G; past = st.past; dead = near.dead;
        tokens = 0;
        for (int r = 0; r < rows; ++r) tokens |= (unsigned long long)(r / G) << (4 * r);
        named_barrier(1, kThreads);                         // the unit before has been worked off
#pragma unroll
        for (int e = tid; e < NC * (D / 4); e += kThreads) {
            const int r = e / (D / 4), k = e % (D / 4) * 4;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r < rows) v = *reinterpret_cast<const float4 *>(static_cast<const float *>(query_row(a, x.b, x.h, r, 4)) + k);
            *reinterpret_cast<float4 *>(scratch + (r * 4 + k / QP) * QS + k % QP) = v;
        }
        named_barrier(1, kThreads);
#pragma unroll
        for (int r = 0; r < NC; ++r) {
            m[r] = -INFINITY; l[r] = 0.f;
#pragma unroll
            for (int e = 0; e < DV; ++e) o[r][e] = 0.f;
        }
    }

    // 8 slots j0 .. j0+7, rows `row0` .. of the tile
    __device__ void tile(const AttendArgs &a, uint8_t *K, uint8_t *V, int row0, int j0, int used, float *logits, int, float *scratch)
    {
        const int lane = threadIdx.x & 31, s = lane & 7, part = lane >> 3;
        float *P = scratch + NC * 4 * QS + ((threadIdx.x >> 5) - 1) * 8 * NC;
        float acc[NC];
#pragma unroll
        for (int r = 0; r < NC; ++r) acc[r] = 0.f;
        const float *qq = scratch + part * QS;
#pragma unroll 4
        for (int k = 0; k < QP; k += 4) {
            const float4 kk = *reinterpret_cast<const float4 *>(K + tile_offset<tile_slots<float, D>>(row0 + s, (part * QP + k) / 4));
#pragma unroll
            for (int r = 0; r < NC; ++r) {
                const float4 q = *reinterpret_cast<const float4 *>(qq + r * 4 * QS + k);
                acc[r] = fmaf(q.x, kk.x, acc[r]);
                acc[r] = fmaf(q.y, kk.y, acc[r]);
                acc[r] = fmaf(q.z, kk.z, acc[r]);
                acc[r] = fmaf(q.w, kk.w, acc[r]);
            }
        }
        const int j = j0 + s;
        __syncwarp();                                       // the previous tile's probabilities have been read
        // references move as in Body16
        bool beyond = false;
#pragma unroll
        for (int r = 0; r < NC; ++r) {
            acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], 8);
            acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], 16);
            const int top = past + seen_by(r);
            const bool seen = j < top && (!Win || j >= top - a.pv.window || j < a.pv.sinks);
            acc[r] = seen ? acc[r] * a.pv.sl2 : -INFINITY;
            if (logits && part == r % 4) logits[(size_t)j * NC + r] = acc[r];
            beyond |= acc[r] - m[r] > kSlack<float>;
        }
        if (__any_sync(0xffffffffu, beyond)) {
#pragma unroll
            for (int r = 0; r < NC; ++r) {
                float mx = acc[r];
#pragma unroll
                for (int w = 4; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
                const float mn = fmaxf(m[r], mx), f = mn == -INFINITY ? 1.f : exp2f(m[r] - mn);
                m[r] = mn;
                l[r] *= f;
#pragma unroll
                for (int e = 0; e < DV; ++e) o[r][e] *= f;
            }
        }
#pragma unroll
        for (int r = 0; r < NC; ++r) {
            const float p = exp2f(acc[r] - (m[r] == -INFINITY ? 0.f : m[r]));
            l[r] += p;                                      // every quarter-warp holds the sum over its 8 slots
            if (part == r % 4) P[s * NC + r] = p;
        }
        __syncwarp();
        const int n = min(8, used - j0);                    // values behind the sequence are not touched
#pragma unroll 4
        for (int x = 0; x < n; ++x) {
            if (Win && j0 + x < dead && j0 + x >= a.pv.sinks) continue;
            float v[DV], p[NC];
            const uint8_t *src = V + tile_offset<tile_slots<float, D>>(row0 + x, lane * DV / 4) + (lane * DV % 4) * 4;
#pragma unroll
            for (int e = 0; e < DV; e += 2) *reinterpret_cast<float2 *>(v + e) = *reinterpret_cast<const float2 *>(src + e * 4);
#pragma unroll
            for (int r = 0; r < NC; ++r) p[r] = P[x * NC + r];
#pragma unroll
            for (int r = 0; r < NC; ++r)
#pragma unroll
                for (int e = 0; e < DV; ++e) o[r][e] = fmaf(p[r], v[e], o[r][e]);
        }
    }

    __device__ void end(float2 *ml, float *op, int)
    {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int r = 0; r < NC; ++r) {
            float sum = l[r];
#pragma unroll
            for (int w = 4; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
            if (lane == 0) ml[r] = make_float2(m[r], sum);
            if (m[r] == -INFINITY) continue;
#pragma unroll
            for (int e = 0; e < DV; e += 2) *reinterpret_cast<float2 *>(op + (size_t)r * D + lane * DV + e) = make_float2(o[r][e], o[r][e + 1]);
        }
    }
};

template <typename T, int D, int NC, bool Win> struct BodyOf { typedef Body16<T, D, NC, Win> type; static constexpr size_t kScratch = 0; };
template <int D, int NC, bool Win> struct BodyOf<float, D, NC, Win> {
    typedef Body32<D, NC, Win> type;
    static constexpr size_t kScratch = (size_t)(NC * 4 * (D / 4 + 4) + warps_of<float> * 8 * NC) * sizeof(float);
};

struct FewShared {
    uint64_t full[6], empty[6];
    int abort_flag;
    int32_t prefix[A2SF_PAGED_MAX_SEQUENCES + 1];
};

template <typename T, int D, int NC, bool Win>
__global__ void __launch_bounds__(32 * (warps_of<T> + 1))
paged_few_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                 const __grid_constant__ AttendArgs a, const __grid_constant__ FewWs ws, int NP)
{
    using R = Ring<T, D>;
    using Body = typename BodyOf<T, D, NC, Win>::type;
    constexpr int kTile = R::kTile, kWarps = warps_of<T>, kSlots = kTile / kWarps;     // slots per warp and tile
    extern __shared__ uint8_t smem_raw[];
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ FewShared sh;
    const PagedView &pv = a.pv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int *abort_flag = &sh.abort_flag;

    if (warp == 0) {
        if (lane == 0) {
            for (int s = 0; s < R::kStages; ++s) { mbar_init(&sh.full[s], 1); mbar_init(&sh.empty[s], kWarps); }
            sh.abort_flag = 0;
            fence_mbar_init();
            prefetch_tmap(&map_k);
            prefetch_tmap(&map_v);
        }
        dependency_wait();
        tile_prefix<kTile, Win>(sh.prefix, pv);
    }
    if (warp != 0) dependency_wait();
    __syncthreads();
    if (blockIdx.x == 0)
        for (int b = threadIdx.x; b <= pv.B; b += 32 * (kWarps + 1)) ws.prefix[b] = sh.prefix[b];
    dependents_may_start();
    const long long total = (long long)pv.H * sh.prefix[pv.B];
    const long long share = (total + gridDim.x - 1) / gridDim.x;
    const long long w0 = blockIdx.x * share, w1 = w0 + share < total ? w0 + share : total;
    if (w0 >= w1) return;
    Where x = locate(sh.prefix, pv.B, pv.H, w0);

    if (warp == 0) {
        // ---- producer: lane i copies box i of the tile --------------------------------------------
        const int box = box_rows<Win>(pv, kTile), boxes = kTile / box;
        const uint64_t policy = policy_evict_first();     // read once: the logits are to stay in L2 instead
        int it = 0;
        for (long long w = w0; w < w1;) {
            Near near;
            const SeqState st = near_state<Win>(pv, x.b, near);
            const int used = st.past + st.len;
            const int32_t *table = pv.table + (size_t)x.b * pv.max_pages;
            for (; x.t < x.tiles && w < w1; ++x.t, ++w, ++it) {
                const int s = it % R::kStages;
                const int slot = x.t * kTile + lane * box;
                const int nbox = min(boxes, (used - x.t * kTile + box - 1) / box);
                int row = 0;
                if (lane < nbox) {
                    const int real = real_slot<Win>(pv, near, slot);
                    row = (int)pool_row(pv, page_for_read(pv, table, real), x.h, real);
                }
                int ok = 1;
                if (lane == 0) {
                    if (it >= R::kStages) ok = mbar_wait(&sh.empty[s], ((it / R::kStages) & 1) ^ 1, abort_flag) ? 1 : 0;
                    if (ok) mbar_arrive_expect_tx(&sh.full[s], (uint32_t)(nbox * box * R::kRowBytes * 2));
                }
                if (!__shfl_sync(0xffffffffu, ok, 0)) goto drained;
                if (lane < nbox) {
                    uint8_t *dst = ring + (size_t)s * 2 * R::kTileBytes + lane * box * 128;
#pragma unroll
                    for (int ch = 0; ch < R::kChunks; ++ch) {
                        tma_load_2d(dst + ch * (kTile * 128), &map_k, &sh.full[s], ch * (128 / (int)sizeof(T)), row, policy);
                        tma_load_2d(dst + R::kTileBytes + ch * (kTile * 128), &map_v, &sh.full[s], ch * (128 / (int)sizeof(T)), row, policy);
                    }
                }
                __syncwarp();
            }
            if (w < w1) next_unit(x, sh.prefix, pv.B, pv.H);
        }
drained:
        if (lane == 0 && *abort_flag) {
            // copies still in flight get a bounded chance to land before the CTA exits
            int dummy = 0;
            for (int k = max(0, it - R::kStages); k < it; ++k)
                mbar_wait(&sh.full[k % R::kStages], (k / R::kStages) & 1, &dummy);
            *pv.status = A2SF_ERR_TIMEOUT;
        }
    } else {
        // ---- consumers ---------------------------------------------------------------------------
        const int cw = warp - 1;
        float *scratch = reinterpret_cast<float *>(ring + (size_t)R::kStages * 2 * R::kTileBytes);
        Body body;
        int it = 0;
        for (long long w = w0; w < w1;) {
            Near near;
            const SeqState st = near_state<Win>(pv, x.b, near);
            const int used = st.past + st.len;
            const int unit = x.b * pv.H + x.h;
            float *logits = !Win && a.scores ? ws.logits + (size_t)unit * ws.slots * NP : nullptr;
            body.begin(a, x, st, near, scratch);
            for (; x.t < x.tiles && w < w1; ++x.t, ++w, ++it) {
                const int s = it % R::kStages;
                if (!*abort_flag && !mbar_wait(&sh.full[s], (it / R::kStages) & 1, abort_flag)) *pv.status = A2SF_ERR_TIMEOUT;
                const int j0 = x.t * kTile + cw * kSlots;
                uint8_t *K = ring + (size_t)s * 2 * R::kTileBytes;
                if (j0 < used && A2SF_IN_RANGE(j0 + kSlots - 1, ws.slots, kDbgPagedFew)) body.tile(a, K, K + R::kTileBytes, cw * kSlots, j0, used, logits, NP, scratch);
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.empty[s]);
            }
            // segment = CTA + unit: both only grow along the list, one of them at every boundary
            const size_t seg = ((size_t)blockIdx.x + unit) * kWarps + cw;
            if (A2SF_IN_RANGE(seg, ws.segs, kDbgPagedFew)) body.end(ws.ml + seg * NP, ws.o + seg * NP * D, NP);
            if (w < w1) next_unit(x, sh.prefix, pv.B, pv.H);
        }
    }
}

// ---- short caches: whole units ---------------------------------------------------------------------
// Sequences of at most so many tiles: the second kernel of the split costs more (us, split and whole: 32 heads x 205 slots,
// d 128, 8.6 and 7.3; 12 x 4, d 64, 7.8 and 4.5) than a share of fewer tiles saves (8 heads x 496: 8.2 and 11.3).  Where
// there are units for every SM, twice as many (256 heads x 496: 19.1 and 15.7; 400 x 1001, again twice: 40 and 51).
constexpr int kWholeTiles = 4, kWholeTilesMany = 8;

// Shared memory behind the ring and the scratch: (maximum, sum) and output of every warp, logits of all slots.
__host__ __device__ constexpr size_t whole_bytes(int warps, int D, int NP, int slots) { return (size_t)NP * (warps * (8 + D * 4) + slots * 4); }

struct WholeShared {
    uint64_t full[3], empty[3];
    int abort_flag;
    float row_m[kFewRows], row_inv[kFewRows], row_c[kFewRows];
};

template <typename T, int D, int NC, bool Win>
__global__ void __launch_bounds__(32 * (warps_of<T> + 1))
paged_few_whole_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                       const __grid_constant__ AttendArgs a, int NP, int slots)
{
    using R = Ring<T, D>;
    using Body = typename BodyOf<T, D, NC, Win>::type;
    constexpr int kTile = R::kTile, kWarps = warps_of<T>, kSlots = kTile / kWarps, kConsumers = 32 * kWarps;
    constexpr int kPer = kWholeTiles * kTile / kConsumers;          // slots of a thread whose old scores are asked for early
    extern __shared__ uint8_t smem_raw[];
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ WholeShared sh;
    const PagedView &pv = a.pv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, units = pv.B * pv.H;
    volatile int *abort_flag = &sh.abort_flag;
    if (threadIdx.x == 0) {
        for (int s = 0; s < R::kStages; ++s) { mbar_init(&sh.full[s], 1); mbar_init(&sh.empty[s], kWarps); }
        sh.abort_flag = 0;
        fence_mbar_init();
        prefetch_tmap(&map_k);
        prefetch_tmap(&map_v);
    }
    dependency_wait();
    __syncthreads();
    dependents_may_start();

    if (warp == 0) {
        const int box = box_rows<Win>(pv, kTile), boxes = kTile / box;
        int it = 0;
        for (int u = blockIdx.x; u < units; u += gridDim.x) {
            const int b = u / pv.H, h = u - b * pv.H;
            Near near;
            const SeqState st = near_state<Win>(pv, b, near);
            const int used = st.len > 0 ? st.past + st.len : 0;
            const int32_t *table = pv.table + (size_t)b * pv.max_pages;
            for (int t = 0; t * kTile < used; ++t, ++it) {
                const int s = it % R::kStages;
                const int slot = t * kTile + lane * box;
                const int nbox = min(boxes, (used - t * kTile + box - 1) / box);
                int row = 0;
                if (lane < nbox) {
                    const int real = real_slot<Win>(pv, near, slot);
                    row = (int)pool_row(pv, page_for_read(pv, table, real), h, real);
                }
                int ok = 1;
                if (lane == 0) {
                    if (it >= R::kStages) ok = mbar_wait(&sh.empty[s], ((it / R::kStages) & 1) ^ 1, abort_flag) ? 1 : 0;
                    if (ok) mbar_arrive_expect_tx(&sh.full[s], (uint32_t)(nbox * box * R::kRowBytes * 2));
                }
                if (!__shfl_sync(0xffffffffu, ok, 0)) goto drained;
                if (lane < nbox) {
                    uint8_t *dst = ring + (size_t)s * 2 * R::kTileBytes + lane * box * 128;
#pragma unroll
                    for (int ch = 0; ch < R::kChunks; ++ch) {
                        tma_load_2d(dst + ch * (kTile * 128), &map_k, &sh.full[s], ch * (128 / (int)sizeof(T)), row);
                        tma_load_2d(dst + R::kTileBytes + ch * (kTile * 128), &map_v, &sh.full[s], ch * (128 / (int)sizeof(T)), row);
                    }
                }
                __syncwarp();
            }
        }
drained:
        if (lane == 0 && *abort_flag) {
            int dummy = 0;                                   // copies still in flight get a bounded chance to land
            for (int k = max(0, it - R::kStages); k < it; ++k)
                mbar_wait(&sh.full[k % R::kStages], (k / R::kStages) & 1, &dummy);
            *pv.status = A2SF_ERR_TIMEOUT;
        }
        return;
    }
    const int cw = warp - 1, ct = threadIdx.x - 32;
    float *scratch = reinterpret_cast<float *>(ring + (size_t)R::kStages * 2 * R::kTileBytes);
    const bool scores = !Win && a.scores;
    float2 *ml = reinterpret_cast<float2 *>(reinterpret_cast<uint8_t *>(scratch) + BodyOf<T, D, NC, Win>::kScratch);
    float *o = reinterpret_cast<float *>(ml + kWarps * NP);
    float *logits = scores ? o + (size_t)kWarps * NP * D : nullptr;
    Body body;
    int it = 0;
    for (int u = blockIdx.x; u < units; u += gridDim.x) {
        Where x = {};
        x.b = u / pv.H;
        x.h = u - x.b * pv.H;
        Near near;
        const SeqState st = near_state<Win>(pv, x.b, near);
        if (st.len <= 0) continue;
        const int used = st.past + st.len, rows = st.len * pv.G;
        const int32_t *table = pv.table + (size_t)x.b * pv.max_pages;
        // old scores are asked for here and used at the unit's end
        int row[kPer];
        float old[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int j = ct + e * kConsumers;
            row[e] = scores && j < used ? page_for_write(pv, table, j) : -1;
        }
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (row[e] >= 0) {
                row[e] = (int)pool_row(pv, row[e], x.h, ct + e * kConsumers);
                old[e] = pv.scores[row[e]];
            }
        body.begin(a, x, st, near, scratch);
        for (int t = 0; t * kTile < used; ++t, ++it) {
            const int s = it % R::kStages;
            if (!*abort_flag && !mbar_wait(&sh.full[s], (it / R::kStages) & 1, abort_flag)) *pv.status = A2SF_ERR_TIMEOUT;
            const int j0 = t * kTile + cw * kSlots;
            uint8_t *K = ring + (size_t)s * 2 * R::kTileBytes;
            if (j0 < used && A2SF_IN_RANGE(j0 + kSlots - 1, slots, kDbgPagedFew)) body.tile(a, K, K + R::kTileBytes, cw * kSlots, j0, used, logits, NP, scratch);
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.empty[s]);
        }
        body.end(ml + cw * NP, o + (size_t)cw * NP * D, NP);
        named_barrier(1, kConsumers);
        if (ct < NP) {
            float mx = -INFINITY, l = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) mx = fmaxf(mx, ml[w * NP + ct].x);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float2 y = ml[w * NP + ct];
                l += y.y != 0.f ? ex2(y.x - mx) * y.y : 0.f;     // 0: saw nothing; a NaN stays one, also beside no maximum
            }
            const float z = mx + log2f(l);
            const int i = ct / pv.G, g = ct - i * pv.G;
            sh.row_m[ct] = mx;
            sh.row_inv[ct] = 1.f / l;
            sh.row_c[ct] = ct < rows ? z + age_exponent(st.len - 1 - i, a.nl2a) : INFINITY;
            if (ct < rows && a.lse) a.lse[((size_t)u * pv.G + g) * pv.c + i] = z * 0.6931471805599453f;
        }
        named_barrier(1, kConsumers);
        const float decay = exp2f(-age_exponent(st.len, a.nl2a));
        auto gain = [&](int j) {                             // rows that do not see the slot, or are none, have -inf there
            const float *z = logits + j * NP;
            float sum = 0.f;
            for (int r = 0; r < NP; ++r) sum += ex2(z[r] - sh.row_c[r]);
            return sum;
        };
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (row[e] >= 0) pv.scores[row[e]] = fmaf(old[e], decay, gain(ct + e * kConsumers));
        if (scores)
            for (int j = ct + kPer * kConsumers; j < used; j += kConsumers) {
                const int page = page_for_write(pv, table, j);
                if (page < 0) continue;
                float *dst = pv.scores + pool_row(pv, page, x.h, j);
                *dst = fmaf(*dst, decay, gain(j));
            }
        for (int e = ct; e < rows * (D / 4); e += kConsumers) {
            const int r = e / (D / 4), d4 = e - r * (D / 4);
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = ex2(ml[w * NP + r].x - sh.row_m[r]);
                if (!(f > 0.f)) continue;                    // a warp that saw nothing wrote no output
                const float4 v = reinterpret_cast<const float4 *>(o + (size_t)(w * NP + r) * D)[d4];
                sum.x = fmaf(f, v.x, sum.x); sum.y = fmaf(f, v.y, sum.y);
                sum.z = fmaf(f, v.z, sum.z); sum.w = fmaf(f, v.w, sum.w);
            }
            const int i = r / pv.G, g = r - i * pv.G;
            const float inv = sh.row_inv[r];
            T *dst = static_cast<T *>(a.out) + x.b * a.so.b + (int64_t)(x.h * pv.G + g) * a.so.h + (int64_t)i * a.so.t + d4 * 4;
            dst[0] = Elem<T>::from_float(sum.x * inv);
            dst[1] = Elem<T>::from_float(sum.y * inv);
            dst[2] = Elem<T>::from_float(sum.z * inv);
            dst[3] = Elem<T>::from_float(sum.w * inv);
        }
        named_barrier(1, kConsumers);                        // all has been read
    }
}

// ---- windowed, few units: a cluster per unit ---------------------------------------------------------
// What a unit sees is bounded, so where there are no more units than CTAs fit at once, the CTAs of a cluster share the tiles of one
// unit evenly, and it is joined through their shared memory: no partial results in the workspace, no second kernel (us, split list
// with finish kernel and clusters, bf16: 32 heads x 205 slots 7.1 and 6.0; 32 x 1,024: 10.8 and 8.2; 32 x 4,096: 18.0 and 15.8; 64 x
// 4,224 of fp16, 16 rows: 34 and 29).  The list divides what is there, a cluster has its unit's tiles whatever the others have.  So the list
// serves calls whose clusters would leave a quarter of the device idle (38 x 4,096: 19.5 and 20.7; 32 bits, 38 x 4,096: 36 and 52; 75 x
// 4,096: 62 and 98) and long parts of a unit, which one of two sequences in a batch of short ones would make all wait for (32 x 8 units,
// two sequences at 4,096 and the others below 100, parts of 64 tiles: 18.5 and 62, where 256 full units take 89 and 81; 8 x 8
// units, one sequence at 4,096, parts of 16: 13.3 and 19.6).
constexpr int kRanks = 8;                    // CTAs of a cluster at most
constexpr int kRankTiles = 8;                // tiles of a CTA at most, whatever stays idle
constexpr int kMostRankTiles = 20;           // ... with a full device

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// address of p's place in the shared memory of CTA `rank` of the cluster
__device__ __forceinline__ uint32_t remote(const void *p, int rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ float2 remote2(uint32_t at)
{
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ float4 remote4(uint32_t at)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}

template <typename T, int D, int NC>
__global__ void __launch_bounds__(32 * (warps_of<T> + 1))
paged_few_cluster_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                         const __grid_constant__ AttendArgs a, int NP, int ranks)
{
    using R = Ring<T, D>;
    using Body = typename BodyOf<T, D, NC, true>::type;
    constexpr int kTile = R::kTile, kWarps = warps_of<T>, kSlots = kTile / kWarps, kConsumers = 32 * kWarps;
    // behind the last tile the warps' results, and the CTA's, stand in the ring's place
    static_assert((size_t)R::kStages * 2 * R::kTileBytes >= (size_t)kFewRows * ((kWarps + 1) * (D * 4 + 8)), "results fit");
    extern __shared__ uint8_t smem_raw[];
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ uint64_t full[R::kStages], empty[R::kStages];
    __shared__ int abort_word;
    const PagedView &pv = a.pv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int u = blockIdx.x / ranks, rank = blockIdx.x - u * ranks;
    volatile int *abort_flag = &abort_word;
    if (threadIdx.x == 0) {
        for (int s = 0; s < R::kStages; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], kWarps); }
        abort_word = 0;
        fence_mbar_init();
        prefetch_tmap(&map_k);
        prefetch_tmap(&map_v);
    }
    dependency_wait();
    __syncthreads();
    dependents_may_start();
    Where x = {};
    x.b = u / pv.H;
    x.h = u - x.b * pv.H;
    Near near;
    const SeqState st = near_state<true>(pv, x.b, near);
    const int used = st.len > 0 ? st.past + st.len : 0, tiles = (used + kTile - 1) / kTile;
    const int t0 = tiles * rank / ranks, t1 = tiles * (rank + 1) / ranks;
    float *o = reinterpret_cast<float *>(ring), *joined = o + (size_t)kWarps * NP * D;
    float2 *ml = reinterpret_cast<float2 *>(joined + NP * D), *joined_ml = ml + kWarps * NP;

    if (warp == 0) {
        const int box = box_rows<true>(pv, kTile), boxes = kTile / box;
        const int32_t *table = pv.table + (size_t)x.b * pv.max_pages;
        const uint64_t policy = policy_evict_first();
        int it = 0, ok = 1;
        for (int t = t0; t < t1; ++t, ++it) {
            const int s = it % R::kStages;
            const int slot = t * kTile + lane * box;
            const int nbox = min(boxes, (used - t * kTile + box - 1) / box);
            int row = 0;
            if (lane < nbox) {
                const int real = real_slot<true>(pv, near, slot);
                row = (int)pool_row(pv, page_for_read(pv, table, real), x.h, real);
            }
            if (lane == 0) {
                if (it >= R::kStages) ok = mbar_wait(&empty[s], ((it / R::kStages) & 1) ^ 1, abort_flag) ? 1 : 0;
                if (ok) mbar_arrive_expect_tx(&full[s], (uint32_t)(nbox * box * R::kRowBytes * 2));
            }
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (!ok) break;
            if (lane < nbox) {
                uint8_t *dst = ring + (size_t)s * 2 * R::kTileBytes + lane * box * 128;
#pragma unroll
                for (int ch = 0; ch < R::kChunks; ++ch) {
                    tma_load_2d(dst + ch * (kTile * 128), &map_k, &full[s], ch * (128 / (int)sizeof(T)), row, policy);
                    tma_load_2d(dst + R::kTileBytes + ch * (kTile * 128), &map_v, &full[s], ch * (128 / (int)sizeof(T)), row, policy);
                }
            }
            __syncwarp();
        }
        if (lane == 0 && *abort_flag) {
            int dummy = 0;                                   // copies still in flight get a bounded chance to land
            for (int k = max(0, it - R::kStages); k < it; ++k)
                mbar_wait(&full[k % R::kStages], (k / R::kStages) & 1, &dummy);
            *pv.status = A2SF_ERR_TIMEOUT;
        }
    } else if (used > 0) {
        const int cw = warp - 1, ct = threadIdx.x - 32;
        float *scratch = reinterpret_cast<float *>(ring + (size_t)R::kStages * 2 * R::kTileBytes);
        Body body;
        body.begin(a, x, st, near, scratch);
        for (int t = t0, it = 0; t < t1; ++t, ++it) {
            const int s = it % R::kStages;
            if (!*abort_flag && !mbar_wait(&full[s], (it / R::kStages) & 1, abort_flag)) *pv.status = A2SF_ERR_TIMEOUT;
            const int j0 = t * kTile + cw * kSlots;
            uint8_t *K = ring + (size_t)s * 2 * R::kTileBytes;
            if (j0 < used && A2SF_IN_RANGE(j0, pv.max_pages << pv.ps_shift, kDbgPagedFew)) body.tile(a, K, K + R::kTileBytes, cw * kSlots, j0, used, nullptr, NP, scratch);
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[s]);
        }
        named_barrier(1, kConsumers);                        // the ring has been read
        body.end(ml + cw * NP, o + (size_t)cw * NP * D, NP);
        named_barrier(1, kConsumers);
        for (int e = ct; e < NP * (D / 4); e += kConsumers) {
            const int r = e / (D / 4), d4 = e - r * (D / 4);
            float mx = -INFINITY, l = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) mx = fmaxf(mx, ml[w * NP + r].x);
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float2 y = ml[w * NP + r];
                if (y.y == 0.f) continue;                    // a warp that saw nothing wrote no output; a NaN stays one
                const float f = ex2(y.x - mx);
                const float4 v = reinterpret_cast<const float4 *>(o + (size_t)(w * NP + r) * D)[d4];
                l = fmaf(f, y.y, l);
                sum.x = fmaf(f, v.x, sum.x); sum.y = fmaf(f, v.y, sum.y);
                sum.z = fmaf(f, v.z, sum.z); sum.w = fmaf(f, v.w, sum.w);
            }
            reinterpret_cast<float4 *>(joined + r * D)[d4] = sum;
            if (d4 == 0) joined_ml[r] = make_float2(mx, l);
        }
    }
    __syncwarp();
    cluster_sync();
    if (warp != 0) {
        const int rows = st.len * pv.G;                      // 0 where the sequence takes no part
        for (int e = rank * kConsumers + (int)threadIdx.x - 32; e < rows * (D / 4); e += ranks * kConsumers) {
            const int r = e / (D / 4), d4 = e - r * (D / 4);
            if (!A2SF_IN_RANGE(r, NP, kDbgPagedFew) || !A2SF_IN_RANGE(r / pv.G, pv.c, kDbgPagedFew) || !A2SF_IN_RANGE(x.b, pv.B, kDbgPagedFew)) continue;
            float2 y[kRanks];
            float mx = -INFINITY, l = 0.f;
#pragma unroll
            for (int k = 0; k < kRanks; ++k) {
                y[k] = k < ranks ? remote2(remote(joined_ml + r, k)) : make_float2(-INFINITY, 0.f);
                mx = fmaxf(mx, y[k].x);
            }
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < kRanks; ++k) {
                if (k >= ranks) continue;
                const float4 v = remote4(remote(joined + r * D + d4 * 4, k));
                const float f = y[k].y != 0.f ? ex2(y[k].x - mx) : 0.f;
                l = fmaf(f, y[k].y, l);
                sum.x = fmaf(f, v.x, sum.x); sum.y = fmaf(f, v.y, sum.y);
                sum.z = fmaf(f, v.z, sum.z); sum.w = fmaf(f, v.w, sum.w);
            }
            const int i = r / pv.G, g = r - i * pv.G;
            const float inv = 1.f / l;
            T *dst = static_cast<T *>(a.out) + x.b * a.so.b + (int64_t)(x.h * pv.G + g) * a.so.h + (int64_t)i * a.so.t + d4 * 4;
            dst[0] = Elem<T>::from_float(sum.x * inv);
            dst[1] = Elem<T>::from_float(sum.y * inv);
            dst[2] = Elem<T>::from_float(sum.z * inv);
            dst[3] = Elem<T>::from_float(sum.w * inv);
            if (d4 == 0 && a.lse) a.lse[((size_t)u * pv.G + g) * pv.c + i] = (mx + log2f(l)) * 0.6931471805599453f;
        }
    }
    __syncwarp();
    cluster_sync();                                          // no CTA ends while its results are read
}

// CTAs of a cluster, or 0 where the other forms serve: as many as fit at once, each with a tile at least.  What fits is counted for
// the whole chip, since the size of the workspace, which clusters do without, must not depend on a device.  A cluster stays inside one of the
// chip's parts, which leave some SMs over: of one and of two CTAs an SM 74 and 148 clusters of 2 fit, 33 and 71 of 4, 15 and 33 of 8
// (one more than fit, 32 bits, 16 x 4,096 slots: 34 us where 14 units take 18).
constexpr int clusters_fit(int slots, int ranks) { return (ranks > 2 ? slots - 5 * (ranks - 1) : slots) / ranks; }
static_assert(clusters_fit(kSms, 4) == 33 && clusters_fit(2 * kSms, 4) == 70 && clusters_fit(kSms, 8) == 14 && clusters_fit(2 * kSms, 8) == 32, "at most what fits");

template <typename T, int D, int NC> int cluster_ranks(const PagedView &pv)
{
    constexpr size_t smem = Ring<T, D>::kBytes + BodyOf<T, D, NC, true>::kScratch;
    constexpr int slots = kSms * (2 * (smem + 2 * 1024) <= 228 * 1024 ? 2 : 1);
    const long long units = (long long)pv.B * pv.H;
    const int tiles = (near_capacity(pv, true, pv.c) + Ring<T, D>::kTile - 1) / Ring<T, D>::kTile;
    if (units > slots) return 0;
    int ranks = 1;
    while (ranks < kRanks && units <= clusters_fit(slots, 2 * ranks) && 2 * ranks <= tiles) ranks *= 2;
    const int most = 4 * units * ranks < 3 * slots ? kRankTiles : kMostRankTiles;
    return (tiles + ranks - 1) / ranks > most ? 0 : ranks;
}

// The finish kernel: `blocks` blocks per unit.  Block y joins the output rows y, y + blocks, .. and brings the
// scores of slots y * chunk .. up to date.  All of it is latency: dependent loads around a few bytes.  So the page
// numbers and old scores of the first slots are read while the main kernel still drains, the logits and the
// partial maxima and sums are requested together, and a thread has several slots in flight.

constexpr int finish_ctas(int NP) { return NP <= 2 ? 5 : 4; }     // of an SM: one round of blocks covers a call, where it can
constexpr int kMlCache = 2048;            // partial (maximum, sum) pairs that fit in shared memory

template <int NP> struct SlotBatch {
    static constexpr int kScoreSlots = NP >= 8 ? 2 : 4;
    int32_t row[kScoreSlots];                 // of the pool, or -1
    float old[kScoreSlots], x[kScoreSlots][NP];

    __device__ void addresses(const PagedView &pv, const int32_t *table, int h, int jb, int j1)
    {
#pragma unroll
        for (int e = 0; e < kScoreSlots; ++e) {
            const int j = jb + e * kFinishThreads;
            row[e] = j < j1 ? page_for_write(pv, table, j) : -1;
        }
#pragma unroll
        for (int e = 0; e < kScoreSlots; ++e) {
            if (row[e] < 0) continue;
            row[e] = (int32_t)pool_row(pv, row[e], h, jb + e * kFinishThreads);
            old[e] = pv.scores[row[e]];
        }
    }
    __device__ void logits(const float *src, int jb)
    {
#pragma unroll
        for (int e = 0; e < kScoreSlots; ++e) {
            if (row[e] < 0) continue;
            const float *s = src + (size_t)(jb + e * kFinishThreads) * NP;
            if constexpr (NP == 1) x[e][0] = s[0];
            else if constexpr (NP == 2) {
                const float2 v = *reinterpret_cast<const float2 *>(s);
                x[e][0] = v.x; x[e][1] = v.y;
            } else {
#pragma unroll
                for (int r = 0; r < NP; r += 4) {
                    const float4 v = *reinterpret_cast<const float4 *>(s + r);
                    x[e][r] = v.x; x[e][r + 1] = v.y; x[e][r + 2] = v.z; x[e][r + 3] = v.w;
                }
            }
        }
    }
    __device__ void store(float *scores, const float *row_c, float decay)
    {
#pragma unroll
        for (int e = 0; e < kScoreSlots; ++e) {
            if (row[e] < 0) continue;
            float gain = 0.f;              // rows that do not see the slot, or are none, have -inf there
#pragma unroll
            for (int r = 0; r < NP; ++r) gain += ex2(x[e][r] - row_c[r]);
            scores[row[e]] = fmaf(old[e], decay, gain);
        }
    }
};

template <typename T, int D, int NP>
__global__ void __launch_bounds__(kFinishThreads, NP <= 2 ? 5 : 4)
paged_few_finish_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ FewWs ws, int ctas, int blocks, int chunk)
{
    constexpr int kWarps = warps_of<T>;
    constexpr int GR = kFinishThreads / (D / 4);             // thread groups of an output row, 4 elements a thread
    __shared__ float4 red[kFinishThreads];
    __shared__ float row_m[kFewRows], row_l[kFewRows], row_c[kFewRows];
    __shared__ float2 ml_cache[kMlCache];
    const PagedView &pv = a.pv;
    const int tid = threadIdx.x;
    const int u = blockIdx.x / blocks, y = blockIdx.x - u * blocks, b = u / pv.H, h = u - b * pv.H;
    const SeqState st = seq_state(pv, b);
    const int rows = st.len * pv.G, used = st.past + st.len;
    const int j0 = y * chunk, j1 = a.scores ? min(used, j0 + chunk) : 0;
    const int32_t *table = pv.table + (size_t)b * pv.max_pages;
    SlotBatch<NP> batch;
    const bool working = rows > 0 && (y < rows || j0 < j1);
    if (working) batch.addresses(pv, table, h, j0 + tid, j1);
    dependency_wait();
    if (!working || !A2SF_IN_RANGE(u, pv.B * pv.H, kDbgPagedFew)) return;
    const float *logits = ws.logits + (size_t)u * ws.slots * NP;
    batch.logits(logits, j0 + tid);
    // the CTAs of the main kernel that had a part of this unit
    const long long total = (long long)pv.H * ws.prefix[pv.B], share = (total + ctas - 1) / ctas;
    const int tiles = ws.prefix[b + 1] - ws.prefix[b];
    const long long u0 = (long long)pv.H * ws.prefix[b] + (long long)h * tiles;
    const int k0 = (int)(u0 / share), k1 = (int)((u0 + tiles - 1) / share);
    const size_t seg0 = ((size_t)k0 + u) * kWarps;
    const int parts = (k1 - k0 + 1) * kWarps;
    if (!A2SF_IN_RANGE(seg0 + parts - 1, ws.segs, kDbgPagedFew)) return;
    // (maximum, sum) of part p and row r at ml[r * row_step + p * part_step]
    const float2 *ml = ws.ml + seg0 * NP;
    int row_step = 1, part_step = NP;
    if (parts * NP <= kMlCache) {
        for (int x = tid; x < parts * NP; x += kFinishThreads) ml_cache[x % NP * parts + x / NP] = ml[x];
        ml = ml_cache;
        row_step = parts; part_step = 1;
        __syncthreads();
    }
    // a row's maximum, sum, and its constant for the scores: log-sum-exp and the weight's exponent (log2 units)
    constexpr int LR = NP <= 8 ? 32 : 16;                    // lanes per row: all rows at once
    if (tid < NP * LR) {
        const int r = tid / LR, l0 = tid % LR;
        const float2 *row = ml + r * row_step;
        float mx = -INFINITY, l = 0.f;
        for (int p = l0; p < parts; p += LR) mx = fmaxf(mx, row[p * part_step].x);
#pragma unroll
        for (int o = LR / 2; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        for (int p = l0; p < parts; p += LR) {
            const float2 x = row[p * part_step];
            l += x.y != 0.f ? ex2(x.x - mx) * x.y : 0.f;     // as in the whole-unit kernel
        }
#pragma unroll
        for (int o = LR / 2; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        if (l0 == 0) {
            row_m[r] = mx;
            row_l[r] = l;
            row_c[r] = r < rows ? mx + log2f(l) + age_exponent(st.len - 1 - r / pv.G, a.nl2a) : INFINITY;
        }
    }
    __syncthreads();
    const float decay = exp2f(-age_exponent(st.len, a.nl2a));
    batch.store(pv.scores, row_c, decay);
    for (int jb = j0 + SlotBatch<NP>::kScoreSlots * kFinishThreads; jb < j1; jb += SlotBatch<NP>::kScoreSlots * kFinishThreads) {
        batch.addresses(pv, table, h, jb + tid, j1);
        batch.logits(logits, jb + tid);
        batch.store(pv.scores, row_c, decay);
    }
    for (int r = y; r < rows; r += blocks) {
        // thread groups take every GR-th partial result; joined in a fixed order
        const int d4 = tid % (D / 4), grp = tid / (D / 4);
        const float4 *op = reinterpret_cast<const float4 *>(ws.o + (seg0 * NP + r) * D) + d4;
        const float2 *row = ml + r * row_step;
        const float mx = row_m[r];
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int p = grp; p < parts; p += GR) {
            const float f = ex2(row[p * part_step].x - mx);
            const float4 v = f > 0.f ? op[(size_t)p * (NP * D / 4)] : make_float4(0.f, 0.f, 0.f, 0.f);
            o.x = fmaf(f, v.x, o.x); o.y = fmaf(f, v.y, o.y); o.z = fmaf(f, v.z, o.z); o.w = fmaf(f, v.w, o.w);
        }
        __syncthreads();
        red[tid] = o;
        __syncthreads();
        if (grp == 0) {
#pragma unroll
            for (int x = 1; x < GR; ++x) {
                const float4 v = red[x * (D / 4) + d4];
                o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
            }
            const int i = r / pv.G, g = r - i * pv.G;
            const float l = row_l[r], inv = 1.f / l;
            T *dst = static_cast<T *>(a.out) + b * a.so.b + (int64_t)(h * pv.G + g) * a.so.h + (int64_t)i * a.so.t + d4 * 4;
            dst[0] = Elem<T>::from_float(o.x * inv);
            dst[1] = Elem<T>::from_float(o.y * inv);
            dst[2] = Elem<T>::from_float(o.z * inv);
            dst[3] = Elem<T>::from_float(o.w * inv);
            if (d4 == 0 && a.lse)
                a.lse[((size_t)u * pv.G + g) * pv.c + i] = (mx + log2f(l)) * 0.6931471805599453f;
        }
    }
}

size_t pad(size_t x) { return (x + 255) / 256 * 256; }
int padded_slots(const PagedView &pv, bool windowed) { return (near_capacity(pv, windowed, pv.c) + 127) / 128 * 128; }       // of either tile

FewWs carve(int dtype, const PagedView &pv, bool windowed, void *ws, size_t *bytes)
{
    const size_t U = (size_t)pv.B * pv.H, NP = rows_padded(pv.c * pv.G);
    // the size must not depend on a device: room for any SM count up to 256
    const size_t segs = (U + 512) * (dtype == A2SF_F32 ? warps_of<float> : warps_of<__half>);
    FewWs w;
    size_t off = 0;
    char *base = static_cast<char *>(ws);
    w.slots = padded_slots(pv, windowed);
    w.segs = (int)segs;
    w.logits = reinterpret_cast<float *>(base + off); off += windowed ? 0 : pad(U * w.slots * NP * 4);
    w.ml = reinterpret_cast<float2 *>(base + off); off += pad(segs * NP * 8);
    w.o = reinterpret_cast<float *>(base + off); off += pad(segs * NP * pv.d * 4);
    w.prefix = reinterpret_cast<int32_t *>(base + off); off += pad(((size_t)pv.B + 1) * 4);
    if (bytes) *bytes = off;
    return w;
}

// Shared memory of the whole-unit kernel, or 0 where it does not serve: longer caches, or more rows than fit.
template <typename T, int D, int NC, bool Win> size_t whole_smem(const PagedView &pv)
{
    using R = Ring<T, D>;
    const int slots = (near_capacity(pv, Win, pv.c) + R::kTile - 1) / R::kTile * R::kTile;
    const size_t smem = R::kBytes + BodyOf<T, D, NC, Win>::kScratch + whole_bytes(warps_of<T>, D, rows_padded(pv.c * pv.G), Win ? 0 : slots);
    const int most = pv.B * pv.H >= kSms ? kWholeTilesMany : kWholeTiles;
    return slots <= most * R::kTile && smem + sizeof(WholeShared) <= 227 * 1024 ? smem : 0;
}

template <typename T, int D, int NC, bool Win>
cudaError_t launch_nc(int dtype, const AttendArgs &a, cudaStream_t s)
{
    using R = Ring<T, D>;
    constexpr size_t smem = R::kBytes + BodyOf<T, D, NC, Win>::kScratch;
    cudaError_t e = allow_dynamic_smem<paged_few_kernel<T, D, NC, Win>>(smem);
    if (e != cudaSuccess) return e;
    CUtensorMap mk, mv;
    const int row = Win ? kGrain : a.pv.ps, box = row < R::kTile ? row : R::kTile;
    if (!make_pool_map(&mk, dtype, a.pv.k, a.pv, box) || !make_pool_map(&mv, dtype, a.pv.v, a.pv, box)) return cudaErrorInvalidValue;
    const int NP = rows_padded(a.pv.c * a.pv.G);
    if constexpr (Win) {
        if (const int ranks = cluster_ranks<T, D, NC>(a.pv)) {
            if ((e = allow_dynamic_smem<paged_few_cluster_kernel<T, D, NC>>(smem)) != cudaSuccess) return e;
            e = launch_clusters(paged_few_cluster_kernel<T, D, NC>, (unsigned)(a.pv.B * a.pv.H * ranks), ranks, 32 * (warps_of<T> + 1), smem, s, mk, mv, a, NP, ranks);
            if (e == cudaSuccess) count_launch();
            return e;
        }
    }
    if (const size_t whole = whole_smem<T, D, NC, Win>(a.pv)) {
        if ((e = allow_dynamic_smem<paged_few_whole_kernel<T, D, NC, Win>>(whole)) != cudaSuccess) return e;
        const long long resident = device_sm_count() * (2 * (whole + sizeof(WholeShared) + 1024) <= 228 * 1024 ? 2 : 1), units = (long long)a.pv.B * a.pv.H;
        const int slots = (near_capacity(a.pv, Win, a.pv.c) + R::kTile - 1) / R::kTile * R::kTile;
        e = launch_chained(paged_few_whole_kernel<T, D, NC, Win>, (unsigned)(units < resident ? units : resident), 32 * (warps_of<T> + 1), whole, s, mk, mv, a, NP, slots);
        if (e == cudaSuccess) count_launch();
        return e;
    }
    const FewWs ws = carve(dtype, a.pv, Win, a.ws, nullptr);
    const int ctas = device_sm_count() * (2 * (smem + sizeof(FewShared) + 1024) <= 228 * 1024 ? 2 : 1);   // what is resident
    if (ctas < 1 || ctas > 512) return cudaErrorInvalidValue;
    if ((e = launch_chained(paged_few_kernel<T, D, NC, Win>, ctas, 32 * (warps_of<T> + 1), smem, s, mk, mv, a, ws, NP)) != cudaSuccess) return e;
    count_launch();
    // blocks per unit: enough for the rows and the slots, as far as that fills the device
    const int cap = Win ? 1 : a.pv.max_pages << a.pv.ps_shift;
    const long long units = (long long)a.pv.B * a.pv.H;
    const long long want = (long long)finish_ctas(NP) * device_sm_count() / units;
    int blocks = (cap + kFinishThreads - 1) / kFinishThreads;
    if (blocks < a.pv.c * a.pv.G) blocks = a.pv.c * a.pv.G;
    if (blocks > want) blocks = want > 0 ? (int)want : 1;
    const int chunk = ((cap + blocks - 1) / blocks + 31) / 32 * 32;
    const long long grid = units * blocks;
    if (grid > 0x7fffffffll) return cudaErrorInvalidValue;
    auto finish = [&](auto kernel) { return launch_chained(kernel, (unsigned)grid, kFinishThreads, 0, s, a, ws, ctas, blocks, chunk); };
    switch (NP) {
    case 1: e = finish(paged_few_finish_kernel<T, D, 1>); break;
    case 2: e = finish(paged_few_finish_kernel<T, D, 2>); break;
    case 4: e = finish(paged_few_finish_kernel<T, D, 4>); break;
    case 8: e = finish(paged_few_finish_kernel<T, D, 8>); break;
    default: e = finish(paged_few_finish_kernel<T, D, 16>); break;
    }
    if (e == cudaSuccess) count_launch();
    return e;
}

// The kernels' types, head size and rows for a call, as a value that a generic function takes apart.
template <typename T, int D, int NC> struct Form {};

template <typename T, int D, typename F> auto with_rows(int rows, F f)
{
    if constexpr (sizeof(T) == 4) {
        switch (rows_padded(rows)) {
        case 1: return f(Form<T, D, 1>());
        case 2: return f(Form<T, D, 2>());
        case 4: return f(Form<T, D, 4>());
        case 8: return f(Form<T, D, 8>());
        default: return f(Form<T, D, 16>());
        }
    } else {
        return rows <= 4 ? f(Form<T, D, 4>()) : rows <= 8 ? f(Form<T, D, 8>()) : f(Form<T, D, 16>());
    }
}
template <typename F> auto with_form(int dtype, const PagedView &pv, F f)
{
    const int rows = pv.c * pv.G;
    const bool wide = pv.d == 128;
    switch (dtype) {
    case A2SF_F32: return wide ? with_rows<float, 128>(rows, f) : with_rows<float, 64>(rows, f);
    case A2SF_BF16: return wide ? with_rows<__nv_bfloat16, 128>(rows, f) : with_rows<__nv_bfloat16, 64>(rows, f);
    default: return wide ? with_rows<__half, 128>(rows, f) : with_rows<__half, 64>(rows, f);
    }
}

template <bool Win, typename T, int D, int NC> cudaError_t launch(Form<T, D, NC>, int dtype, const AttendArgs &a, cudaStream_t s)
{
    if constexpr (Win && sizeof(T) == 4 && NC == kFewRows) return cudaErrorInvalidValue;      // mma.sync has these
    else return launch_nc<T, D, NC, Win>(dtype, a, s);
}
template <typename T, int D, int NC> int ranks_of(Form<T, D, NC>, const PagedView &pv) { return cluster_ranks<T, D, NC>(pv); }

}  // namespace

size_t attend_few_ws_bytes(int dtype, const PagedView &pv, bool windowed)
{
    if (windowed && with_form(dtype, pv, [&](auto form) { return ranks_of(form, pv); }) > 0) return 0;
    size_t bytes = 0;
    carve(dtype, pv, windowed, nullptr, &bytes);
    return bytes;
}

cudaError_t launch_attend_few(int dtype, const AttendArgs &a, cudaStream_t s)
{
    return with_form(dtype, a.pv, [&](auto form) { return a.windowed ? launch<true>(form, dtype, a, s) : launch<false>(form, dtype, a, s); });
}

}  // namespace a2sf
