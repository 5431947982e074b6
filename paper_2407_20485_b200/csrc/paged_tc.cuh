// What the tcgen05 kernels of attention over the paged cache share: packed fp32 arithmetic, tiles of 128 rows in shared memory, and
// their copies from pages and queries.
#pragma once

#include "paged.cuh"
#include "tc_sm100.cuh"

namespace a2sf {
namespace paged_tc {

using namespace tc;

constexpr int kBlk = 128;                    // rows per tile = TMEM lanes; key slots per tile

__device__ __forceinline__ float ex2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two fp32 operations per instruction (packed arithmetic on register pairs).
__device__ __forceinline__ uint64_t pack_f32x2(uint32_t lo, uint32_t hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
    return r;
}
__device__ __forceinline__ void unpack_f32x2(uint64_t v, float &lo, float &hi)
{
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add_f32x2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b)
{
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// Four lanes hold four 16-byte pieces of a row each; afterwards lane i holds piece i of all four rows, so that a
// store instruction covers 64 consecutive bytes of 8 rows and not 16 bytes of 32.
__device__ __forceinline__ void transpose4(uint4 (&p)[4])
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int step = 1; step <= 2; step <<= 1) {
        const bool up = lane & step;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            if (x & step) continue;
            const int y = x | step;                         // keep x (lower lane) or y (upper lane), exchange the other
            uint4 send = up ? p[x] : p[y], got;
            got.x = __shfl_xor_sync(0xffffffffu, send.x, step);
            got.y = __shfl_xor_sync(0xffffffffu, send.y, step);
            got.z = __shfl_xor_sync(0xffffffffu, send.z, step);
            got.w = __shfl_xor_sync(0xffffffffu, send.w, step);
            if (up) p[x] = got;
            else    p[y] = got;
        }
    }
}

template <int D> struct Tile {
    static constexpr int kHalves = D / 64;                  // 64-element swizzled columns
    static constexpr int kHalfBytes = kBlk * 128;
    static constexpr int kBytes = kHalves * kHalfBytes;
};

__device__ __forceinline__ uint64_t kmajor_desc(uint32_t smem_addr) { return make_sdesc_sw128(smem_addr, 16, 1024); }

// S = A B^T over D elements: step k starts (k / 4) halves + (k % 4) * 32 bytes into the tiles
template <int D>
__device__ __forceinline__ void issue_qk(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc)
{
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
        const uint64_t off = (uint64_t)(((k >> 2) * Tile<D>::kHalfBytes + (k & 3) * 32) >> 4);
        umma_ss(d_tmem, a_desc + off, b_desc + off, idesc, k > 0);
    }
}

// Boxes of key tile t that hold tokens, and one lane's share of the copy (lane i: box i).
struct PageTile {
    int box, boxes;
};
template <bool Win = false> __device__ __forceinline__ PageTile page_tile(const PagedView &pv, int t, int used)
{
    PageTile p;
    p.box = box_rows<Win>(pv, kBlk);
    p.boxes = min(kBlk / p.box, (used - t * kBlk + p.box - 1) / p.box);
    return p;
}
template <int D>
__device__ __forceinline__ void copy_page_tile(uint8_t *dst, const CUtensorMap *map, uint64_t *bar, const PageTile &p, int row)
{
    const int lane = threadIdx.x & 31;
    if (lane < p.boxes)
#pragma unroll
        for (int x = 0; x < Tile<D>::kHalves; ++x) tma_load_2d(dst + x * Tile<D>::kHalfBytes + lane * p.box * 128, map, bar, x * 64, row);
}
template <int D>
__device__ __forceinline__ void copy_query_tile(uint8_t *dst, const CUtensorMap *map, uint64_t *bar, int head, int token, int b)
{
#pragma unroll
    for (int x = 0; x < Tile<D>::kHalves; ++x) tma_load_4d(dst + x * Tile<D>::kHalfBytes, map, bar, x * 64, head, token, b);
}

}  // namespace paged_tc
}  // namespace a2sf
