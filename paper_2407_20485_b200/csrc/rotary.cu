// Rotary positions, alone and on the way into a paged cache.
//
//   y1 = m (x1 cos - x2 sin),  y2 = m (x2 cos + x1 sin),  angle = position * f_k
//
// The angle is held in turns as a 64-bit fixed-point fraction: position * turn[k] modulo 2^64 drops
// whole turns exactly, so a far position costs no accuracy and no reduction.  Of its top 32 bits the
// quarter turns are taken off; an eighth of a turn at most is rounded to fp32 (off by 2^-28 turns, 2.4e-8
// of an angle) and goes to sincospif.
//
// Bound by memory: every element is read and written once.  A thread owns W neighbouring elements
// (two groups of W, in the split layout) of one token and walks over the heads, so the sines and
// cosines -- about 30 instructions each, more than the memory time of a single head would hide --
// are computed once per token and not once per head, and no table of them is read.  kHeads heads are
// in flight at a time.  In append the same walk takes the keys into their pages, and the values.
//
// With several axes (kAxes) pair k turns by the position on its own axis, positions[axis[k]][b][t]; all else is the same.
#include <type_traits>

#include "paged.cuh"

namespace a2sf {

A2SF_DEBUG_TRANSLATION_UNIT(rotary)

static __device__ int g_paged_status = 0;

namespace {

constexpr int kRotThreads = 256;
constexpr int kHeads = 2;        // heads in flight per thread: with four blocks an SM, 64 KB on the way (neighbouring pairs: 32)

// W consecutive elements of 16- or 32-bit storage, moved as one access of up to 16 bytes
template <typename T, int W> struct alignas(sizeof(T) * W) Pack { T e[W]; };

template <typename P> __device__ __forceinline__ void store_pack(void *dst, const P &v)
{
    if constexpr (sizeof(P) == 16) __stcs(reinterpret_cast<uint4 *>(dst), *reinterpret_cast<const uint4 *>(&v));
    else                           *reinterpret_cast<P *>(dst) = v;
}

template <bool kAxes> struct PlanArg {
    unsigned long long turn[A2SF_ROTARY_MAX_PAIRS];
};
template <> struct PlanArg<true> {
    unsigned long long turn[A2SF_ROTARY_MAX_PAIRS];
    uint8_t axis[A2SF_ROTARY_MAX_PAIRS];
};
template <bool kAxes> using PlanOf = std::conditional_t<kAxes, a2sf_rotary_axes_plan, a2sf_rotary_plan>;

// One thread item of a row: W elements at `a`, and in the split layout W more at `b`.
// Items 0 .. rot_items-1 rotate, the following ones copy W elements each.
template <typename T, int W, bool Interleaved, bool Append, bool kAxes>
__global__ void __launch_bounds__(kRotThreads, 4)
rotary_kernel(const __grid_constant__ PlanArg<kAxes> plan, const __grid_constant__ RotaryArgs r,
              const __grid_constant__ PagedView pv, int r_dim, float magnitude, int rot_items, int items,
              int heads_per_block, int splits)
{
    constexpr int NP = Interleaved ? (W + 1) / 2 : W;        // pairs of an item
    using P = Pack<T, W>;
    dependency_wait();
    dependents_may_start();
    const int split = blockIdx.x % splits;
    const long long idx = (long long)(blockIdx.x / splits) * kRotThreads + threadIdx.x;
    const long long tok = idx / items;
    const int item = (int)(idx - tok * items);
    if (tok >= (long long)r.B * r.n) return;
    const int b = (int)(tok / r.n), t = (int)(tok - (long long)b * r.n);

    int len, slot = 0, base;
    if (Append) {
        const SeqState st = seq_state(pv, b);
        len = st.len;
        slot = st.past + t;
        base = r.start ? r.start[b] : st.past;
    } else {
        len = r.lens ? r.lens[b] : r.n;
        base = r.start ? r.start[b] : 0;
    }
    if (t >= len) return;
    const int pos = (!Append && !kAxes && r.positions) ? r.positions[(size_t)b * r.n + t] : base + t;

    const bool rotates = item < rot_items;
    const int a_off = rotates ? item * W : r_dim + (item - rot_items) * W;
    const int b_off = item * W + r_dim / 2;                 // split layout only
    if (!A2SF_IN_RANGE(a_off + W - 1, r.d, kDbgRotary) || (!Interleaved && rotates && !A2SF_IN_RANGE(b_off + W - 1, r.d, kDbgRotary))) return;
    float cs[NP], sn[NP];
    if (rotates) {
#pragma unroll
        for (int e = 0; e < NP; ++e) {
            const int k = Interleaved ? item * NP + e : item * W + e;
            if (!A2SF_IN_RANGE(k, A2SF_ROTARY_MAX_PAIRS, kDbgRotary)) return;
            int at = pos;
            if constexpr (kAxes) at = r.positions[((size_t)plan.axis[k] * r.B + b) * r.n + t];
            const unsigned long long turn = plan.turn[k] * (unsigned long long)(long long)at;
            // the nearest quarter turn is in the top two bits of `near`; an eighth of a turn is left either way (half turns: [-1/4, 1/4])
            const unsigned top = (unsigned)(turn >> 32), near = top + 0x20000000u;
            float s0, c0;
            sincospif((float)(int)(top - (near & 0xc0000000u)) * (1.f / 2147483648.f), &s0, &c0);
            const bool odd = near & 0x40000000u;
            sn[e] = __uint_as_float(__float_as_uint(odd ? c0 : s0) ^ (near & 0x80000000u)) * (r.transpose ? -magnitude : magnitude);
            cs[e] = __uint_as_float(__float_as_uint(odd ? s0 : c0) ^ ((near + 0x40000000u) & 0x80000000u)) * magnitude;
        }
    }

    int64_t page_row = -1;                                   // pool row of (head 0, this slot)
    if (Append) {
        const int page = page_for_write(pv, pv.table + (size_t)b * pv.max_pages, slot);
        if (page >= 0) page_row = pool_row(pv, page, 0, slot);
    }
    const int total = r.Hq + (Append ? 2 * r.Hk : 0);
    const int h0 = split * heads_per_block, h1 = min(total, h0 + heads_per_block);

    for (int hb = h0; hb < h1; hb += kHeads) {
        const T *src[kHeads];
        T *dst[kHeads];
        bool turn_it[kHeads];
#pragma unroll
        for (int x = 0; x < kHeads; ++x) {
            const int h = hb + x;
            src[x] = nullptr; dst[x] = nullptr; turn_it[x] = rotates;
            if (h >= h1) continue;
            if (h < r.Hq) {
                src[x] = static_cast<const T *>(r.x) + b * r.sx.b + h * r.sx.h + (int64_t)t * r.sx.t;
                dst[x] = static_cast<T *>(r.y) + b * r.sy.b + h * r.sy.h + (int64_t)t * r.sy.t;
            } else if (Append && page_row >= 0) {
                const bool val = h >= r.Hq + r.Hk;
                const int hk = h - r.Hq - (val ? r.Hk : 0);
                const int64_t row = page_row + ((int64_t)hk << pv.ps_shift);
                src[x] = static_cast<const T *>(val ? r.v : r.k) + b * r.skv.b + hk * r.skv.h + (int64_t)t * r.skv.t;
                dst[x] = reinterpret_cast<T *>(val ? pv.v : pv.k) + row * r.d;
                if (val) turn_it[x] = false;
                else if (item == 0) {
                    pv.positions[row] = pos;
                    pv.scores[row] = 0.f;
                }
            }
        }
        P va[kHeads], vb[kHeads];
#pragma unroll
        for (int x = 0; x < kHeads; ++x) {
            if (!src[x]) continue;
            va[x] = *reinterpret_cast<const P *>(src[x] + a_off);
            if (!Interleaved && rotates) vb[x] = *reinterpret_cast<const P *>(src[x] + b_off);
        }
#pragma unroll
        for (int x = 0; x < kHeads; ++x) {
            if (!src[x]) continue;
            if (turn_it[x]) {
#pragma unroll
                for (int e = 0; e < NP; ++e) {
                    const float x1 = Elem<T>::to_float(Interleaved ? va[x].e[(2 * e) % W] : va[x].e[e]);
                    const float x2 = Elem<T>::to_float(Interleaved ? va[x].e[(2 * e + 1) % W] : vb[x].e[e]);
                    const T y1 = Elem<T>::from_float(x1 * cs[e] - x2 * sn[e]);
                    const T y2 = Elem<T>::from_float(x2 * cs[e] + x1 * sn[e]);
                    if (Interleaved) { va[x].e[(2 * e) % W] = y1; va[x].e[(2 * e + 1) % W] = y2; }
                    else             { va[x].e[e] = y1; vb[x].e[e] = y2; }
                }
            }
            store_pack(dst[x] + a_off, va[x]);
            if (!Interleaved && rotates) store_pack(dst[x] + b_off, vb[x]);
        }
    }
}

template <typename T, int W, bool Interleaved, bool Append, bool kAxes>
cudaError_t launch_w(const PlanOf<kAxes> *plan, const RotaryArgs &r, const PagedView &pv, cudaStream_t s)
{
    const int r_dim = plan ? plan->rotary_dim : 0;
    // in place, elements beyond the rotated ones are already where they belong -- unless keys and
    // values travel into pages in the same walk
    const bool copies = Append || r.x != r.y;
    const int rot_items = Interleaved ? r_dim / W : r_dim / 2 / W;
    const int items = rot_items + (copies ? (r.d - r_dim) / W : 0);
    PlanArg<kAxes> pa;
    for (int k = 0; k < A2SF_ROTARY_MAX_PAIRS; ++k) {
        pa.turn[k] = plan ? plan->turn[k] : 0;
        if constexpr (kAxes) pa.axis[k] = plan->axis[k];
    }
    const long long threads = (long long)r.B * r.n * items;
    const long long gx = (threads + kRotThreads - 1) / kRotThreads;
    if (gx > 0x7fffffffll) return cudaErrorInvalidValue;
    // The heads are split over blocks as far as it takes to fill the device twice (8 ragged prompts of up to 2047 tokens: 22.2 us,
    // once 26.7, four times 22.7), but where once is enough for four heads a block, no further: a second, partial round costs more
    // than longer blocks do (4 x 300 tokens, 48 heads: 8.6 against 10.0 us).
    const int total = r.Hq + (Append ? 2 * r.Hk : 0);
    const long long once = 4ll * device_sm_count();
    long long gy = once / gx;
    if (gy * 4 < total) gy = (2 * once + gx - 1) / gx;
    const int hpb = (int)(((total + gy - 1) / gy + kHeads - 1) / kHeads) * kHeads;
    const int splits = (total + hpb - 1) / hpb;
    if (gx * splits > 0x7fffffffll) return cudaErrorInvalidValue;
    const cudaError_t e = launch_chained(rotary_kernel<T, W, Interleaved, Append, kAxes>, (unsigned)(gx * splits), kRotThreads, 0, s, pa, r, pv, r_dim,
                                         plan ? plan->magnitude : 1.f, rot_items, items, hpb, splits);
    if (e == cudaSuccess) count_launch();
    return e;
}

template <typename T, bool Append, bool kAxes>
cudaError_t launch_t(const PlanOf<kAxes> *plan, const RotaryArgs &r, const PagedView &pv, cudaStream_t s)
{
    // the widest access that divides the rotated part: the whole 16 bytes for the usual sizes
    const bool il = plan && plan->interleaved;
    const int part = plan ? (il ? plan->rotary_dim : plan->rotary_dim / 2) : r.d;
    constexpr int VEC = Elem<T>::kVec;
    if (il) {
        if (part % VEC == 0) return launch_w<T, VEC, true, Append, kAxes>(plan, r, pv, s);
        if (part % 4 == 0) return launch_w<T, 4, true, Append, kAxes>(plan, r, pv, s);
        return launch_w<T, 2, true, Append, kAxes>(plan, r, pv, s);
    }
    if (part % VEC == 0) return launch_w<T, VEC, false, Append, kAxes>(plan, r, pv, s);
    if (part % 4 == 0) return launch_w<T, 4, false, Append, kAxes>(plan, r, pv, s);
    if (part % 2 == 0) return launch_w<T, 2, false, Append, kAxes>(plan, r, pv, s);
    return launch_w<T, 1, false, Append, kAxes>(plan, r, pv, s);
}

template <bool kAxes>
cudaError_t launch(int dtype, const PlanOf<kAxes> *plan, const RotaryArgs &r, const PagedView *pages, cudaStream_t s)
{
    PagedView none = {};
    const PagedView &pv = pages ? *pages : none;
    switch (dtype) {
    case A2SF_F32: return pages ? launch_t<float, true, kAxes>(plan, r, pv, s) : launch_t<float, false, kAxes>(plan, r, pv, s);
    case A2SF_BF16:
        return pages ? launch_t<__nv_bfloat16, true, kAxes>(plan, r, pv, s) : launch_t<__nv_bfloat16, false, kAxes>(plan, r, pv, s);
    default: return pages ? launch_t<__half, true, kAxes>(plan, r, pv, s) : launch_t<__half, false, kAxes>(plan, r, pv, s);
    }
}

}  // namespace

cudaError_t launch_rotary(int dtype, const a2sf_rotary_plan *plan, const RotaryArgs &r, const PagedView *pages, cudaStream_t s)
{
    return launch<false>(dtype, plan, r, pages, s);
}

cudaError_t launch_rotary_axes(int dtype, const a2sf_rotary_axes_plan *plan, const RotaryArgs &r, const PagedView *pages, cudaStream_t s)
{
    return launch<true>(dtype, plan, r, pages, s);
}

int *paged_status_word()
{
    static std::once_flag once[kMaxDevices];
    static int *ptr[kMaxDevices] = {};
    const int dev = current_device_index();
    std::call_once(once[dev], [dev] {
        void *p = nullptr;
        if (cudaGetSymbolAddress(&p, g_paged_status) == cudaSuccess) ptr[dev] = static_cast<int *>(p);
    });
    return ptr[dev];
}

int read_and_clear_paged_status(cudaStream_t s)
{
    int v = 0, zero = 0;
    if (cudaMemcpyFromSymbolAsync(&v, g_paged_status, sizeof(int), 0, cudaMemcpyDeviceToHost, s) != cudaSuccess)
        return A2SF_ERR_CUDA;
    if (cudaStreamSynchronize(s) != cudaSuccess) return A2SF_ERR_CUDA;
    if (v != 0 &&
        cudaMemcpyToSymbolAsync(g_paged_status, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, s) != cudaSuccess)
        return A2SF_ERR_CUDA;
    return v;
}

}  // namespace a2sf
