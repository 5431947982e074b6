// Host side of the paged-cache and rotary entry points: argument validation, workspaces, dispatch.
// No data is touched on the host.
#include <cfloat>
#include <cmath>
#include <mutex>

#include "paged.cuh"

namespace a2sf {
namespace {

constexpr int32_t kPlanCheck = 0x52504c4e, kAxesPlanCheck = 0x52415850;

inline size_t align_up(size_t x, size_t a = 256) { return (x + a - 1) / a * a; }
inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline int elem_bytes(int dtype) { return dtype == A2SF_F32 ? 4 : 2; }

int check_shape(int dtype, int d)
{
    if (dtype != A2SF_F32 && dtype != A2SF_BF16 && dtype != A2SF_F16) return A2SF_ERR_UNSUPPORTED;
    return d == 64 || d == 128 ? A2SF_OK : A2SF_ERR_UNSUPPORTED;
}

// a [B][H][n][d] tensor: rows of d elements, 16-byte aligned; axes of extent 1 may have any stride
int check_tensor(const void *p, int dtype, int d, const int64_t extent[3], const int64_t stride[3])
{
    if (!p || !aligned(p, 16)) return A2SF_ERR_INVALID_ARG;
    const int vec = 16 / elem_bytes(dtype);
    for (int x = 0; x < 3; ++x) {
        if (extent[x] <= 1) continue;
        if (stride[x] < d || stride[x] % vec) return A2SF_ERR_INVALID_ARG;
    }
    return A2SF_OK;
}

int check_plan(const a2sf_rotary_plan *p, int d)
{
    if (!p || p->check != kPlanCheck || p->rotary_dim < 2 || p->rotary_dim > 2 * A2SF_ROTARY_MAX_PAIRS || p->rotary_dim % 2)
        return A2SF_ERR_INVALID_ARG;
    return p->rotary_dim <= d ? A2SF_OK : A2SF_ERR_INVALID_ARG;
}

int check_axes_plan(const a2sf_rotary_axes_plan *p, int d)
{
    if (!p || p->check != kAxesPlanCheck || p->rotary_dim < 2 || p->rotary_dim > 2 * A2SF_ROTARY_MAX_PAIRS || p->rotary_dim % 2 ||
        p->axes < 1 || p->axes > A2SF_ROTARY_MAX_AXES)
        return A2SF_ERR_INVALID_ARG;
    for (int k = 0; k < p->rotary_dim / 2; ++k)
        if (p->axis[k] >= p->axes) return A2SF_ERR_INVALID_ARG;
    return p->rotary_dim <= d ? A2SF_OK : A2SF_ERR_INVALID_ARG;
}

// x and y of a rotation: valid tensors, and in place only with the same strides
int check_rotation(int dtype, int d, const int64_t extent[3], const void *x, const int64_t xs[3], const void *y, const int64_t ys[3])
{
    int rc;
    if ((rc = check_tensor(x, dtype, d, extent, xs)) != A2SF_OK || (rc = check_tensor(y, dtype, d, extent, ys)) != A2SF_OK) return rc;
    if (x == y)
        for (int i = 0; i < 3; ++i)
            if (extent[i] > 1 && xs[i] != ys[i]) return A2SF_ERR_INVALID_ARG;
    return A2SF_OK;
}

int check_paged(const a2sf_paged *p, int c)
{
    if (!p) return A2SF_ERR_INVALID_ARG;
    const int rc = check_shape(p->dtype, p->d);
    if (rc != A2SF_OK) return rc;
    if (p->page_size != 16 && p->page_size != 32 && p->page_size != 64 && p->page_size != 128) return A2SF_ERR_UNSUPPORTED;
    if (p->group < 1 || p->group > A2SF_MAX_GROUP || p->B > A2SF_PAGED_MAX_SEQUENCES) return A2SF_ERR_UNSUPPORTED;
    if (p->B < 1 || p->H < 1 || p->num_pages < 1 || p->max_pages < 1 || c < 1 || p->reserved != 0) return A2SF_ERR_INVALID_ARG;
    if (!(p->scale >= 0.f) || std::isinf(p->scale)) return A2SF_ERR_INVALID_ARG;
    // slots of a sequence, units, folded rows and tiles of a call all stay 32-bit numbers
    if ((int64_t)p->max_pages * p->page_size > (1 << 28) || (int64_t)c * p->group > (1 << 28) ||
        (int64_t)p->B * p->H * p->group > (1 << 24) || (int64_t)p->num_pages * p->H * p->page_size >= (1ll << 31) ||
        ((int64_t)p->max_pages * p->page_size / 128 + 1) * ((int64_t)c * p->group / 64 + 1) >= (1ll << 31))
        return A2SF_ERR_UNSUPPORTED;
    if (!p->k_pages || !p->v_pages || !p->scores || !p->positions || !p->page_table || !p->past) return A2SF_ERR_INVALID_ARG;
    if (!aligned(p->k_pages, 16) || !aligned(p->v_pages, 16) || !aligned(p->scores, 16) || !aligned(p->positions, 16) ||
        !aligned(p->page_table, 4) || !aligned(p->past, 4) || !aligned(p->start, 4))
        return A2SF_ERR_INVALID_ARG;
    return A2SF_OK;
}

PagedView make_view(const a2sf_paged *p, int c, const int32_t *lens)
{
    PagedView v;
    v.k = static_cast<char *>(p->k_pages); v.v = static_cast<char *>(p->v_pages);
    v.scores = p->scores; v.positions = p->positions;
    v.table = p->page_table; v.past = p->past; v.start = p->start; v.lens = lens;
    v.status = nullptr;
    v.B = p->B; v.H = p->H; v.G = p->group; v.d = p->d; v.ps = p->page_size;
    v.ps_shift = p->page_size == 16 ? 4 : p->page_size == 32 ? 5 : p->page_size == 64 ? 6 : 7;
    v.max_pages = p->max_pages; v.num_pages = p->num_pages; v.c = c;
    v.sl2 = (p->scale > 0.f ? p->scale : 1.f / std::sqrt((float)p->d)) * kLog2e;
    return v;
}

PagedView make_window_view(const a2sf_paged *p, int c, const int32_t *lens, int window, int sinks)
{
    PagedView v = make_view(p, c, lens);
    const int cap = p->max_pages * p->page_size;              // nothing is beyond it
    v.window = window < cap ? window : cap;
    v.sinks = sinks < cap ? sinks : cap;
    v.sink_end = (v.sinks + kGrain - 1) / kGrain * kGrain;
    return v;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn()
{
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
    });
    return fn;
}

// Which attention: few rows are bound by the cache's bytes whatever the type; more rows of 32-bit storage by products of
// split operands, of 16-bit storage by tcgen05 -- whose plan, 128-row tiles and one CTA per SM cost more than a small call
// takes.  Small goes by the multiply-adds of Q K^T at the cache's capacity (us, tcgen05 and mma.sync, bf16): 12 heads, 244 tokens,
// 5e7: 14.9 and 12.4; 36 heads, 302 tokens, 2e8: 21.2 and 18.5; 8 heads, 928 tokens, 5e8: 32.1 and 31.7; 32 heads, 100 behind
// 2,000, 9e8: 42 and 70.  One tile of 64 rows: 640 heads, 64 behind 100, 1e9: 71 and 52; 64 x 64 behind 4,000, 2e9: 83 and 96.
enum Path { kFew, kTc, kMma };
// Windowed, a row tile of tcgen05 (256 rows) sees the near capacity of its tokens and that is what counts; long items are cut, and one
// row tile serves earlier (us, tcgen05 and mma.sync, bf16, d 128, kv heads x rows, window): 32 x 32, 1,024, 1.4e8: 28 and 16; 64 x
// 40, 1,000, 3.5e8: 31 and 32; 32 x 64, 4,096, 1.1e9: 34 and 68; 32 x 100, 256, 1.6e8: 16 and 16; 48 x 244, 128, 3.7e8: 15 and 19.
// In 32 bits the few-row kernels, on the CUDA cores, take more than the bytes' time from 8 rows on, and mma.sync can cut a window's keys
// (few rows and mma.sync: 99 heads x 13 rows, 556: 62 and 26; 8 x 16, 8,192: 57 and 38; 8 x 16, 300: 15.5 and 9.5; 32 x 8, 1,024: 18
// and 18; 256 x 8, 300: 37 and 73).
Path path_of(const PagedView &v, bool windowed, int dtype)
{
    const int64_t rows = (int64_t)v.c * v.G;
    if (rows <= (windowed && dtype == A2SF_F32 ? kFewRows / 2 : kFewRows)) return kFew;
    if (dtype == A2SF_F32) return kMma;
    const int tokens = 256 / v.G < v.c ? 256 / v.G : v.c;
    const double work = (double)v.B * v.H * rows * near_capacity(v, windowed, tokens) * v.d;
    return work < (rows > 64 ? 3e8 : windowed ? 4e8 : 1.2e9) ? kMma : kTc;
}

size_t attend_ws_bytes(const PagedView &v, bool windowed, int dtype)
{
    const Path path = path_of(v, windowed, dtype);
    const size_t bytes = align_up(path == kFew ? attend_few_ws_bytes(dtype, v, windowed) : path == kMma ? attend_mma_ws_bytes(dtype, v, windowed)
                                  : windowed ? window_tc_ws_bytes(v) : attend_tc_ws_bytes(v));
    return bytes ? bytes : A2SF_NO_WORKSPACE_BYTES;            // 0 says that arguments are invalid
}

cudaError_t launch_attend(int dtype, const AttendArgs &a, cudaStream_t s)
{
    const Path path = path_of(a.pv, a.windowed, dtype);
    return path == kFew ? launch_attend_few(dtype, a, s) : path == kMma ? launch_attend_mma(dtype, a, s)
           : a.windowed ? launch_window_tc(dtype, a, s) : launch_attend_tc(dtype, a, s);
}

}  // namespace

bool make_pool_map(CUtensorMap *map, int dtype, const void *pool, const PagedView &pv, int box_rows)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const int e = elem_bytes(dtype);
    const cuuint64_t dims[2] = {(cuuint64_t)pv.d, (cuuint64_t)pv.num_pages * pv.H * pv.ps};
    const cuuint64_t strides[1] = {(cuuint64_t)pv.d * e};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / e), (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    const CUtensorMapDataType dt = dtype == A2SF_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == A2SF_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    return fn(map, dt, 2, const_cast<void *>(pool), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Query rows in tiles of 128: box of 64 elements x group heads x 128/group tokens, so that row
// r = token * group + head of a tile stands at row r of shared memory.
bool make_query_map(CUtensorMap *map, int dtype, const void *q, const PagedView &pv, const Strides &st)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)pv.d, (cuuint64_t)pv.H * pv.G, (cuuint64_t)pv.c, (cuuint64_t)pv.B};
    // an axis of extent 1 may come with any stride: one that the map accepts takes its place
    const cuuint64_t row = (cuuint64_t)pv.d * 2;
    const cuuint64_t strides[3] = {dims[1] > 1 ? (cuuint64_t)st.h * 2 : row, dims[2] > 1 ? (cuuint64_t)st.t * 2 : row,
                                   dims[3] > 1 ? (cuuint64_t)st.b * 2 : row};
    const cuuint32_t box[4] = {64, (cuuint32_t)pv.G, (cuuint32_t)(128 / pv.G), 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    const CUtensorMapDataType dt = dtype == A2SF_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    return fn(map, dt, 4, const_cast<void *>(q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace a2sf

using namespace a2sf;

extern "C" {

int a2sf_rotary_plan_init(const a2sf_rotary_config *c, a2sf_rotary_plan *plan)
{
    if (!c || !plan) return A2SF_ERR_INVALID_ARG;
    const int r = c->rotary_dim;
    if (r < 2 || r > 2 * A2SF_ROTARY_MAX_PAIRS || r % 2 || (c->interleaved != 0 && c->interleaved != 1)) return A2SF_ERR_INVALID_ARG;
    if (c->scaling < A2SF_ROTARY_PLAIN || c->scaling > A2SF_ROTARY_RAMP) return A2SF_ERR_INVALID_ARG;
    if (!(c->theta > 1.0) || !std::isfinite(c->theta) || !(c->factor >= 1.0) || !std::isfinite(c->factor)) return A2SF_ERR_INVALID_ARG;
    if (!(c->magnitude >= 0.0) || !std::isfinite(c->magnitude)) return A2SF_ERR_INVALID_ARG;
    if (c->scaling == A2SF_ROTARY_NTK && r < 4) return A2SF_ERR_INVALID_ARG;
    const bool by_length = c->scaling == A2SF_ROTARY_BANDS || c->scaling == A2SF_ROTARY_RAMP;
    if (by_length && (c->original_length < 1 || !(c->low > 0.0) || !(c->high > c->low) || !std::isfinite(c->high))) return A2SF_ERR_INVALID_ARG;

    // A position times a frequency keeps the error of the frequency 2^31 times: 53 bits leave 3e-7 of an angle, 64 bits 1e-10.
    typedef long double wide;
    static_assert(LDBL_MANT_DIG >= 64, "frequencies need 64 bits");
    const wide two_pi = 6.283185307179586476925286766559006L;
    const wide L = c->original_length, factor = c->factor;
    const wide theta = c->scaling == A2SF_ROTARY_NTK ? c->theta * std::pow(factor, r / (r - 2.0L)) : (wide)c->theta;
    // RAMP: pair index at which `beta` turns fit into the original length
    wide lo = 0.0L, hi = 0.0L;
    if (c->scaling == A2SF_ROTARY_RAMP) {
        lo = std::floor(r * std::log(L / (c->high * two_pi)) / (2.0L * std::log((wide)c->theta)));
        hi = std::ceil(r * std::log(L / (c->low * two_pi)) / (2.0L * std::log((wide)c->theta)));
        lo = lo > 0.0L ? lo : 0.0L;
        hi = hi < r - 1.0L ? hi : r - 1.0L;
    }
    for (int k = 0; k < A2SF_ROTARY_MAX_PAIRS; ++k) {
        plan->turn[k] = 0;
        if (k >= r / 2) continue;
        wide f = std::pow(theta, -2.0L * k / r);
        wide keep = 1.0L;                                             // share that is not interpolated
        if (c->scaling == A2SF_ROTARY_LINEAR) keep = 0.0L;
        if (c->scaling == A2SF_ROTARY_BANDS) keep = (L * f / two_pi - c->low) / ((wide)c->high - c->low);
        if (c->scaling == A2SF_ROTARY_RAMP) keep = 1.0L - (k - lo) / (hi - lo > 0.001L ? hi - lo : 0.001L);
        keep = keep < 0.0L ? 0.0L : keep > 1.0L ? 1.0L : keep;
        f = keep * f + (1.0L - keep) * f / factor;
        // turns per position are below 1/6: 2^64 times that fits
        plan->turn[k] = (uint64_t)std::ldexp(f / two_pi, 64);
    }
    plan->rotary_dim = r;
    plan->interleaved = c->interleaved;
    plan->magnitude = (float)(c->magnitude > 0.0 ? c->magnitude
                                                 : c->scaling == A2SF_ROTARY_RAMP ? 0.1 * std::log(c->factor) + 1.0 : 1.0);
    plan->check = kPlanCheck;
    return A2SF_OK;
}

int a2sf_rotary(const a2sf_rotary_plan *plan, int32_t dtype, int32_t B, int32_t H, int32_t n, int32_t d, const void *x,
                int64_t x_stride_b, int64_t x_stride_h, int64_t x_stride_t, void *y, int64_t y_stride_b,
                int64_t y_stride_h, int64_t y_stride_t, const int32_t *positions, const int32_t *start,
                const int32_t *lens, int32_t flags, void *cuda_stream)
{
    A2SF_TRACE("a2sf_rotary");
    int rc = check_shape(dtype, d);
    if (rc != A2SF_OK) return rc;
    if (B < 1 || H < 1 || n < 1 || (flags & ~A2SF_ROTARY_TRANSPOSE)) return A2SF_ERR_INVALID_ARG;
    if ((rc = check_plan(plan, d)) != A2SF_OK) return rc;
    const int64_t extent[3] = {B, H, n};
    const int64_t xs[3] = {x_stride_b, x_stride_h, x_stride_t}, ys[3] = {y_stride_b, y_stride_h, y_stride_t};
    if ((rc = check_tensor(x, dtype, d, extent, xs)) != A2SF_OK || (rc = check_tensor(y, dtype, d, extent, ys)) != A2SF_OK) return rc;
    if (!aligned(positions, 4) || !aligned(start, 4) || !aligned(lens, 4)) return A2SF_ERR_INVALID_ARG;
    if (x == y)
        for (int i = 0; i < 3; ++i)
            if (extent[i] > 1 && xs[i] != ys[i]) return A2SF_ERR_INVALID_ARG;
    RotaryArgs r = {};
    r.x = x; r.y = y;
    r.sx = Strides{x_stride_b, x_stride_h, x_stride_t};
    r.sy = Strides{y_stride_b, y_stride_h, y_stride_t};
    r.positions = positions; r.start = start; r.lens = lens;
    r.B = B; r.n = n; r.d = d; r.Hq = H; r.Hk = 0;
    r.transpose = flags & A2SF_ROTARY_TRANSPOSE;
    return launch_rotary(dtype, plan, r, nullptr, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? A2SF_OK : A2SF_ERR_CUDA;
}

int a2sf_rotary_axes_plan_init(int32_t axes, const int32_t *pairs, int32_t order, const a2sf_rotary_plan *plans, int32_t n_plans,
                               a2sf_rotary_axes_plan *plan)
{
    if (axes < 1 || axes > A2SF_ROTARY_MAX_AXES || !pairs || !plans || !plan || (n_plans != 1 && n_plans != axes)) return A2SF_ERR_INVALID_ARG;
    if (order != A2SF_ROTARY_BLOCKS && order != A2SF_ROTARY_CYCLE) return A2SF_ERR_INVALID_ARG;
    int total = 0;
    for (int a = 0; a < axes; ++a) {
        if (pairs[a] < 1 || pairs[a] > A2SF_ROTARY_MAX_PAIRS) return A2SF_ERR_INVALID_ARG;
        total += pairs[a];
    }
    if (total > A2SF_ROTARY_MAX_PAIRS) return A2SF_ERR_INVALID_ARG;
    for (int p = 0; p < n_plans; ++p) {
        if (check_plan(&plans[p], 2 * A2SF_ROTARY_MAX_PAIRS) != A2SF_OK || plans[p].rotary_dim != 2 * (n_plans == 1 ? total : pairs[p]) ||
            plans[p].interleaved != plans[0].interleaved || plans[p].magnitude != plans[0].magnitude)
            return A2SF_ERR_INVALID_ARG;
    }
    int taken[A2SF_ROTARY_MAX_AXES] = {};
    int turn = 0;                                             // whose it is
    for (int k = 0; k < A2SF_ROTARY_MAX_PAIRS; ++k) {
        plan->turn[k] = 0;
        plan->axis[k] = 0;
        if (k >= total) continue;
        while (taken[turn] == pairs[turn]) turn = (turn + 1) % axes;
        plan->axis[k] = (uint8_t)turn;
        plan->turn[k] = n_plans == 1 ? plans[0].turn[k] : plans[turn].turn[taken[turn]];
        ++taken[turn];
        if (order == A2SF_ROTARY_CYCLE) turn = (turn + 1) % axes;
    }
    plan->rotary_dim = 2 * total;
    plan->interleaved = plans[0].interleaved;
    plan->magnitude = plans[0].magnitude;
    plan->axes = axes;
    plan->reserved = 0;
    plan->check = kAxesPlanCheck;
    return A2SF_OK;
}

int a2sf_rotary_axes(const a2sf_rotary_axes_plan *plan, int32_t dtype, int32_t B, int32_t H, int32_t n, int32_t d, const void *x,
                     int64_t x_stride_b, int64_t x_stride_h, int64_t x_stride_t, void *y, int64_t y_stride_b, int64_t y_stride_h,
                     int64_t y_stride_t, const int32_t *positions, const int32_t *lens, int32_t flags, void *cuda_stream)
{
    A2SF_TRACE("a2sf_rotary_axes");
    int rc = check_shape(dtype, d);
    if (rc != A2SF_OK) return rc;
    if (B < 1 || H < 1 || n < 1 || (flags & ~A2SF_ROTARY_TRANSPOSE)) return A2SF_ERR_INVALID_ARG;
    if ((rc = check_axes_plan(plan, d)) != A2SF_OK) return rc;
    const int64_t extent[3] = {B, H, n};
    const int64_t xs[3] = {x_stride_b, x_stride_h, x_stride_t}, ys[3] = {y_stride_b, y_stride_h, y_stride_t};
    if ((rc = check_rotation(dtype, d, extent, x, xs, y, ys)) != A2SF_OK) return rc;
    if (!positions || !aligned(positions, 4) || !aligned(lens, 4)) return A2SF_ERR_INVALID_ARG;
    RotaryArgs r = {};
    r.x = x; r.y = y;
    r.sx = Strides{x_stride_b, x_stride_h, x_stride_t};
    r.sy = Strides{y_stride_b, y_stride_h, y_stride_t};
    r.positions = positions; r.lens = lens;
    r.B = B; r.n = n; r.d = d; r.Hq = H; r.Hk = 0;
    r.transpose = flags & A2SF_ROTARY_TRANSPOSE;
    return launch_rotary_axes(dtype, plan, r, nullptr, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? A2SF_OK : A2SF_ERR_CUDA;
}

int a2sf_paged_append_axes(const a2sf_paged *cache, const a2sf_rotary_axes_plan *plan, const int32_t *positions, int32_t c, const int32_t *lens,
                           const void *k, const void *v, int64_t kv_stride_b, int64_t kv_stride_h, int64_t kv_stride_t,
                           const void *q, int64_t q_stride_b, int64_t q_stride_h, int64_t q_stride_t, void *q_out,
                           int64_t qo_stride_b, int64_t qo_stride_h, int64_t qo_stride_t, void *cuda_stream)
{
    A2SF_TRACE("a2sf_paged_append_axes");
    int rc = check_paged(cache, c);
    if (rc != A2SF_OK) return rc;
    if ((rc = check_axes_plan(plan, cache->d)) != A2SF_OK) return rc;
    if (!positions || !aligned(positions, 4) || !aligned(lens, 4)) return A2SF_ERR_INVALID_ARG;
    const int64_t ekv[3] = {cache->B, cache->H, c}, eq[3] = {cache->B, (int64_t)cache->H * cache->group, c};
    const int64_t skv[3] = {kv_stride_b, kv_stride_h, kv_stride_t};
    const int64_t sq[3] = {q_stride_b, q_stride_h, q_stride_t}, so[3] = {qo_stride_b, qo_stride_h, qo_stride_t};
    if ((rc = check_tensor(k, cache->dtype, cache->d, ekv, skv)) != A2SF_OK || (rc = check_tensor(v, cache->dtype, cache->d, ekv, skv)) != A2SF_OK)
        return rc;
    if (q && (rc = check_rotation(cache->dtype, cache->d, eq, q, sq, q_out, so)) != A2SF_OK) return rc;
    PagedView pv = make_view(cache, c, lens);
    if (!(pv.status = paged_status_word())) return A2SF_ERR_CUDA;
    RotaryArgs r = {};
    r.x = q; r.y = q_out; r.k = k; r.v = v;
    r.sx = Strides{q_stride_b, q_stride_h, q_stride_t};
    r.sy = Strides{qo_stride_b, qo_stride_h, qo_stride_t};
    r.skv = Strides{kv_stride_b, kv_stride_h, kv_stride_t};
    r.positions = positions; r.start = cache->start; r.lens = lens;
    r.B = cache->B; r.n = c; r.d = cache->d;
    r.Hq = q ? cache->H * cache->group : 0;
    r.Hk = cache->H;
    return launch_rotary_axes(cache->dtype, plan, r, &pv, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? A2SF_OK : A2SF_ERR_CUDA;
}

int a2sf_paged_append(const a2sf_paged *cache, const a2sf_rotary_plan *rotary, int32_t c, const int32_t *lens,
                      const void *k, const void *v, int64_t kv_stride_b, int64_t kv_stride_h, int64_t kv_stride_t,
                      const void *q, int64_t q_stride_b, int64_t q_stride_h, int64_t q_stride_t, void *q_out,
                      int64_t qo_stride_b, int64_t qo_stride_h, int64_t qo_stride_t, void *cuda_stream)
{
    A2SF_TRACE("a2sf_paged_append");
    int rc = check_paged(cache, c);
    if (rc != A2SF_OK) return rc;
    if (rotary && (rc = check_plan(rotary, cache->d)) != A2SF_OK) return rc;
    if (q && (!rotary || !q_out)) return A2SF_ERR_INVALID_ARG;
    if (!aligned(lens, 4)) return A2SF_ERR_INVALID_ARG;
    const int64_t ekv[3] = {cache->B, cache->H, c}, eq[3] = {cache->B, (int64_t)cache->H * cache->group, c};
    const int64_t skv[3] = {kv_stride_b, kv_stride_h, kv_stride_t};
    const int64_t sq[3] = {q_stride_b, q_stride_h, q_stride_t}, so[3] = {qo_stride_b, qo_stride_h, qo_stride_t};
    if ((rc = check_tensor(k, cache->dtype, cache->d, ekv, skv)) != A2SF_OK ||
        (rc = check_tensor(v, cache->dtype, cache->d, ekv, skv)) != A2SF_OK)
        return rc;
    if (q) {
        if ((rc = check_tensor(q, cache->dtype, cache->d, eq, sq)) != A2SF_OK ||
            (rc = check_tensor(q_out, cache->dtype, cache->d, eq, so)) != A2SF_OK)
            return rc;
        if (q == q_out)
            for (int i = 0; i < 3; ++i)
                if (eq[i] > 1 && sq[i] != so[i]) return A2SF_ERR_INVALID_ARG;
    }
    PagedView pv = make_view(cache, c, lens);
    if (!(pv.status = paged_status_word())) return A2SF_ERR_CUDA;
    RotaryArgs r = {};
    r.x = q; r.y = q_out; r.k = k; r.v = v;
    r.sx = Strides{q_stride_b, q_stride_h, q_stride_t};
    r.sy = Strides{qo_stride_b, qo_stride_h, qo_stride_t};
    r.skv = Strides{kv_stride_b, kv_stride_h, kv_stride_t};
    r.start = cache->start; r.lens = lens;
    r.B = cache->B; r.n = c; r.d = cache->d;
    r.Hq = q ? cache->H * cache->group : 0;
    r.Hk = cache->H;
    return launch_rotary(cache->dtype, rotary, r, &pv, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? A2SF_OK : A2SF_ERR_CUDA;
}

size_t a2sf_paged_attend_workspace_bytes(const a2sf_paged *cache, int32_t c)
{
    if (check_paged(cache, c) != A2SF_OK) return 0;
    return attend_ws_bytes(make_view(cache, c, nullptr), false, cache->dtype);
}

int a2sf_paged_attend(const a2sf_paged *cache, int32_t c, const int32_t *lens, float alpha, const void *q,
                      int64_t q_stride_b, int64_t q_stride_h, int64_t q_stride_t, void *out, int64_t out_stride_b,
                      int64_t out_stride_h, int64_t out_stride_t, float *lse, int32_t flags, void *workspace,
                      size_t workspace_bytes, void *cuda_stream)
{
    A2SF_TRACE("a2sf_paged_attend");
    int rc = check_paged(cache, c);
    if (rc != A2SF_OK) return rc;
    if (!(alpha >= 0.f && alpha <= 1.f) || (flags & ~A2SF_ATTEND_NO_SCORES)) return A2SF_ERR_INVALID_ARG;
    const int64_t eq[3] = {cache->B, (int64_t)cache->H * cache->group, c};
    const int64_t sq[3] = {q_stride_b, q_stride_h, q_stride_t}, so[3] = {out_stride_b, out_stride_h, out_stride_t};
    if ((rc = check_tensor(q, cache->dtype, cache->d, eq, sq)) != A2SF_OK ||
        (rc = check_tensor(out, cache->dtype, cache->d, eq, so)) != A2SF_OK)
        return rc;
    if (!aligned(lens, 4) || !aligned(lse, 4) || !workspace || !aligned(workspace, 256)) return A2SF_ERR_INVALID_ARG;
    if (q == out) return A2SF_ERR_INVALID_ARG;               // the scores read the queries after the outputs are written
    if (workspace_bytes < a2sf_paged_attend_workspace_bytes(cache, c)) return A2SF_ERR_WORKSPACE;
    AttendArgs a;
    a.pv = make_view(cache, c, lens);
    if (!(a.pv.status = paged_status_word())) return A2SF_ERR_CUDA;
    a.q = q; a.out = out; a.lse = lse;
    a.sq = Strides{q_stride_b, q_stride_h, q_stride_t};
    a.so = Strides{out_stride_b, out_stride_h, out_stride_t};
    a.alpha = alpha; a.nl2a = neg_log2(alpha);
    a.scores = !(flags & A2SF_ATTEND_NO_SCORES);
    a.windowed = false;
    a.ws = workspace;
    return launch_attend(cache->dtype, a, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? A2SF_OK : A2SF_ERR_CUDA;
}

size_t a2sf_paged_attend_window_workspace_bytes(const a2sf_paged *cache, int32_t c, int32_t window, int32_t sinks)
{
    if (check_paged(cache, c) != A2SF_OK || window < 1 || sinks < 0) return 0;
    return attend_ws_bytes(make_window_view(cache, c, nullptr, window, sinks), true, cache->dtype);
}

int a2sf_paged_attend_window(const a2sf_paged *cache, int32_t c, const int32_t *lens, int32_t window, int32_t sinks, const void *q,
                             int64_t q_stride_b, int64_t q_stride_h, int64_t q_stride_t, void *out, int64_t out_stride_b,
                             int64_t out_stride_h, int64_t out_stride_t, float *lse, void *workspace, size_t workspace_bytes,
                             void *cuda_stream)
{
    A2SF_TRACE("a2sf_paged_attend_window");
    int rc = check_paged(cache, c);
    if (rc != A2SF_OK) return rc;
    if (window < 1 || sinks < 0) return A2SF_ERR_INVALID_ARG;
    const int64_t eq[3] = {cache->B, (int64_t)cache->H * cache->group, c};
    const int64_t sq[3] = {q_stride_b, q_stride_h, q_stride_t}, so[3] = {out_stride_b, out_stride_h, out_stride_t};
    if ((rc = check_tensor(q, cache->dtype, cache->d, eq, sq)) != A2SF_OK ||
        (rc = check_tensor(out, cache->dtype, cache->d, eq, so)) != A2SF_OK)
        return rc;
    if (!aligned(lens, 4) || !aligned(lse, 4) || !workspace || !aligned(workspace, 256)) return A2SF_ERR_INVALID_ARG;
    if (q == out) return A2SF_ERR_INVALID_ARG;
    AttendArgs a;
    a.pv = make_window_view(cache, c, lens, window, sinks);
    if (workspace_bytes < attend_ws_bytes(a.pv, true, cache->dtype)) return A2SF_ERR_WORKSPACE;
    if (!(a.pv.status = paged_status_word())) return A2SF_ERR_CUDA;
    a.q = q; a.out = out; a.lse = lse;
    a.sq = Strides{q_stride_b, q_stride_h, q_stride_t};
    a.so = Strides{out_stride_b, out_stride_h, out_stride_t};
    a.alpha = 1.f; a.nl2a = 0.f;
    a.scores = false;
    a.windowed = true;
    a.ws = workspace;
    return launch_attend(cache->dtype, a, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? A2SF_OK : A2SF_ERR_CUDA;
}

int a2sf_paged_slide(const a2sf_paged *cache, int32_t c, const int32_t *lens, int32_t window, int32_t sinks, int32_t *table_out,
                     int32_t *freed, int32_t *freed_count, int32_t *past_out, int32_t *start_out, void *cuda_stream)
{
    A2SF_TRACE("a2sf_paged_slide");
    const int rc = check_paged(cache, c);
    if (rc != A2SF_OK) return rc;
    if (window < 1 || sinks < 0 || !table_out || !past_out || !start_out) return A2SF_ERR_INVALID_ARG;
    // a block reads one sequence's entries and writes its outputs: an output may be the array it comes from, and else touches
    // no input and no other output
    const size_t B = cache->B, pages = B * cache->max_pages;
    const struct { const int32_t *p, *from; size_t n; } outs[] = {{table_out, cache->page_table, pages}, {past_out, cache->past, B},
                                                                  {start_out, cache->start, B}, {freed, nullptr, pages}, {freed_count, nullptr, B}};
    const struct { const int32_t *p; size_t n; } ins[] = {{cache->page_table, pages}, {cache->past, B}, {cache->start, B}, {lens, B}};
    auto meet = [](const int32_t *a, size_t na, const int32_t *b, size_t nb) {
        const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
        return a && b && x < y + nb * 4 && y < x + na * 4;
    };
    for (int x = 0; x < 5; ++x) {
        if (!aligned(outs[x].p, 4)) return A2SF_ERR_INVALID_ARG;
        for (int y = 0; y < x; ++y)
            if (meet(outs[x].p, outs[x].n, outs[y].p, outs[y].n)) return A2SF_ERR_INVALID_ARG;
        for (const auto &in : ins)
            if (meet(outs[x].p, outs[x].n, in.p, in.n) && !(outs[x].p == outs[x].from && in.p == outs[x].from)) return A2SF_ERR_INVALID_ARG;
    }
    if (!aligned(lens, 4)) return A2SF_ERR_INVALID_ARG;
    PagedView pv = make_view(cache, c, lens);
    if (!(pv.status = paged_status_word())) return A2SF_ERR_CUDA;
    const int cap = cache->max_pages * cache->page_size;       // nothing is beyond it
    const SlideArgs a = {table_out, freed, freed_count, past_out, start_out, window < cap ? window : cap, sinks < cap ? sinks : cap};
    return launch_slide(pv, a, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? A2SF_OK : A2SF_ERR_CUDA;
}

size_t a2sf_paged_evict_workspace_bytes(const a2sf_paged *cache, int32_t budget)
{
    if (check_paged(cache, 1) != A2SF_OK || budget < 1) return 0;
    const int64_t cap = (int64_t)cache->max_pages * cache->page_size;
    return evict_ws_bytes((size_t)cache->B * cache->H, budget < cap ? budget : (int)cap);
}

int a2sf_paged_evict(const a2sf_paged *cache, int32_t c, const int32_t *lens, int32_t budget, int32_t recent,
                     const int32_t *dst_table, int32_t dst_max_pages, int32_t *past_out, int32_t *start_out,
                     void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    A2SF_TRACE("a2sf_paged_evict");
    const int rc = check_paged(cache, c);
    if (rc != A2SF_OK) return rc;
    if (budget < 1 || recent < 0 || recent > budget || !past_out || !start_out) return A2SF_ERR_INVALID_ARG;
    if (!aligned(lens, 4) || !aligned(dst_table, 4) || !aligned(past_out, 4) || !aligned(start_out, 4) || past_out == start_out)
        return A2SF_ERR_INVALID_ARG;
    const int64_t cap = (int64_t)cache->max_pages * cache->page_size;
    const int M = budget < cap ? budget : (int)cap;           // n never exceeds the capacity
    if (dst_table && (dst_max_pages < 1 || (int64_t)dst_max_pages * cache->page_size < M)) return A2SF_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256)) return A2SF_ERR_INVALID_ARG;
    if (workspace_bytes < a2sf_paged_evict_workspace_bytes(cache, budget)) return A2SF_ERR_WORKSPACE;
    PagedView pv = make_view(cache, c, lens);
    if (!(pv.status = paged_status_word())) return A2SF_ERR_CUDA;
    return launch_evict(elem_bytes(cache->dtype), pv, M, recent, dst_table, dst_max_pages, past_out, start_out, workspace,
                        static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? A2SF_OK : A2SF_ERR_CUDA;
}

}  // extern "C"
