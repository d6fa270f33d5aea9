// extern "C" boundary of libnystra: argument validation, option resolution,
// kernel-family selection and launch.  Every check runs before anything is
// enqueued; the layer allocates nothing and never synchronises.
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <mutex>

#include "../../include/nystra.h"
#include "internal.hpp"

namespace nystra {

bool make_geometry(int N, int m, int mode, Geometry *g)
{
    if (N < 1 || m < 1 || m > N)
        return false;
    if (mode == NYSTRA_LM_POOL2D) {
        int w = int(sqrt(double(N)) + 0.5);
        if (w * w != N)
            return false;
        int best = 0;
        for (int gc = 1; gc * gc <= m; ++gc)
            if (m % gc == 0 && w % gc == 0 && w % (m / gc) == 0)
                best = gc;
        if (best == 0)
            return false;
        *g = Geometry{w, w, w / (m / best), w / best, best};
        return true;
    }
    if (mode == NYSTRA_LM_SEGMENT1D) {
        if (N % m != 0)
            return false;
        *g = Geometry{1, N, 1, N / m, m};
        return true;
    }
    return false;
}

size_t generic_lds_bytes(int m, int d);

}  // namespace nystra

using nystra::Problem;

namespace {

// Tokens per window: up to 2^20 (a 1024 x 1024 map as one global window).  The
// kernels stream over tokens with 64-bit offsets and size LDS independently of N.
constexpr int kMaxN = 1 << 20;
constexpr int kMaxD = 128;
constexpr int kMaxM = 64;
constexpr int kMaxIters = 64;
// Units per call: every kernel's grid is at most 256 work-items per unit in its
// x dimension, and a launch holds fewer than 2^32 work-items per dimension.
constexpr int64_t kMaxUnits = (int64_t(1) << 24) - 1;

thread_local char g_last_error[256] = "";

void set_last_error(const char *msg)
{
    strncpy(g_last_error, msg ? msg : "", sizeof(g_last_error) - 1);
    g_last_error[sizeof(g_last_error) - 1] = '\0';
}

int dtype_bytes(int dtype) { return dtype == NYSTRA_F32 ? 4 : 2; }

bool misaligned(const void *p, int bytes) { return (uintptr_t(p) % uintptr_t(bytes)) != 0; }

bool overlaps(const void *a, int64_t an, const void *b, int64_t bn)
{
    const uintptr_t a0 = uintptr_t(a), b0 = uintptr_t(b);
    return a0 < b0 + uintptr_t(bn) && b0 < a0 + uintptr_t(an);
}

// Shape, dtype and count checks shared by every device entry point.
int check_common(int n_windows, int heads, int N, int d, int dtype, int64_t *units)
{
    if (dtype != NYSTRA_F32 && dtype != NYSTRA_BF16)
        return NYSTRA_ERR_DTYPE;
    if (n_windows < 0 || heads < 0 || N < 1 || N > kMaxN || d < 1 || d > kMaxD)
        return NYSTRA_ERR_SHAPE;
    const int64_t u = int64_t(n_windows) * int64_t(heads);
    if (u > kMaxUnits)
        return NYSTRA_ERR_SHAPE;
    *units = u;
    return NYSTRA_OK;
}

// Pointer checks: non-null, element-aligned, O disjoint from the inputs.
int check_tensors(const void *Q, const void *K, const void *V, const void *O, int64_t bytes,
                  int ebytes)
{
    if (!Q || !K || !V || !O)
        return NYSTRA_ERR_NULL;
    if (misaligned(Q, ebytes) || misaligned(K, ebytes) || misaligned(V, ebytes) ||
        misaligned(O, ebytes))
        return NYSTRA_ERR_ALIGN;
    if (overlaps(O, bytes, Q, bytes) || overlaps(O, bytes, K, bytes) ||
        overlaps(O, bytes, V, bytes))
        return NYSTRA_ERR_OVERLAP;
    return NYSTRA_OK;
}

// hipGetLastError() reports the last error of any HIP call on this thread.
// Each entry point clears it right before its first launch, so that the
// status it returns speaks of its own launches only.
void clear_stale_error() { (void)hipGetLastError(); }

int finish_launch(hipError_t e)
{
    if (e != hipSuccess) {
        set_last_error(hipGetErrorString(e));
        return NYSTRA_ERR_HIP;
    }
    return NYSTRA_OK;
}

// Token-split kernels pay off for long windows: from 64 x 64 tokens on they beat
// one workgroup per unit at every unit count measured (384 to 1536 units),
// from 2048 tokens when the units are too few to fill the GPU (< 512).  At
// 32 x 32 windows with 1536 units the one-pass kernel is faster.
bool split_preferred(const Problem &p)
{
    return p.N >= 4096 || (p.N >= 2048 && p.units < 512);
}

// What AUTO runs on a shape that only the generic family accepts by name (N not
// a multiple of 16) but the tiled kernels cover with a partial last tile: 10 x 10
// windows, m = 25, d_h = 16, 3072 units fp32 took 1270 us in the generic kernel
// and 86 us tiled.  nystra_select_variant() reports it as GENERIC, and
// forcing TILED on such a shape stays refused.
constexpr int kVariantRagged = 100;

// Resolves options and the problem; does not touch device memory.  with_ws
// says whether the entry point takes a workspace (and so may run the
// token-split kernels).
int build_problem(const void *Q, const void *K, const void *V, void *O, int n_windows,
                  int heads, int N, int d, int m, int dtype, const nystra_opts *opts,
                  bool with_ws, Problem *p, int *variant)
{
    nystra_opts o;
    nystra_default_opts(&o);
    if (opts)
        o = *opts;
    int64_t units = 0;
    int rc = check_common(n_windows, heads, N, d, dtype, &units);
    if (rc != NYSTRA_OK)
        return rc;
    if (m < 1 || m > N || m > kMaxM)
        return NYSTRA_ERR_SHAPE;
    if (o.pinv_iters < 0 || o.pinv_iters > kMaxIters || !isfinite(o.scale) ||
        (o.landmark_mode != NYSTRA_LM_POOL2D && o.landmark_mode != NYSTRA_LM_SEGMENT1D) ||
        o.variant < NYSTRA_VARIANT_AUTO || o.variant > NYSTRA_VARIANT_SPLIT)
        return NYSTRA_ERR_ARG;
    nystra::Geometry g;
    if (!nystra::make_geometry(N, m, o.landmark_mode, &g))
        return NYSTRA_ERR_SHAPE;
    p->q = Q;
    p->k = K;
    p->v = V;
    p->o = O;
    p->units = units;
    p->N = N;
    p->d = d;
    p->m = m;
    p->iters = o.pinv_iters;
    p->dtype = dtype;
    p->scale = o.scale > 0.f ? o.scale : float(1.0 / sqrt(double(d)));
    p->geo = g;
    const bool tiled = nystra::tiled_supported(*p);
    const bool split = with_ws && nystra::split_supported(*p);
    switch (o.variant) {
    case NYSTRA_VARIANT_GENERIC:
        *variant = NYSTRA_VARIANT_GENERIC;
        return NYSTRA_OK;
    case NYSTRA_VARIANT_TILED:
        *variant = NYSTRA_VARIANT_TILED;
        return tiled ? NYSTRA_OK : NYSTRA_ERR_UNSUPPORTED;
    case NYSTRA_VARIANT_SPLIT:
        *variant = NYSTRA_VARIANT_SPLIT;
        return split ? NYSTRA_OK : NYSTRA_ERR_UNSUPPORTED;
    default:
        *variant = (split && split_preferred(*p)) ? NYSTRA_VARIANT_SPLIT
                   : tiled                        ? NYSTRA_VARIANT_TILED
                   : nystra::ragged_supported(*p) ? kVariantRagged
                                                  : NYSTRA_VARIANT_GENERIC;
        return NYSTRA_OK;
    }
}

// The families that take no scratch memory.
hipError_t launch_one_pass(const Problem &p, int variant, hipStream_t s)
{
    if (variant == NYSTRA_VARIANT_TILED)
        return nystra::launch_tiled_forward(p, s);
    if (variant == kVariantRagged)
        return nystra::launch_tiled_large(p, s);
    return nystra::launch_generic_forward(p, s);
}

}  // namespace

extern "C" {

int nystra_default_opts(nystra_opts *opts)
{
    if (!opts)
        return NYSTRA_ERR_NULL;
    opts->pinv_iters = 6;
    opts->landmark_mode = NYSTRA_LM_POOL2D;
    opts->scale = 0.f;
    opts->variant = NYSTRA_VARIANT_AUTO;
    return NYSTRA_OK;
}

int nystra_attn_forward_ex(const void *Q, const void *K, const void *V, void *O, int n_windows,
                           int heads, int N, int d_h, int m, int dtype, const nystra_opts *opts,
                           void *stream)
{
    Problem p;
    int variant = 0;
    int rc = build_problem(Q, K, V, O, n_windows, heads, N, d_h, m, dtype, opts, false, &p,
                           &variant);
    if (rc != NYSTRA_OK)
        return rc;
    if (p.units == 0)
        return NYSTRA_OK;
    const int64_t bytes = p.units * N * d_h * dtype_bytes(dtype);
    rc = check_tensors(Q, K, V, O, bytes, dtype_bytes(dtype));
    if (rc != NYSTRA_OK)
        return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    clear_stale_error();
    return finish_launch(launch_one_pass(p, variant, s));
}

int nystra_attn_workspace_size(int n_windows, int heads, int N, int d_h, int m, int dtype,
                               const nystra_opts *opts, size_t *bytes)
{
    if (!bytes)
        return NYSTRA_ERR_NULL;
    Problem p;
    int variant = 0;
    int rc = build_problem(nullptr, nullptr, nullptr, nullptr, n_windows, heads, N, d_h, m,
                           dtype, opts, true, &p, &variant);
    if (rc != NYSTRA_OK)
        return rc;
    *bytes = (variant == NYSTRA_VARIANT_SPLIT && p.units > 0)
                 ? nystra::split_workspace_bytes(p) : 0;
    return NYSTRA_OK;
}

int nystra_attn_forward_ws(const void *Q, const void *K, const void *V, void *O,
                           int n_windows, int heads, int N, int d_h, int m, int dtype,
                           const nystra_opts *opts, void *workspace, size_t workspace_bytes,
                           void *stream)
{
    Problem p;
    int variant = 0;
    int rc = build_problem(Q, K, V, O, n_windows, heads, N, d_h, m, dtype, opts, true, &p,
                           &variant);
    if (rc != NYSTRA_OK)
        return rc;
    if (p.units == 0)
        return NYSTRA_OK;
    const int64_t bytes = p.units * N * d_h * dtype_bytes(dtype);
    rc = check_tensors(Q, K, V, O, bytes, dtype_bytes(dtype));
    if (rc != NYSTRA_OK)
        return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (variant == NYSTRA_VARIANT_SPLIT) {
        const size_t need = nystra::split_workspace_bytes(p);
        if (!workspace || workspace_bytes < need || misaligned(workspace, 256))
            return NYSTRA_ERR_WORKSPACE;
        const int64_t wn = int64_t(need);
        if (overlaps(workspace, wn, Q, bytes) || overlaps(workspace, wn, K, bytes) ||
            overlaps(workspace, wn, V, bytes) || overlaps(workspace, wn, O, bytes))
            return NYSTRA_ERR_WORKSPACE;
        clear_stale_error();
        return finish_launch(nystra::launch_split(p, workspace, s));
    }
    clear_stale_error();
    return finish_launch(launch_one_pass(p, variant, s));
}

}  // extern "C"

namespace {

// Scratch of the allocation-free entry point: the token-split workspace as a
// static device array.  Every device the library runs on holds its own copy
// at its own address, until the process ends.  In host code `scratch` names a
// host-side stand-in only; kernels receive the device address looked up below.
static __device__ __align__(256) unsigned char scratch[NYSTRA_STATIC_SCRATCH_BYTES];

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void *g_scratch_ptr[kMaxDevices] = {};

// Device address of `scratch` on device `dev`, looked up once per device with
// that device current (the caller's current device, checked by the caller).
hipError_t scratch_address(int dev, void **ptr)
{
    std::lock_guard<std::mutex> lock(g_scratch_mu);
    if (!g_scratch_ptr[dev]) {
        void *p = nullptr;
        const hipError_t e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess)
            return e;
        g_scratch_ptr[dev] = p;
    }
    *ptr = g_scratch_ptr[dev];
    return hipSuccess;
}

}  // namespace

extern "C" {

int nystra_attn_forward_noalloc(const void *Q, const void *K, const void *V, void *O,
                                int n_windows, int heads, int N, int d_h, int m, int dtype,
                                const nystra_opts *opts, void *stream)
{
    Problem p;
    int variant = 0;
    int rc = build_problem(Q, K, V, O, n_windows, heads, N, d_h, m, dtype, opts, true, &p,
                           &variant);
    if (rc != NYSTRA_OK)
        return rc;
    if (p.units == 0)
        return NYSTRA_OK;
    const int64_t bytes = p.units * N * d_h * dtype_bytes(dtype);
    rc = check_tensors(Q, K, V, O, bytes, dtype_bytes(dtype));
    if (rc != NYSTRA_OK)
        return rc;
    const size_t need = variant == NYSTRA_VARIANT_SPLIT ? nystra::split_workspace_bytes(p) : 0;
    if (need > size_t(NYSTRA_STATIC_SCRATCH_BYTES)) {
        set_last_error("token-split workspace exceeds NYSTRA_STATIC_SCRATCH_BYTES");
        return NYSTRA_ERR_WORKSPACE;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    clear_stale_error();
    if (variant != NYSTRA_VARIANT_SPLIT)   // these kernels use no scratch memory
        return finish_launch(launch_one_pass(p, variant, s));
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess)
        return finish_launch(e);
    if (dev < 0 || dev >= kMaxDevices) {
        set_last_error("device index beyond the scratch table");
        return NYSTRA_ERR_ARG;
    }
    if (s) {   // the kernels run on the stream's device; its scratch copy must be the one used
        int sdev = -1;
        e = hipStreamGetDevice(s, &sdev);
        if (e != hipSuccess)
            return finish_launch(e);
        if (sdev != dev) {
            set_last_error("stream does not belong to the current device");
            return NYSTRA_ERR_ARG;
        }
    }
    void *ws = nullptr;
    e = scratch_address(dev, &ws);
    if (e != hipSuccess)
        return finish_launch(e);
    return finish_launch(nystra::launch_split(p, ws, s));
}

int nystra_attn_forward(const void *Q, const void *K, const void *V, void *O, int n_windows,
                        int heads, int N, int d_h, int m, int dtype, void *stream)
{
    return nystra_attn_forward_ex(Q, K, V, O, n_windows, heads, N, d_h, m, dtype, nullptr,
                                  stream);
}

int nystra_exact_attn_forward(const void *Q, const void *K, const void *V, void *O,
                              int n_windows, int heads, int N, int d_h, int dtype, float scale,
                              void *stream)
{
    int64_t units = 0;
    int rc = check_common(n_windows, heads, N, d_h, dtype, &units);
    if (rc != NYSTRA_OK)
        return rc;
    if (!isfinite(scale))
        return NYSTRA_ERR_ARG;
    if (units == 0)
        return NYSTRA_OK;
    const int64_t bytes = units * N * d_h * dtype_bytes(dtype);
    rc = check_tensors(Q, K, V, O, bytes, dtype_bytes(dtype));
    if (rc != NYSTRA_OK)
        return rc;
    Problem p{};
    p.q = Q;
    p.k = K;
    p.v = V;
    p.o = O;
    p.units = units;
    p.N = N;
    p.d = d_h;
    p.m = 0;
    p.dtype = dtype;
    p.scale = scale > 0.f ? scale : float(1.0 / sqrt(double(d_h)));
    clear_stale_error();
    return finish_launch(nystra::launch_exact(p, static_cast<hipStream_t>(stream)));
}

int nystra_landmark_pool(const void *Q, const void *K, float *Qbar, float *Kbar, int32_t *map,
                         int n_windows, int heads, int N, int d_h, int m, int dtype, int mode,
                         void *stream)
{
    int64_t units = 0;
    int rc = check_common(n_windows, heads, N, d_h, dtype, &units);
    if (rc != NYSTRA_OK)
        return rc;
    if (m < 1 || m > N || m > kMaxM)
        return NYSTRA_ERR_SHAPE;
    if (mode != NYSTRA_LM_POOL2D && mode != NYSTRA_LM_SEGMENT1D)
        return NYSTRA_ERR_ARG;
    nystra::Geometry g;
    if (!nystra::make_geometry(N, m, mode, &g))
        return NYSTRA_ERR_SHAPE;
    if (units == 0)
        return NYSTRA_OK;
    const int eb = dtype_bytes(dtype);
    if (!Q || !K || !Qbar || !Kbar)
        return NYSTRA_ERR_NULL;
    if (misaligned(Q, eb) || misaligned(K, eb) || misaligned(Qbar, 4) || misaligned(Kbar, 4) ||
        (map && misaligned(map, 4)))
        return NYSTRA_ERR_ALIGN;
    const int64_t in_bytes = units * N * d_h * eb, out_bytes = units * m * d_h * 4;
    if (overlaps(Qbar, out_bytes, Q, in_bytes) || overlaps(Qbar, out_bytes, K, in_bytes) ||
        overlaps(Kbar, out_bytes, Q, in_bytes) || overlaps(Kbar, out_bytes, K, in_bytes) ||
        overlaps(Qbar, out_bytes, Kbar, out_bytes))
        return NYSTRA_ERR_OVERLAP;
    Problem p{};
    p.q = Q;
    p.k = K;
    p.units = units;
    p.N = N;
    p.d = d_h;
    p.m = m;
    p.dtype = dtype;
    p.geo = g;
    clear_stale_error();
    return finish_launch(
        nystra::launch_landmark_pool(p, Qbar, Kbar, map, static_cast<hipStream_t>(stream)));
}

int nystra_landmark_map(int N, int m, int mode, int32_t *map_host)
{
    if (mode != NYSTRA_LM_POOL2D && mode != NYSTRA_LM_SEGMENT1D)
        return NYSTRA_ERR_ARG;
    if (N < 1 || N > kMaxN || m < 1 || m > N || m > kMaxM)
        return NYSTRA_ERR_SHAPE;
    nystra::Geometry g;
    if (!nystra::make_geometry(N, m, mode, &g))
        return NYSTRA_ERR_SHAPE;
    if (!map_host)
        return NYSTRA_ERR_NULL;
    for (int t = 0; t < N; ++t) {
        const int r = t / g.cols, c = t % g.cols;
        map_host[t] = (r / g.pr) * g.gc + c / g.pc;
    }
    return NYSTRA_OK;
}

int nystra_select_variant(int N, int d_h, int m, int dtype, const nystra_opts *opts)
{
    Problem p;
    int variant = 0;
    int rc = build_problem(nullptr, nullptr, nullptr, nullptr, 1, 1, N, d_h, m, dtype, opts,
                           false, &p, &variant);
    if (rc != NYSTRA_OK)
        return -rc;
    return variant == kVariantRagged ? int(NYSTRA_VARIANT_GENERIC) : variant;
}

}  // extern "C"

namespace {

// Workspace layout of the block: Q, K, V, O, the packed weights of the two
// GEMMs (when C <= 256), then the attention's own.
struct BlockPlan {
    Problem p;          // the attention problem on the workspace tensors
    int variant;        // attention kernel family (Nystrom) or -1 (exact)
    size_t qkvo_bytes;  // one of the four tensors, padded to 256 bytes
    size_t pk_qkv, pk_proj;   // packed W_qkv and W_proj, padded to 256 bytes (0: none)
    size_t bytes;       // total
};

size_t pad256(size_t x) { return (x + 255) & ~size_t(255); }

int plan_block(const nystra_block_shape *s, int m, int dtype, const nystra_opts *opts,
               int attention, BlockPlan *bp)
{
    if (!s)
        return NYSTRA_ERR_NULL;
    if (dtype != NYSTRA_F32 && dtype != NYSTRA_BF16)
        return NYSTRA_ERR_DTYPE;
    if (attention != NYSTRA_BLOCK_NYSTROM && attention != NYSTRA_BLOCK_EXACT)
        return NYSTRA_ERR_ARG;
    if (s->batch < 0 || s->height < 1 || s->width < 1 || s->window < 1 || s->heads < 1 ||
        s->channels < 1 || s->channels > 4096 || s->channels % s->heads != 0 ||
        s->height % s->window != 0 || s->width % s->window != 0 || s->shift < 0 ||
        s->shift >= s->window || s->window > 1024)
        return NYSTRA_ERR_SHAPE;
    const int64_t rows = int64_t(s->batch) * s->height * s->width;
    if (rows > int64_t(INT32_MAX) || !nystra::block_gemm_supported(rows, s->channels))
        return NYSTRA_ERR_SHAPE;
    const int64_t nw = int64_t(s->batch) * (s->height / s->window) * (s->width / s->window);
    if (nw > int64_t(INT32_MAX))
        return NYSTRA_ERR_SHAPE;
    const int N = s->window * s->window, d = s->channels / s->heads;
    int rc;
    if (attention == NYSTRA_BLOCK_NYSTROM) {
        rc = build_problem(nullptr, nullptr, nullptr, nullptr, int(nw), s->heads, N, d, m, dtype,
                           opts, true, &bp->p, &bp->variant);
    } else {
        int64_t units = 0;
        rc = check_common(int(nw), s->heads, N, d, dtype, &units);
        if (rc == NYSTRA_OK && opts && !isfinite(opts->scale))
            rc = NYSTRA_ERR_ARG;
        bp->p = Problem{};
        bp->p.units = units;
        bp->p.N = N;
        bp->p.d = d;
        bp->p.dtype = dtype;
        const float sc = opts ? opts->scale : 0.f;
        bp->p.scale = sc > 0.f ? sc : float(1.0 / sqrt(double(d)));
        bp->variant = -1;
    }
    if (rc != NYSTRA_OK)
        return rc;
    bp->qkvo_bytes = pad256(size_t(rows) * s->channels * dtype_bytes(dtype));
    bp->pk_qkv = pad256(nystra::block_wpack_bytes(s->channels, 3 * s->channels, dtype));
    bp->pk_proj = pad256(nystra::block_wpack_bytes(s->channels, s->channels, dtype));
    bp->bytes = 4 * bp->qkvo_bytes + bp->pk_qkv + bp->pk_proj;
    if (bp->variant == NYSTRA_VARIANT_SPLIT && bp->p.units > 0)
        bp->bytes += nystra::split_workspace_bytes(bp->p);
    return NYSTRA_OK;
}

// Bytes of the packed W_qkv and W_proj image (each part padded to 256 bytes;
// 0 when channels > 256).
size_t packed_parts(int C, int dtype, size_t *qkv_part)
{
    const size_t q = pad256(nystra::block_wpack_bytes(C, 3 * C, dtype));
    *qkv_part = q;
    return q + pad256(nystra::block_wpack_bytes(C, C, dtype));
}

// The block of nystra_block_forward.  With with_packed, the GEMMs read the
// weight image at `packed` (required when channels <= 256, ignored above)
// instead of packing W_qkv and W_proj into the workspace first.  With `layer`, a
// whole transformer layer: the QKV product normalises its rows, and the tail
// kernel takes the place of the PROJ product.
int block_forward(const void *X, const void *Wqkv, const void *bqkv, const void *Wproj,
                  const void *bproj, bool with_packed, const void *packed,
                  size_t packed_bytes, void *Y,
                  const nystra_block_shape *shape, int m, int dtype, const nystra_opts *opts,
                  int attention, void *workspace, size_t workspace_bytes, void *stream,
                  const nystra_layer_params *layer = nullptr)
{
    BlockPlan bp;
    int rc = plan_block(shape, m, dtype, opts, attention, &bp);
    if (rc != NYSTRA_OK)
        return rc;
    if (layer && !nystra::layer_supported(int64_t(shape->batch) * shape->height * shape->width,
                                          shape->channels, shape->heads, dtype, layer->hidden))
        return NYSTRA_ERR_UNSUPPORTED;
    if (shape->batch == 0)
        return NYSTRA_OK;
    const bool use_packed = with_packed && bp.pk_qkv != 0;
    if (!X || !Wqkv || !Wproj || !Y || (use_packed && !packed))
        return NYSTRA_ERR_NULL;
    const int eb = dtype_bytes(dtype), C = shape->channels;
    if (misaligned(X, eb) || misaligned(Wqkv, eb) || misaligned(Wproj, eb) || misaligned(Y, eb) ||
        (bqkv && misaligned(bqkv, eb)) || (bproj && misaligned(bproj, eb)))
        return NYSTRA_ERR_ALIGN;
    const int64_t rows = int64_t(shape->batch) * shape->height * shape->width;
    const int64_t xb = rows * C * eb, wqb = int64_t(C) * 3 * C * eb, wpb = int64_t(C) * C * eb;
    if (overlaps(Y, xb, X, xb) || overlaps(Y, xb, Wqkv, wqb) || overlaps(Y, xb, Wproj, wpb) ||
        (bqkv && overlaps(Y, xb, bqkv, 3 * C * eb)) || (bproj && overlaps(Y, xb, bproj, C * eb)))
        return NYSTRA_ERR_OVERLAP;
    if (!workspace || workspace_bytes < bp.bytes || misaligned(workspace, 256))
        return NYSTRA_ERR_WORKSPACE;
    const int64_t wsb = int64_t(bp.bytes);
    if (overlaps(workspace, wsb, X, xb) || overlaps(workspace, wsb, Y, xb) ||
        overlaps(workspace, wsb, Wqkv, wqb) || overlaps(workspace, wsb, Wproj, wpb) ||
        (bqkv && overlaps(workspace, wsb, bqkv, 3 * C * eb)) ||
        (bproj && overlaps(workspace, wsb, bproj, C * eb)))
        return NYSTRA_ERR_WORKSPACE;
    if (use_packed) {   // read by the GEMMs only: no bytes shared with Y or the workspace
        const int64_t pb = int64_t(bp.pk_qkv + bp.pk_proj);
        if (packed_bytes < size_t(pb))
            return NYSTRA_ERR_WORKSPACE;
        if (misaligned(packed, 256))
            return NYSTRA_ERR_ALIGN;
        if (overlaps(packed, pb, Y, xb) || overlaps(packed, pb, workspace, wsb))
            return NYSTRA_ERR_OVERLAP;
    }
    if (layer) {   // four-byte pieces of X, the MLP weights and Y
        const int64_t hb = int64_t(layer->hidden) * eb, cb = int64_t(C) * eb;
        const struct { const void *p; int64_t n; int align; bool need; } t[] = {
            {layer->norm1_w, cb, eb, true}, {layer->norm1_b, cb, eb, true},
            {layer->norm2_w, cb, eb, true}, {layer->norm2_b, cb, eb, true},
            {layer->w1, hb * C, 4, true},   {layer->b1, hb, eb, false},
            {layer->w2, hb * C, 4, true},   {layer->b2, cb, eb, false},
            {X, xb, 4, true},               {Y, 0, 4, true}};
        for (const auto &x : t) {
            if (!x.p) {
                if (x.need)
                    return NYSTRA_ERR_NULL;
                continue;
            }
            if (misaligned(x.p, x.align))
                return NYSTRA_ERR_ALIGN;
            if (x.n && overlaps(Y, xb, x.p, x.n))
                return NYSTRA_ERR_OVERLAP;
            if (x.n && overlaps(workspace, wsb, x.p, x.n))
                return NYSTRA_ERR_WORKSPACE;
        }
    }
    char *ws = static_cast<char *>(workspace);
    void *q = ws, *k = ws + bp.qkvo_bytes, *v = ws + 2 * bp.qkvo_bytes,
         *o = ws + 3 * bp.qkvo_bytes;
    const char *pkq = nullptr, *pkp = nullptr;
    if (bp.pk_qkv) {
        pkq = use_packed ? static_cast<const char *>(packed) : ws + 4 * bp.qkvo_bytes;
        pkp = pkq + bp.pk_qkv;
    }
    char *attn_ws = ws + 4 * bp.qkvo_bytes + bp.pk_qkv + bp.pk_proj;
    hipStream_t st = static_cast<hipStream_t>(stream);
    clear_stale_error();
    if (pkq && !use_packed) {
        const hipError_t e = nystra::launch_block_wpack(Wqkv, Wproj, C, dtype,
                                                        const_cast<char *>(pkq),
                                                        const_cast<char *>(pkp), st);
        if (e != hipSuccess)
            return finish_launch(e);
    }
    nystra::BlockGemm g;
    g.rows = rows;
    g.H = shape->height;
    g.W = shape->width;
    g.C = C;
    g.heads = shape->heads;
    g.w = shape->window;
    g.shift = shape->shift;
    g.dtype = dtype;
    g.proj = false;
    g.a = X;
    g.wt = Wqkv;
    g.wpk = pkq;
    g.bias = bqkv;
    g.out0 = q;
    g.out1 = k;
    g.out2 = v;
    if (layer) {
        g.lnw = layer->norm1_w;
        g.lnb = layer->norm1_b;
        g.eps = layer->eps1;
    }
    hipError_t e = nystra::launch_block_gemm(g, st);
    if (e != hipSuccess)
        return finish_launch(e);
    Problem p = bp.p;
    p.q = q;
    p.k = k;
    p.v = v;
    p.o = o;
    if (bp.variant == -1)
        e = nystra::launch_exact(p, st);
    else if (bp.variant == NYSTRA_VARIANT_SPLIT)
        e = nystra::launch_split(p, attn_ws, st);
    else
        e = launch_one_pass(p, bp.variant, st);
    if (e != hipSuccess)
        return finish_launch(e);
    g.proj = true;
    g.a = o;
    g.wt = Wproj;
    g.wpk = pkp;
    g.bias = bproj;
    g.out0 = Y;
    g.out1 = g.out2 = nullptr;
    if (layer) {
        nystra::LayerTail t;
        t.gemm = g;
        t.x = X;
        t.lnw = layer->norm2_w;
        t.lnb = layer->norm2_b;
        t.w1 = layer->w1;
        t.b1 = layer->b1;
        t.w2 = layer->w2;
        t.b2 = layer->b2;
        t.eps = layer->eps2;
        t.hidden = layer->hidden;
        return finish_launch(nystra::launch_layer_tail(t, st));
    }
    return finish_launch(nystra::launch_block_gemm(g, st));
}


}  // namespace

extern "C" {

int nystra_block_workspace_size(const nystra_block_shape *shape, int m, int dtype,
                                const nystra_opts *opts, int attention, size_t *bytes)
{
    if (!bytes)
        return NYSTRA_ERR_NULL;
    BlockPlan bp;
    const int rc = plan_block(shape, m, dtype, opts, attention, &bp);
    if (rc != NYSTRA_OK)
        return rc;
    *bytes = shape->batch == 0 ? 0 : bp.bytes;
    return NYSTRA_OK;
}

int nystra_block_forward(const void *X, const void *Wqkv, const void *bqkv, const void *Wproj,
                         const void *bproj, void *Y, const nystra_block_shape *shape, int m,
                         int dtype, const nystra_opts *opts, int attention, void *workspace,
                         size_t workspace_bytes, void *stream)
{
    return block_forward(X, Wqkv, bqkv, Wproj, bproj, false, nullptr, 0, Y, shape, m, dtype,
                         opts, attention, workspace, workspace_bytes, stream);
}

int nystra_block_packed_size(int channels, int dtype, size_t *bytes)
{
    if (!bytes)
        return NYSTRA_ERR_NULL;
    if (dtype != NYSTRA_F32 && dtype != NYSTRA_BF16)
        return NYSTRA_ERR_DTYPE;
    if (channels < 1 || channels > 4096)
        return NYSTRA_ERR_SHAPE;
    size_t q;
    *bytes = packed_parts(channels, dtype, &q);
    return NYSTRA_OK;
}

int nystra_block_pack_weights(const void *Wqkv, const void *Wproj, int channels, int dtype,
                              void *packed, size_t packed_bytes, void *stream)
{
    size_t q = 0, need = 0;
    const int rc = nystra_block_packed_size(channels, dtype, &need);
    if (rc != NYSTRA_OK)
        return rc;
    if (need == 0)
        return NYSTRA_OK;   // channels > 256: the block reads the weights as given
    if (!Wqkv || !Wproj || !packed)
        return NYSTRA_ERR_NULL;
    const int eb = dtype_bytes(dtype);
    if (misaligned(Wqkv, eb) || misaligned(Wproj, eb) || misaligned(packed, 256))
        return NYSTRA_ERR_ALIGN;
    if (packed_bytes < need)
        return NYSTRA_ERR_WORKSPACE;
    const int64_t C = channels;
    if (overlaps(packed, int64_t(need), Wqkv, C * 3 * C * eb) ||
        overlaps(packed, int64_t(need), Wproj, C * C * eb))
        return NYSTRA_ERR_OVERLAP;
    packed_parts(channels, dtype, &q);
    char *pk = static_cast<char *>(packed);
    clear_stale_error();
    return finish_launch(nystra::launch_block_wpack(Wqkv, Wproj, channels, dtype, pk, pk + q,
                                                    static_cast<hipStream_t>(stream)));
}

int nystra_block_forward_packed(const void *X, const void *Wqkv, const void *bqkv,
                                const void *Wproj, const void *bproj, const void *packed,
                                size_t packed_bytes, void *Y, const nystra_block_shape *shape,
                                int m, int dtype, const nystra_opts *opts, int attention,
                                void *workspace, size_t workspace_bytes, void *stream)
{
    return block_forward(X, Wqkv, bqkv, Wproj, bproj, true, packed, packed_bytes, Y, shape, m,
                         dtype, opts, attention, workspace, workspace_bytes, stream);
}

int nystra_layer_forward(const void *X, const void *Wqkv, const void *bqkv, const void *Wproj,
                         const void *bproj, const void *packed, size_t packed_bytes,
                         const nystra_layer_params *layer, void *Y,
                         const nystra_block_shape *shape, int m, int dtype,
                         const nystra_opts *opts, int attention, void *workspace,
                         size_t workspace_bytes, void *stream)
{
    if (!layer)
        return NYSTRA_ERR_NULL;
    if (!isfinite(layer->eps1) || !isfinite(layer->eps2))
        return NYSTRA_ERR_ARG;
    return block_forward(X, Wqkv, bqkv, Wproj, bproj, true, packed, packed_bytes, Y, shape, m,
                         dtype, opts, attention, workspace, workspace_bytes, stream, layer);
}

}  // extern "C"

namespace {

constexpr int kMaxNormChannels = 4096;

struct Range {
    const void *p;
    int64_t bytes;
};

bool range_hits(const Range &a, const Range &b)
{
    return a.p && b.p && a.bytes > 0 && b.bytes > 0 && overlaps(a.p, a.bytes, b.p, b.bytes);
}

int check_norm(int64_t rows, int channels, int dtype)
{
    if (dtype != NYSTRA_F32 && dtype != NYSTRA_BF16)
        return NYSTRA_ERR_DTYPE;
    if (rows < 0 || rows >= (int64_t(1) << 31) || channels < 1 || channels > kMaxNormChannels)
        return NYSTRA_ERR_SHAPE;
    return NYSTRA_OK;
}

constexpr int64_t kMaxStride = int64_t(1) << 40;

// Elements that a tensor spans at most: more than any memory holds, and its bytes fit 64 bits.
constexpr int64_t kMaxSpan = int64_t(1) << 46;

bool bad_stride(int64_t stride, int64_t least, int64_t rows)
{
    return stride < least || stride > kMaxStride || (rows - 1) > kMaxSpan / stride;
}

int64_t rows_range(int64_t rows, int64_t stride, int channels, int eb)
{
    return rows > 0 ? ((rows - 1) * stride + channels) * eb : 0;
}

// The call of a differential-attention entry point without its tensors.
int diff_problem(const nystra_diff_shape *s, int dtype, nystra::DiffProblem *p)
{
    if (!s)
        return NYSTRA_ERR_NULL;
    if (dtype != NYSTRA_F32 && dtype != NYSTRA_BF16)
        return NYSTRA_ERR_DTYPE;
    if (s->n_windows < 0 || s->kv_heads < 1 || s->heads < s->kv_heads ||
        s->heads % s->kv_heads != 0 || s->n_q < 1 || s->n_q > kMaxN || s->n_k < 1 ||
        s->n_k > kMaxN || s->d_qk < 1 || s->d_qk > 64 || s->d_v < 1 || s->d_v > 128 ||
        int64_t(s->n_windows) * s->heads > kMaxUnits)
        return NYSTRA_ERR_SHAPE;
    if (s->causal < NYSTRA_CAUSAL_NONE || s->causal > NYSTRA_CAUSAL_END || !isfinite(s->scale))
        return NYSTRA_ERR_ARG;
    *p = nystra::DiffProblem{};
    p->W = s->n_windows;
    p->H = s->heads;
    p->G = s->kv_heads;
    p->R = s->heads / s->kv_heads;
    p->nq = s->n_q;
    p->nk = s->n_k;
    p->d = s->d_qk;
    p->dv = s->d_v;
    p->causal = s->causal;
    p->dtype = dtype;
    p->scale = s->scale > 0.f ? s->scale : float(1.0 / sqrt(double(s->d_qk)));
    p->scale2 = float(double(p->scale) * 1.4426950408889634);
    return nystra::diff_grid_fits(*p) ? NYSTRA_OK : NYSTRA_ERR_SHAPE;
}

// One [windows][heads][tokens][width] view: present, aligned, strides in range, and
// for an output no two elements in one place.
int check_view(const nystra_view *v, int64_t windows, int64_t heads, int64_t tokens, int width,
               int eb, bool output, nystra::DiffView *out, Range *range)
{
    if (!v || !v->data)
        return NYSTRA_ERR_NULL;
    if (misaligned(v->data, eb))
        return NYSTRA_ERR_ALIGN;
    const int64_t size[3] = {windows, heads, tokens};
    int64_t stride[3] = {v->window, v->head, v->token};
    int64_t last = width - 1;
    for (int i = 0; i < 3; ++i) {
        if (size[i] == 1)
            stride[i] = 0;   // never stepped over, whatever the caller holds there
        if (stride[i] < 0 || stride[i] > kMaxStride ||
            (stride[i] > 0 && size[i] - 1 > kMaxSpan / stride[i]))
            return NYSTRA_ERR_SHAPE;
        last += (size[i] - 1) * stride[i];
    }
    if (output) {
        // From the smallest stride up, each dimension steps past all of the ones below.
        int64_t extent = width;
        bool done[3] = {};
        for (int n = 0; n < 3; ++n) {
            int at = -1;
            for (int i = 0; i < 3; ++i)
                if (!done[i] && (at < 0 || size[i] == 1 ||
                                 (size[at] != 1 && stride[i] < stride[at])))
                    at = i;
            done[at] = true;
            if (size[at] == 1)
                continue;
            if (stride[at] < extent)
                return NYSTRA_ERR_OVERLAP;
            extent += (size[at] - 1) * stride[at];
        }
    }
    *out = nystra::DiffView{v->data, stride[0], stride[1], stride[2]};
    *range = Range{v->data, (last + 1) * eb};
    return NYSTRA_OK;
}

int check_workspace(void *workspace, size_t bytes, size_t need, const Range *tensors, int n)
{
    if (need == 0)
        return NYSTRA_OK;
    if (!workspace || bytes < need || misaligned(workspace, 256))
        return NYSTRA_ERR_WORKSPACE;
    for (int i = 0; i < n; ++i)
        if (range_hits(Range{workspace, int64_t(need)}, tensors[i]))
            return NYSTRA_ERR_WORKSPACE;
    return NYSTRA_OK;
}

}  // namespace

extern "C" {

int nystra_layer_norm_forward(const void *X, int64_t x_stride, const void *weight,
                              const void *bias, void *Y, int64_t y_stride, float *mean,
                              float *rstd, int64_t rows, int channels, float eps, int dtype,
                              void *stream)
{
    const int rc = check_norm(rows, channels, dtype);
    if (rc != NYSTRA_OK)
        return rc;
    if (!isfinite(eps) || eps < 0.f)
        return NYSTRA_ERR_ARG;
    if (rows == 0)
        return NYSTRA_OK;
    if (!X || !Y || !mean != !rstd)
        return NYSTRA_ERR_NULL;
    if (bad_stride(x_stride, channels, rows) || bad_stride(y_stride, channels, rows))
        return NYSTRA_ERR_SHAPE;
    const int eb = dtype_bytes(dtype);
    if (misaligned(X, eb) || misaligned(Y, eb) || misaligned(weight, eb) || misaligned(bias, eb) ||
        misaligned(mean, 4) || misaligned(rstd, 4))
        return NYSTRA_ERR_ALIGN;
    const Range in[] = {{X, rows_range(rows, x_stride, channels, eb)},
                        {weight, int64_t(channels) * eb}, {bias, int64_t(channels) * eb}};
    const Range out[] = {{Y, rows_range(rows, y_stride, channels, eb)}, {mean, rows * 4},
                         {rstd, rows * 4}};
    for (int i = 0; i < 3; ++i) {
        for (const Range &r : in)
            if (range_hits(out[i], r))
                return NYSTRA_ERR_OVERLAP;
        for (int j = 0; j < i; ++j)
            if (range_hits(out[i], out[j]))
                return NYSTRA_ERR_OVERLAP;
    }
    nystra::NormProblem p{};
    p.x = X;
    p.w = weight;
    p.b = bias;
    p.y = Y;
    p.mean = mean;
    p.rstd = rstd;
    p.rows = rows;
    p.x_stride = x_stride;
    p.y_stride = y_stride;
    p.C = channels;
    p.dtype = dtype;
    p.eps = eps;
    clear_stale_error();
    return finish_launch(nystra::launch_norm_forward(p, static_cast<hipStream_t>(stream)));
}

int nystra_layer_norm_workspace_size(int64_t rows, int channels, size_t *bytes)
{
    if (!bytes)
        return NYSTRA_ERR_NULL;
    const int rc = check_norm(rows, channels, NYSTRA_F32);
    if (rc != NYSTRA_OK)
        return rc;
    *bytes = nystra::norm_workspace_bytes(rows, channels);
    return NYSTRA_OK;
}

int nystra_layer_norm_backward(const void *dY, int64_t dy_stride, const void *X, int64_t x_stride,
                               const void *weight, const float *mean, const float *rstd, void *dX,
                               int64_t dx_stride, void *dweight, void *dbias, int64_t rows,
                               int channels, int dtype, void *workspace, size_t workspace_bytes,
                               void *stream)
{
    int rc = check_norm(rows, channels, dtype);
    if (rc != NYSTRA_OK)
        return rc;
    if (rows > 0 && (!dY || !X || !mean || !rstd || !dX))
        return NYSTRA_ERR_NULL;
    if (rows > 0 &&
        (bad_stride(dy_stride, channels, rows) || bad_stride(x_stride, channels, rows) ||
         bad_stride(dx_stride, channels, rows)))
        return NYSTRA_ERR_SHAPE;
    const int eb = dtype_bytes(dtype);
    for (const void *t : {dY, X, weight, static_cast<const void *>(dX),
                          static_cast<const void *>(dweight), static_cast<const void *>(dbias)})
        if (misaligned(t, eb))
            return NYSTRA_ERR_ALIGN;
    if (misaligned(mean, 4) || misaligned(rstd, 4))
        return NYSTRA_ERR_ALIGN;
    const int64_t cb = int64_t(channels) * eb;
    const Range t[] = {{dX, rows_range(rows, dx_stride, channels, eb)}, {dweight, cb}, {dbias, cb},
                       {dY, rows_range(rows, dy_stride, channels, eb)},
                       {X, rows_range(rows, x_stride, channels, eb)}, {weight, cb},
                       {mean, rows * 4}, {rstd, rows * 4}};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 8; ++j)
            if (range_hits(t[i], t[j]))
                return NYSTRA_ERR_OVERLAP;
    rc = check_workspace(workspace, workspace_bytes, nystra::norm_workspace_bytes(rows, channels),
                         t, 8);
    if (rc != NYSTRA_OK)
        return rc;
    if (rows == 0 && !dweight && !dbias)
        return NYSTRA_OK;
    nystra::NormProblem p{};
    p.x = X;
    p.w = weight;
    p.dy = dY;
    p.dx = dX;
    p.mean = const_cast<float *>(mean);
    p.rstd = const_cast<float *>(rstd);
    p.rows = rows;
    p.x_stride = x_stride;
    p.dy_stride = dy_stride;
    p.dx_stride = dx_stride;
    p.C = channels;
    p.dtype = dtype;
    clear_stale_error();
    return finish_launch(nystra::launch_norm_backward(p, dweight, dbias,
                                                      static_cast<float *>(workspace),
                                                      static_cast<hipStream_t>(stream)));
}

int nystra_dropout(const void *X, const void *residual, void *Y, int64_t n, float p,
                   uint64_t seed, uint64_t offset, const uint64_t *state, int dtype, void *stream)
{
    if (dtype != NYSTRA_F32 && dtype != NYSTRA_BF16)
        return NYSTRA_ERR_DTYPE;
    if (n < 0 || n > (int64_t(1) << 34))
        return NYSTRA_ERR_SHAPE;
    if (!(p >= 0.f && p <= 1.f))
        return NYSTRA_ERR_ARG;
    if (n == 0)
        return NYSTRA_OK;
    if (!X || !Y)
        return NYSTRA_ERR_NULL;
    const int eb = dtype_bytes(dtype);
    if (misaligned(X, eb) || misaligned(residual, eb) || misaligned(Y, eb) || misaligned(state, 8))
        return NYSTRA_ERR_ALIGN;
    const Range y{Y, n * eb};
    if ((X != Y && range_hits(y, Range{X, n * eb})) ||
        (residual != Y && range_hits(y, Range{residual, n * eb})) ||
        range_hits(y, Range{state, 16}))
        return NYSTRA_ERR_OVERLAP;
    nystra::DropProblem d;
    d.x = X;
    d.residual = residual;
    d.y = Y;
    d.n = n;
    d.seed = seed;
    d.offset = offset;
    d.state = state;
    d.threshold = uint32_t(floor(double(p) * 65536.0 + 0.5));
    d.scale = d.threshold < 65536u ? float(65536.0 / (65536.0 - d.threshold)) : 0.f;
    d.dtype = dtype;
    clear_stale_error();
    return finish_launch(nystra::launch_dropout(d, static_cast<hipStream_t>(stream)));
}

int nystra_diff_attn_workspace_size(const nystra_diff_shape *shape, int backward, int dtype,
                                    size_t *bytes)
{
    if (!bytes)
        return NYSTRA_ERR_NULL;
    nystra::DiffProblem p;
    const int rc = diff_problem(shape, dtype, &p);
    if (rc != NYSTRA_OK)
        return rc;
    *bytes = p.W == 0    ? 0
             : backward ? nystra::diff_backward_workspace(p)
                        : nystra::diff_forward_workspace(p);
    return NYSTRA_OK;
}

int nystra_diff_attn_forward(const nystra_view *Q, const nystra_view *K, const nystra_view *V,
                             const float *lambda, const int32_t *kv_len, const nystra_view *O,
                             float *maps, float *sums, const nystra_diff_shape *shape, int dtype,
                             void *workspace, size_t workspace_bytes, void *stream)
{
    nystra::DiffProblem p;
    int rc = diff_problem(shape, dtype, &p);
    if (rc != NYSTRA_OK)
        return rc;
    if (p.W == 0)
        return NYSTRA_OK;
    const int eb = dtype_bytes(dtype);
    Range t[8] = {};   // O, maps, sums, then the inputs
    if ((rc = check_view(O, p.W, p.H, p.nq, p.dv, eb, true, &p.o, &t[0])) != NYSTRA_OK ||
        (rc = check_view(Q, p.W, 2 * p.H, p.nq, p.d, eb, false, &p.q, &t[3])) != NYSTRA_OK ||
        (rc = check_view(K, p.W, 2 * p.G, p.nk, p.d, eb, false, &p.k, &t[4])) != NYSTRA_OK ||
        (rc = check_view(V, p.W, p.G, p.nk, p.dv, eb, false, &p.v, &t[5])) != NYSTRA_OK)
        return rc;
    if (!lambda)
        return NYSTRA_ERR_NULL;
    if (misaligned(maps, 16) || misaligned(sums, 8) || misaligned(lambda, 4) ||
        misaligned(kv_len, 4))
        return NYSTRA_ERR_ALIGN;
    if ((maps && !sums) || (sums && (maps != nullptr) != nystra::diff_keeps_maps(p)))
        return NYSTRA_ERR_NULL;
    const int64_t rows = int64_t(p.W) * p.H * p.nq;
    t[1] = Range{maps, rows * p.dv * (eb == 2 ? 8 : 4)};
    t[2] = Range{sums, rows * 16};
    t[6] = Range{lambda, int64_t(p.H) * 4};
    t[7] = Range{kv_len, int64_t(p.W) * 4};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 8; ++j)
            if (range_hits(t[i], t[j]))
                return NYSTRA_ERR_OVERLAP;
    rc = check_workspace(workspace, workspace_bytes, nystra::diff_forward_workspace(p), t, 8);
    if (rc != NYSTRA_OK)
        return rc;
    p.maps = maps;
    p.sums = sums;
    p.lambda = lambda;
    p.kv_len = kv_len;
    clear_stale_error();
    return finish_launch(
        nystra::launch_diff_forward(p, workspace, static_cast<hipStream_t>(stream)));
}

int nystra_diff_attn_backward(const nystra_view *dO, const nystra_view *Q, const nystra_view *K,
                              const nystra_view *V, const float *lambda, const int32_t *kv_len,
                              const nystra_view *O, const float *maps, const float *sums,
                              const nystra_view *dQ, const nystra_view *dK, const nystra_view *dV,
                              float *dlambda, const nystra_diff_shape *shape, int dtype,
                              void *workspace, size_t workspace_bytes, void *stream)
{
    nystra::DiffProblem p;
    int rc = diff_problem(shape, dtype, &p);
    if (rc != NYSTRA_OK)
        return rc;
    if (!dlambda)
        return NYSTRA_ERR_NULL;
    if (misaligned(dlambda, 4))
        return NYSTRA_ERR_ALIGN;
    if (p.W > 0) {
        const int eb = dtype_bytes(dtype);
        const int64_t rows = int64_t(p.W) * p.H * p.nq;
        Range t[13] = {};   // dQ, dK, dV, dlambda, then the inputs
        if ((rc = check_view(dQ, p.W, 2 * p.H, p.nq, p.d, eb, true, &p.gq, &t[0])) != NYSTRA_OK ||
            (rc = check_view(dK, p.W, 2 * p.G, p.nk, p.d, eb, true, &p.gk, &t[1])) != NYSTRA_OK ||
            (rc = check_view(dV, p.W, p.G, p.nk, p.dv, eb, true, &p.gv, &t[2])) != NYSTRA_OK ||
            (rc = check_view(dO, p.W, p.H, p.nq, p.dv, eb, false, &p.go, &t[4])) != NYSTRA_OK ||
            (rc = check_view(Q, p.W, 2 * p.H, p.nq, p.d, eb, false, &p.q, &t[5])) != NYSTRA_OK ||
            (rc = check_view(K, p.W, 2 * p.G, p.nk, p.d, eb, false, &p.k, &t[6])) != NYSTRA_OK ||
            (rc = check_view(V, p.W, p.G, p.nk, p.dv, eb, false, &p.v, &t[7])) != NYSTRA_OK ||
            (rc = check_view(O, p.W, p.H, p.nq, p.dv, eb, false, &p.o, &t[8])) != NYSTRA_OK)
            return rc;
        if (!lambda || !sums || (maps != nullptr) != nystra::diff_keeps_maps(p))
            return NYSTRA_ERR_NULL;
        if (misaligned(maps, 16) || misaligned(sums, 8) || misaligned(lambda, 4) ||
            misaligned(kv_len, 4))
            return NYSTRA_ERR_ALIGN;
        t[3] = Range{dlambda, int64_t(p.H) * 4};
        t[9] = Range{maps, rows * p.dv * (eb == 2 ? 8 : 4)};
        t[10] = Range{sums, rows * 16};
        t[11] = Range{lambda, int64_t(p.H) * 4};
        t[12] = Range{kv_len, int64_t(p.W) * 4};
        for (int i = 0; i < 4; ++i)
            for (int j = 3; j < 13; ++j)   // dQ, dK and dV may share a buffer
                if (i != j && range_hits(t[i], t[j]))
                    return NYSTRA_ERR_OVERLAP;
        rc = check_workspace(workspace, workspace_bytes, nystra::diff_backward_workspace(p), t,
                             13);
        if (rc != NYSTRA_OK)
            return rc;
    }
    p.maps = const_cast<float *>(maps);
    p.glam = dlambda;
    p.sums = const_cast<float *>(sums);
    p.lambda = lambda;
    p.kv_len = kv_len;
    clear_stale_error();
    return finish_launch(nystra::launch_diff_backward(p, workspace,
                                                      static_cast<hipStream_t>(stream)));
}

const char *nystra_status_str(int status)
{
    switch (status) {
    case NYSTRA_OK: return "ok";
    case NYSTRA_ERR_NULL: return "null pointer";
    case NYSTRA_ERR_SHAPE: return "shape out of range or no pooling grid";
    case NYSTRA_ERR_DTYPE: return "unsupported dtype";
    case NYSTRA_ERR_ALIGN: return "misaligned pointer";
    case NYSTRA_ERR_OVERLAP: return "output overlaps an input";
    case NYSTRA_ERR_UNSUPPORTED: return "forced kernel variant cannot run this shape";
    case NYSTRA_ERR_HIP: return "HIP launch error";
    case NYSTRA_ERR_ARG: return "invalid argument";
    case NYSTRA_ERR_WORKSPACE: return "workspace missing, too small or misaligned";
    default: return "unknown status";
    }
}

const char *nystra_last_error(void) { return g_last_error; }

}  // extern "C"
