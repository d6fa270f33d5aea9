// LayerNorm over the channels of a list of rows, forward and backward.
//
//   forward   mean = sum x / C, var = sum (x - mean)^2 / C, rstd = (var + eps)^-1/2,
//             y = (x - mean) rstd w + b
//   backward  g = dy w, xh = (x - mean) rstd,
//             dx = rstd (g - sum(g) / C - xh sum(g xh) / C),
//             dw = sum over rows of dy xh, db = sum over rows of dy
//
// Both passes are bound by memory: x is read and y written once (x and dy read,
// dx written), so a row lives in the registers of the LPR lanes that share it,
// at most 16 values a lane, and the sums are taken over registers: first the
// mean, then the squares of the differences, which loses nothing where the mean
// is large against the deviation.  All sums are fp32.
//
// dw and db: a workgroup walks over many rows and each lane keeps the sums of
// its own columns; the workgroup's sums go to the workspace, and a second
// launch adds them up, always in the same order (no atomics).
//
// Measured: 65536 rows of 180 in bf16, forward 12.7 us (47 MB, 3.7 TB/s), backward 15.2 us
// (71 MB, 4.7 TB/s) and 4.0 us for the second launch; 20011 rows of 1021 in fp32, which no
// wide load fits, 27 us (163 MB, 6.0 TB/s), 44 us (245 MB, 5.6 TB/s) and 7.9 us, on
// inputs that the Infinity Cache may hold.
#include "device_common.hpp"
#include "internal.hpp"
#include "tile_common.hpp"

namespace nystra {
namespace {

constexpr int kThreads = 256;

// VEC consecutive elements as they lie in memory; the address is aligned to all of them.
template <class E, int VEC>
struct Raw {
    typedef typename E::T V __attribute__((ext_vector_type(VEC)));
    V v;
};

template <class E>
struct Raw<E, 1> {
    typename E::T v;
};

template <class E, int VEC>
__device__ inline Raw<E, VEC> load_raw(const typename E::T *p)
{
    return Raw<E, VEC>{*reinterpret_cast<const decltype(Raw<E, VEC>::v) *>(p)};
}

template <class E, int VEC>
__device__ inline void unpack(const Raw<E, VEC> &r, float (&x)[VEC])
{
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        typename E::T e;
        if constexpr (VEC == 1)
            e = r.v;
        else
            e = r.v[j];
        if constexpr (E::bytes == 4)
            x[j] = e;
        else
            x[j] = bf16_to_f32(e);
    }
}

template <class E, int VEC>
__device__ inline void load_vec(const typename E::T *p, float (&x)[VEC])
{
    unpack<E, VEC>(load_raw<E, VEC>(p), x);
}

template <class E, int VEC>
__device__ inline void store_vec(typename E::T *p, const float (&x)[VEC])
{
    typedef typename E::T V __attribute__((ext_vector_type(VEC)));
    if constexpr (VEC == 1) {
        E::store(p, 0, x[0]);
    } else {
        if constexpr (E::bytes == 4) {
            V v;
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                v[j] = x[j];
            *reinterpret_cast<V *>(p) = v;
        } else {
            typedef float FV __attribute__((ext_vector_type(VEC)));
            typedef __bf16 BV __attribute__((ext_vector_type(VEC)));
            FV v;
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                v[j] = x[j];
            *reinterpret_cast<BV *>(p) = __builtin_convertvector(v, BV);   // to nearest even
        }
    }
}

// Sums over the LPR lanes of a row, by lane exchanges inside the VALU.  Rows of a whole
// workgroup go through LDS.
template <int LPR, int N>
__device__ inline void row_sums(float (&s)[N], float *lds)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        s[i] = tile::sum_row(s[i]);
        if constexpr (LPR >= 64)
            s[i] = tile::sum_groups(s[i]);
    }
    if constexpr (LPR > 64) {
        constexpr int W = LPR / 64;
        const int wave = threadIdx.x >> 6;
        __syncthreads();
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i)
                lds[wave * N + i] = s[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s[i] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w)
                s[i] += lds[w * N + i];
        }
    }
}

// A lane's part of one row: column (c LPR + lane) VEC of chunk c.  Lanes behind the row load
// its start again; what they hold is dropped where it is used.
template <class E, int VEC, int LPR, int CH>
__device__ inline void load_row(const typename E::T *row, int C, Raw<E, VEC> (&x)[CH])
{
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * LPR + threadIdx.x % LPR) * VEC;
        x[c] = load_raw<E, VEC>(row + (col < C ? col : 0));
    }
}

// Workgroup `blockIdx.x` takes the row groups blockIdx.x, + gridDim.x, ..., the next one's
// loads ahead of the work on one, with weight and bias in registers.
template <class E, int VEC, int LPR, int CH>
__global__ void __launch_bounds__(kThreads)
norm_forward_kernel(NormProblem p)
{
    using T = typename E::T;
    __shared__ float lds[8];
    constexpr int kRows = kThreads / LPR;
    const int lane = threadIdx.x % LPR;
    float w[CH][VEC], b[CH][VEC];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * LPR + lane) * VEC;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            w[c][j] = 1.f;
            b[c][j] = 0.f;
        }
        if (p.w && col < p.C)
            load_vec<E, VEC>(static_cast<const T *>(p.w) + col, w[c]);
        if (p.b && col < p.C)
            load_vec<E, VEC>(static_cast<const T *>(p.b) + col, b[c]);
    }
    const int64_t step = int64_t(gridDim.x) * kRows;
    int64_t row = int64_t(blockIdx.x) * kRows + threadIdx.x / LPR;
    const float inv = 1.f / float(p.C);
    Raw<E, VEC> next[CH];
    const T *x = static_cast<const T *>(p.x);
    load_row<E, VEC, LPR, CH>(x + (row < p.rows ? row : 0) * p.x_stride, p.C, next);
    for (int64_t r0 = int64_t(blockIdx.x) * kRows; r0 < p.rows; r0 += step, row += step) {
        float v[CH][VEC];
        float s[1] = {0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const bool in = (c * LPR + lane) * VEC < p.C;
            unpack<E, VEC>(next[c], v[c]);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                v[c][j] = in ? v[c][j] : 0.f;
                s[0] += v[c][j];
            }
        }
        if (r0 + step < p.rows)
            load_row<E, VEC, LPR, CH>(x + (row + step < p.rows ? row + step : 0) * p.x_stride,
                                      p.C, next);
        row_sums<LPR>(s, lds);
        const float mean = s[0] / float(p.C);   // divided: equal values have no deviation
        s[0] = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const bool in = (c * LPR + lane) * VEC < p.C;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                v[c][j] = in ? v[c][j] - mean : 0.f;
                s[0] = fmaf(v[c][j], v[c][j], s[0]);
            }
        }
        row_sums<LPR>(s, lds);
        const float rstd = 1.f / sqrtf(s[0] * inv + p.eps);
        if (row < p.rows) {
            T *y = static_cast<T *>(p.y) + row * p.y_stride;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = (c * LPR + lane) * VEC;
                if (col < p.C) {
#pragma unroll
                    for (int j = 0; j < VEC; ++j)
                        v[c][j] = fmaf(v[c][j] * rstd, w[c][j], b[c][j]);
                    store_vec<E, VEC>(y + col, v[c]);
                }
            }
            if (lane == 0 && p.mean) {
                p.mean[row] = mean;
                p.rstd[row] = rstd;
            }
        }
    }
}

// Workgroup `blockIdx.x` takes the row groups blockIdx.x, + gridDim.x, ...; its
// column sums go to partial[blockIdx.x][2][C].
template <class E, int VEC, int LPR, int CH>
__global__ void __launch_bounds__(kThreads)
norm_backward_kernel(NormProblem p, float *partial)
{
    using T = typename E::T;
    constexpr int kRows = kThreads / LPR;
    constexpr int kCols = LPR * CH * VEC;
    __shared__ float lds[8];
    __shared__ float sums[LPR < 256 ? 2 * kCols : 1];
    const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
    float w[CH][VEC], aw[CH][VEC], ab[CH][VEC];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * LPR + lane) * VEC;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            w[c][j] = 1.f;
            aw[c][j] = ab[c][j] = 0.f;
        }
        if (p.w && col < p.C)
            load_vec<E, VEC>(static_cast<const T *>(p.w) + col, w[c]);
    }
    // The rows are fetched one ahead: with few rows to a workgroup it is the latency of
    // their loads that bounds it.
    const float inv = 1.f / float(p.C);
    const int64_t step = int64_t(gridDim.x) * kRows;
    int64_t row = int64_t(blockIdx.x) * kRows + group;
    Raw<E, VEC> xn[CH], gn[CH];
    float mean_n = 0.f, rstd_n = 0.f;
    auto fetch = [&](int64_t r) {
        const int64_t rr = r < p.rows ? r : 0;
        const T *x = static_cast<const T *>(p.x) + rr * p.x_stride;
        const T *dy = static_cast<const T *>(p.dy) + rr * p.dy_stride;
        mean_n = p.mean[rr];
        rstd_n = p.rstd[rr];
        load_row<E, VEC, LPR, CH>(x, p.C, xn);
        load_row<E, VEC, LPR, CH>(dy, p.C, gn);
    };
    fetch(row);
    for (int64_t r0 = int64_t(blockIdx.x) * kRows; r0 < p.rows; r0 += step, row += step) {
        const bool live = row < p.rows;
        const float mean = mean_n, rstd = rstd_n;
        float xh[CH][VEC], g[CH][VEC];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const bool in = live && (c * LPR + lane) * VEC < p.C;
            unpack<E, VEC>(xn[c], xh[c]);
            unpack<E, VEC>(gn[c], g[c]);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                xh[c][j] = in ? (xh[c][j] - mean) * rstd : 0.f;
                g[c][j] = in ? g[c][j] : 0.f;
            }
        }
        if (r0 + step < p.rows)
            fetch(row + step);
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                aw[c][j] = fmaf(g[c][j], xh[c][j], aw[c][j]);
                ab[c][j] += g[c][j];
                g[c][j] *= w[c][j];
                s[0] += g[c][j];
                s[1] = fmaf(g[c][j], xh[c][j], s[1]);
            }
        row_sums<LPR>(s, lds);
        const float m0 = s[0] * inv, m1 = s[1] * inv;
        if (live) {
            T *dx = static_cast<T *>(p.dx) + row * p.dx_stride;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = (c * LPR + lane) * VEC;
                if (col < p.C) {
#pragma unroll
                    for (int j = 0; j < VEC; ++j)
                        g[c][j] = rstd * (g[c][j] - m0 - xh[c][j] * m1);
                    store_vec<E, VEC>(dx + col, g[c]);
                }
            }
        }
    }
    float *out = partial + int64_t(blockIdx.x) * 2 * p.C;
    if constexpr (LPR < 256) {
        // The groups of one wave by shuffles, then the four waves in turn.
#pragma unroll
        for (int o = LPR; o < 64; o <<= 1)
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    aw[c][j] += __shfl_xor(aw[c][j], o, 64);
                    ab[c][j] += __shfl_xor(ab[c][j], o, 64);
                }
        for (int wave = 0; wave < kThreads / 64; ++wave) {
            if (int(threadIdx.x >> 6) == wave && (threadIdx.x & 63) < LPR) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const int at = (c * LPR + lane) * VEC + j;
                        sums[at] = (wave ? sums[at] : 0.f) + aw[c][j];
                        sums[kCols + at] = (wave ? sums[kCols + at] : 0.f) + ab[c][j];
                    }
            }
            __syncthreads();
        }
        for (int i = threadIdx.x; i < p.C; i += kThreads) {
            out[i] = sums[i];
            out[p.C + i] = sums[kCols + i];
        }
    } else {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int col = (c * LPR + lane) * VEC + j;
                if (col < p.C) {
                    out[col] = aw[c][j];
                    out[p.C + col] = ab[c][j];
                }
            }
    }
}

// Column sums of partial[n][2C]: eight columns to a workgroup, whose threads take every
// 128th partial sum.
constexpr int kReduce = 1024;

template <class E>
__global__ void __launch_bounds__(kReduce)
norm_reduce_kernel(const float *__restrict__ partial, int n, int C, typename E::T *dw,
                   typename E::T *db)
{
    __shared__ float lds[kReduce / 8][9];
    const int col = blockIdx.x * 8 + threadIdx.x % 8, part = threadIdx.x / 8;
    float s = 0.f;
    if (col < 2 * C) {
#pragma unroll 8
        for (int i = part; i < n; i += kReduce / 8)
            s += partial[int64_t(i) * 2 * C + col];
    }
    lds[part][threadIdx.x % 8] = s;
    for (int half = kReduce / 16; half >= 1; half /= 2) {
        __syncthreads();
        if (part < half)
            lds[part][threadIdx.x % 8] += lds[part + half][threadIdx.x % 8];
    }
    if (part == 0 && col < 2 * C) {
        s = lds[0][threadIdx.x];
        if (col < C) {
            if (dw)
                E::store(dw, col, s);
        } else if (db) {
            E::store(db, col - C, s);
        }
    }
}

int lanes_per_row(int C) { return C <= 256 ? 16 : C <= 1024 ? 64 : 256; }

int backward_groups(int64_t rows, int C)
{
    const int64_t per = kThreads / lanes_per_row(C);
    const int64_t blocks = (rows + per - 1) / per;
    return int(blocks < 1024 ? blocks : 1024);
}

// Elements to one load: a whole 16 or 8 bytes where every row of every tensor
// starts and ends on such a boundary, one element otherwise.
int vector_width(const NormProblem &p, int bytes)
{
    for (int vec = 16 / bytes; vec > 1; vec /= 2) {
        const uintptr_t a = uintptr_t(p.x) | uintptr_t(p.y) | uintptr_t(p.dy) | uintptr_t(p.dx) |
                            uintptr_t(p.w) | uintptr_t(p.b);
        const int64_t n = p.C | p.x_stride | p.y_stride | p.dy_stride | p.dx_stride;
        if (a % (vec * bytes) == 0 && n % vec == 0)
            return vec;
        if (vec * bytes == 8)
            break;
    }
    return 1;
}

template <class E, int VEC, int LPR, int EPL>
void launch(const NormProblem &p, float *partial, int groups, hipStream_t s)
{
    constexpr int CH = EPL / VEC;
    if (partial) {
        norm_backward_kernel<E, VEC, LPR, CH><<<groups, kThreads, 0, s>>>(p, partial);
    } else {
        // At most eight workgroups to a CU.
        const int64_t per = kThreads / LPR, blocks = (p.rows + per - 1) / per;
        norm_forward_kernel<E, VEC, LPR, CH>
            <<<dim3(unsigned(blocks < 2048 ? blocks : 2048)), kThreads, 0, s>>>(p);
    }
}

// A lane holds 8, 12 or 16 values, the fewest that do (12 not of wide loads, which they
// cannot be made of).
template <class E, int VEC, int LPR>
void launch_lanes(const NormProblem &p, float *partial, int groups, hipStream_t s)
{
    if (p.C <= 8 * LPR)
        return launch<E, VEC, LPR, 8>(p, partial, groups, s);
    if constexpr (12 % VEC == 0) {
        if (p.C <= 12 * LPR)
            return launch<E, VEC, LPR, 12>(p, partial, groups, s);
    }
    launch<E, VEC, LPR, 16>(p, partial, groups, s);
}

// At most 16 values a lane: 16 lanes hold a row of up to 256 channels (four
// rows to a wave), a wave up to 1024, a workgroup up to 4096.
template <class E, int VEC>
void launch_vec(const NormProblem &p, float *partial, int groups, hipStream_t s)
{
    const int lanes = lanes_per_row(p.C);
    if (lanes == 16)
        launch_lanes<E, VEC, 16>(p, partial, groups, s);
    else if (lanes == 64)
        launch_lanes<E, VEC, 64>(p, partial, groups, s);
    else
        launch_lanes<E, VEC, 256>(p, partial, groups, s);
}

void launch_any(const NormProblem &p, float *partial, int groups, hipStream_t s)
{
    if (p.dtype == 0) {
        switch (vector_width(p, 4)) {
        case 4: return launch_vec<F32, 4>(p, partial, groups, s);
        case 2: return launch_vec<F32, 2>(p, partial, groups, s);
        default: return launch_vec<F32, 1>(p, partial, groups, s);
        }
    }
    switch (vector_width(p, 2)) {
    case 8: return launch_vec<BF16, 8>(p, partial, groups, s);
    case 4: return launch_vec<BF16, 4>(p, partial, groups, s);
    default: return launch_vec<BF16, 1>(p, partial, groups, s);
    }
}

}  // namespace

size_t norm_workspace_bytes(int64_t rows, int C)
{
    return size_t(backward_groups(rows, C)) * 2 * size_t(C) * sizeof(float);
}

hipError_t launch_norm_forward(const NormProblem &p, hipStream_t s)
{
    launch_any(p, nullptr, 0, s);
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormProblem &p, void *dw, void *db, float *workspace,
                                hipStream_t s)
{
    const int groups = backward_groups(p.rows, p.C);
    if (groups > 0) {
        launch_any(p, workspace, groups, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    if (dw || db) {
        const int blocks = (2 * p.C + 7) / 8;
        if (p.dtype == 0)
            norm_reduce_kernel<F32><<<blocks, kReduce, 0, s>>>(
                workspace, groups, p.C, static_cast<float *>(dw), static_cast<float *>(db));
        else
            norm_reduce_kernel<BF16><<<blocks, kReduce, 0, s>>>(
                workspace, groups, p.C, static_cast<uint16_t *>(dw), static_cast<uint16_t *>(db));
    }
    return hipGetLastError();
}

}  // namespace nystra
