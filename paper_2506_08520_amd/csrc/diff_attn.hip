// Differential attention: the difference of two softmax maps over one set of
// values, with a learned weight per head,
//   S_a = s Q_a K_a^T (a = 1, 2),  P_a = softmax of S_a over the visible keys,
//   O = (P_1 - lam P_2) V,
// and its backward pass, with X = dO V^T and D_a = rowsum(P_a X):
//   dS_1 = P_1 (X - D_1),  dS_2 = -lam P_2 (X - D_2),
//   dQ_a = s dS_a K_a,  dK_a = s dS_a^T Q_a,  dV = (P_1 - lam P_2)^T dO,
//   dlam = -sum over rows of D_2.
//
// A "unit" is a window and a key/value head; its rows are the queries of all R
// query heads that share those keys, head after head (R n_q rows), so that a
// single token of grouped heads still fills a tile.  One wave owns 32 rows (in
// the dK, dV kernel 32 keys) and walks the other axis in tiles of 32 through
// LDS.  Scores are formed transposed, S^T = K Q^T, so that a lane column is a
// query: the running maximum and sum stay in the lane, and the probabilities
// are the right-hand operand of O^T += V^T P^T as they stand.
//
// Fragments.  A 32 x 32 product over 16 contraction indices takes from lane
// (g = lane / 32, c = lane % 32) eight values of row c of the left operand and
// of column c of the right one, and returns D[8 (r / 4) + 4 g + r % 4][c] in
// register r.  Which index a slot stands for is free as long as both operands
// agree: operands read along rows (row_frag) use 8 g + j, those that meet a
// product's result (col_frag) use that result's order, 8 (j / 4) + 4 g + j % 4.
// bf16 runs it as one matrix instruction, fp32 as eight of depth two.
#include "device_common.hpp"
#include "internal.hpp"

namespace nystra {
namespace {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));

constexpr int kMerge = 64;   // threads of the merge kernel: one row

template <class E>
struct Frag;

template <>
struct Frag<BF16> {
    bf8 x;
};

template <>
struct Frag<F32> {
    float x[8];
};

__device__ inline f16v mma(const Frag<BF16> &a, const Frag<BF16> &b, f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.x, b.x, c, 0, 0, 0);
}

__device__ inline f16v mma(const Frag<F32> &a, const Frag<F32> &b, f16v c)
{
#pragma unroll
    for (int j = 0; j < 8; ++j)
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x[j], b.x[j], c, 0, 0, 0);
    return c;
}

// Eight consecutive elements as they lie in memory.
template <class E>
struct alignas(16) Chunk {
    uint32_t w[2 * E::bytes];
};

// Elements 0..n-1 of eight (n may be <= 0 or above 8), the others zero, by loads of `vec`
// bytes: the row's first element and width are multiples of that many bytes.
template <class E>
__device__ inline Chunk<E> load_chunk(const typename E::T *p, int n, int vec)
{
    Chunk<E> c = {};
    if (vec == 16) {
        constexpr int per = 16 / E::bytes;
#pragma unroll
        for (int h = 0; h < 8 / per; ++h)
            if (h * per < n)
                *reinterpret_cast<uint4 *>(&c.w[4 * h]) =
                    *reinterpret_cast<const uint4 *>(p + h * per);
    } else if (vec == 4 || E::bytes == 4) {
        constexpr int per = 4 / E::bytes;
#pragma unroll
        for (int h = 0; h < 8 / per; ++h)
            if (h * per < n)
                c.w[h] = *reinterpret_cast<const uint32_t *>(p + h * per);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n)
                c.w[j * E::bytes / 4] |= uint32_t(*reinterpret_cast<const uint16_t *>(p + j))
                                         << (16 * (j & 1));
    }
    return c;
}

template <class E>
__device__ inline Frag<E> as_frag(const Chunk<E> &c)
{
    return __builtin_bit_cast(Frag<E>, c);
}

__device__ inline Frag<BF16> frag_of(const f16v &s, int c, BF16)
{
    typedef float f8 __attribute__((ext_vector_type(8)));
    f8 v;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        v[j] = s[8 * c + j];
    return Frag<BF16>{__builtin_convertvector(v, bf8)};   // to nearest even
}

__device__ inline Frag<F32> frag_of(const f16v &s, int c, F32)
{
    Frag<F32> f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        f.x[j] = s[8 * c + j];
    return f;
}

// Row lane % 32 of a tile in LDS, contraction indices (columns) 16 c + 8 g + j.
template <class E>
__device__ inline Frag<E> row_frag(const typename E::T *tile, int pitch, int c)
{
    const int lane = threadIdx.x & 63;
    return as_frag<E>(*reinterpret_cast<const Chunk<E> *>(
        tile + (lane & 31) * pitch + 16 * c + 8 * (lane >> 5)));
}

// Column col0 + lane % 32 of a tile, contraction indices (rows) in the order of a
// product's result: 16 c + 8 (j / 4) + 4 g + j % 4.  In bf16 the transposing LDS
// read takes four rows of 16 columns from 16 lanes (lane p: row p / 4, columns
// 4 (p % 4) ..) and gives each lane its column of them.
template <class E>
__device__ inline Frag<E> col_frag(const typename E::T *tile, int pitch, int c, int col0)
{
    const int lane = threadIdx.x & 63, g = lane >> 5;
    if constexpr (E::bytes == 2) {
        typedef __attribute__((address_space(3))) s4 ls4;
        const int row = 16 * c + 4 * g + ((lane & 15) >> 2);
        const int col = col0 + (lane & 16) + 4 * (lane & 3);
        const uint16_t *p = tile + row * pitch + col;
        struct {
            s4 lo, hi;
        } v;
        v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ls4 *)(p));
        v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ls4 *)(p + 8 * pitch));
        return __builtin_bit_cast(Frag<BF16>, v);
    } else {
        Frag<F32> f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            f.x[j] = tile[(16 * c + 8 * (j >> 2) + 4 * g + (j & 3)) * pitch + col0 + (lane & 31)];
        return f;
    }
}

// Row pitches in LDS.  Tiles read along rows are 16 bytes longer than their
// width, so that eight rows' 16-byte reads fall on different banks.
template <class E>
constexpr int pitch_of(int cols) { return cols + 16 / E::bytes; }

// `rows` x `COLS` elements of a tensor into LDS, zero outside its `valid` rows and
// `cols` columns.
template <class E, int COLS, int ROWS>
__device__ inline void stage(typename E::T *lds, int pitch, const typename E::T *src,
                             int64_t stride, int valid, int cols, int vec)
{
    constexpr int kChunks = COLS / 8;
    for (int i = threadIdx.x; i < ROWS * kChunks; i += blockDim.x) {
        const int row = i / kChunks, c = i % kChunks;
        const Chunk<E> x = load_chunk<E>(src + (row < valid ? row : 0) * stride + 8 * c,
                                         row < valid ? cols - 8 * c : 0, vec);
        *reinterpret_cast<Chunk<E> *>(lds + row * pitch + 8 * c) = x;
    }
}

__device__ inline float other_half(float x)
{
    return __shfl_xor(x, 32, 64);
}

// Position of a row of the unit: its query head and token.
struct Row {
    int head, token;
};

__device__ inline Row row_of(const DiffProblem &p, int g, int r)
{
    const int hh = r / p.nq;
    return Row{g * p.R + hh, r - hh * p.nq};
}

// Keys that a query token sees: those below the returned index.
__device__ inline int key_limit(const DiffProblem &p, int len, int token)
{
    if (p.causal == 0)
        return len;
    const int n = p.causal == 1 ? token + 1 : len - p.nq + token + 1;
    return n < 0 ? 0 : n < len ? n : len;
}

__device__ inline int window_len(const DiffProblem &p, int w)
{
    if (!p.kv_len)
        return p.nk;
    const int n = p.kv_len[w];
    return n < 0 ? 0 : n < p.nk ? n : p.nk;
}

// Keys that the rows r0 .. r1 see at most: the limit grows with the token, and
// rows of several heads hold the last token of the first one.
__device__ inline int tile_limit(const DiffProblem &p, int len, int r0, int r1)
{
    if (r0 / p.nq != r1 / p.nq)
        return key_limit(p, len, p.nq - 1);
    return key_limit(p, len, r1 % p.nq);
}

template <class E>
__device__ inline const typename E::T *at(const DiffView &v, int64_t w, int64_t head, int64_t token)
{
    return static_cast<const typename E::T *>(v.data) + w * v.window + head * v.head +
           token * v.token;
}

template <class E>
__device__ inline typename E::T *at_out(const DiffView &v, int64_t w, int64_t head, int64_t token)
{
    return static_cast<typename E::T *>(v.data) + w * v.window + head * v.head + token * v.token;
}

// Four consecutive elements of an output row from column `col`, those below `n`; `vec`
// says that such groups are whole and aligned.
template <class E>
__device__ inline void store4(typename E::T *row, int col, int n, bool vec, float a, float b,
                              float c, float d)
{
    if (vec) {
        if (col < n) {
            if constexpr (E::bytes == 4) {
                *reinterpret_cast<float4 *>(row + col) = make_float4(a, b, c, d);
            } else {
                ushort4 u;
                u.x = f32_to_bf16(a);
                u.y = f32_to_bf16(b);
                u.z = f32_to_bf16(c);
                u.w = f32_to_bf16(d);
                *reinterpret_cast<ushort4 *>(row + col) = u;
            }
        }
        return;
    }
    const float x[4] = {a, b, c, d};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (col + j < n)
            E::store(row, col + j, x[j]);
}

// The transposed tile's register r: its row.
__device__ inline int reg_row(int r, int g) { return 8 * (r >> 2) + 4 * g + (r & 3); }

// Online softmax of a 32 x 32 tile of S^T: s becomes exp2(scale2 s - m), l the
// running sum of this lane's keys, and the return value the factor for what was
// summed before.
__device__ inline float softmax_step(f16v &s, float scale2, float &m, float &l, int limit,
                                     int k0, int g, bool masked)
{
    if (masked) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
            s[r] = k0 + reg_row(r, g) < limit ? s[r] : -INFINITY;
    }
    float t = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r)
        t = fmaxf(t, s[r]);
    t = fmaxf(t, other_half(t)) * scale2;
    const float mn = fmaxf(m, t);
    // A row that has seen no key yet has nothing to subtract.
    const float base = mn == -INFINITY ? 0.f : mn;
    const float alpha = fast_exp2(m - base);
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        s[r] = fast_exp2(fmaf(s[r], scale2, -base));
        sum += s[r];
    }
    l = fmaf(l, alpha, sum);
    m = mn;
    return alpha;
}

// Blocks of one unit run on one XCD (blocks go to the eight of them in turn), so
// that the unit's keys and values are fetched into one L2 only.
__device__ inline int64_t xcd_order(int64_t b, int64_t n)
{
    const int64_t per = n / 8, full = per * 8;
    return b < full ? (b % 8) * per + b / 8 : b;
}

// ---- forward ------------------------------------------------------------------

template <class E>
constexpr int kv_tile() { return E::bytes == 2 ? 64 : 32; }

template <class E, int DK, int DV, int NW>
__global__ void __launch_bounds__(64 * NW)
diff_forward_kernel(DiffProblem p)
{
    using T = typename E::T;
    constexpr int KT = kv_tile<E>();
    constexpr int PK = pitch_of<E>(DK), PV = pitch_of<E>(DV);
    __shared__ alignas(16) T ks[2][KT * PK];
    __shared__ alignas(16) T vs[KT * PV];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5, c = lane & 31;
    int64_t b = xcd_order(blockIdx.x, gridDim.x);
    const int split = int(b % p.splits);
    b /= p.splits;
    const int tile = int(b % p.tiles);
    const int64_t unit = b / p.tiles;
    const int w = int(unit / p.G), kvh = int(unit % p.G);
    const int nrows = p.R * p.nq;
    const int r0 = tile * 32 * NW, r = r0 + wave * 32 + c;
    const bool live = r < nrows;
    const Row row = row_of(p, kvh, live ? r : r0);
    const int len = window_len(p, w);
    const int limit = live ? key_limit(p, len, row.token) : 0;
    const int r1 = min(r0 + 32 * NW, nrows) - 1;
    const int kbegin = split * p.chunk;
    const int kend = min(tile_limit(p, len, r0, r1), kbegin + p.chunk);

    Frag<E> q[2][DK / 16];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        const T *src = at<E>(p.q, w, 2 * row.head + a, row.token);
#pragma unroll
        for (int i = 0; i < DK / 16; ++i)
            q[a][i] = as_frag<E>(load_chunk<E>(src + 16 * i + 8 * g,
                                               live ? p.d - 16 * i - 8 * g : 0, p.vec_q));
    }
    f16v acc[2][DV / 32] = {};
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

    for (int k0 = kbegin; k0 < kend; k0 += KT) {
        __syncthreads();
        const int valid = kend - k0;
        stage<E, DK, KT>(ks[0], PK, at<E>(p.k, w, 2 * kvh, k0), p.k.token, valid, p.d, p.vec_k);
        stage<E, DK, KT>(ks[1], PK, at<E>(p.k, w, 2 * kvh + 1, k0), p.k.token, valid, p.d,
                         p.vec_k);
        stage<E, DV, KT>(vs, PV, at<E>(p.v, w, kvh, k0), p.v.token, valid, p.dv, p.vec_v);
        __syncthreads();
        for (int s0 = 0; s0 < KT; s0 += 32) {
            const int key = k0 + s0;
            if (!__any(key < limit && key < kend))
                break;
            f16v s[2] = {};
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int i = 0; i < DK / 16; ++i)
                    s[a] = mma(row_frag<E>(ks[a] + s0 * PK, PK, i), q[a][i], s[a]);
            const int lim = min(limit, kend);
            const bool masked = !__all(key + 32 <= lim);
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const float alpha = softmax_step(s[a], p.scale2, m[a], l[a], lim, key, g, masked);
                if (__any(alpha != 1.f))
#pragma unroll
                    for (int i = 0; i < DV / 32; ++i)
                        acc[a][i] *= alpha;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Frag<E> p1 = frag_of(s[0], h, E()), p2 = frag_of(s[1], h, E());
#pragma unroll
                for (int i = 0; i < DV / 32; ++i) {
                    const Frag<E> v = col_frag<E>(vs + s0 * PV, PV, h, 32 * i);
                    acc[0][i] = mma(v, p1, acc[0][i]);
                    acc[1][i] = mma(v, p2, acc[1][i]);
                }
            }
        }
    }
#pragma unroll
    for (int a = 0; a < 2; ++a)
        l[a] += other_half(l[a]);
    if (!live)
        return;
    if (p.splits > 1) {
        float *out = p.partial + ((unit * p.splits + split) * nrows + r) * p.partial_row;
#pragma unroll
        for (int a = 0; a < 2; ++a) {
#pragma unroll
            for (int i = 0; i < DV / 32; ++i)
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    store4<F32>(out + a * p.dv4, 32 * i + 8 * t + 4 * g, p.dv4, true,
                                acc[a][i][4 * t], acc[a][i][4 * t + 1], acc[a][i][4 * t + 2],
                                acc[a][i][4 * t + 3]);
            if (g == 0) {
                out[2 * p.dv4 + 2 * a] = m[a];
                out[2 * p.dv4 + 2 * a + 1] = l[a];
            }
        }
        return;
    }
    const float inv1 = l[0] == 0.f ? 0.f : 1.f / l[0];
    const float inv2 = l[1] == 0.f ? 0.f : 1.f / l[1];
    const float lam = p.lambda[row.head];
    T *o = at_out<E>(p.o, w, row.head, row.token);
    T *o2 = p.o2 ? static_cast<T *>(p.o2) + ((int64_t(w) * p.H + row.head) * p.nq + row.token) * p.dv
                 : nullptr;
#pragma unroll
    for (int i = 0; i < DV / 32; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            float x[4], y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                y[j] = acc[1][i][4 * t + j] * inv2;
                x[j] = acc[0][i][4 * t + j] * inv1 - lam * y[j];
            }
            const int col = 32 * i + 8 * t + 4 * g;
            store4<E>(o, col, p.dv, p.vec_o, x[0], x[1], x[2], x[3]);
            if (o2)
                store4<E>(o2, col, p.dv, p.vec_o2, y[0], y[1], y[2], y[3]);
        }
    if (p.lse && g == 0) {
        float *lse = p.lse + (int64_t(w) * 2 * p.H + 2 * row.head) * p.nq + row.token;
        lse[0] = l[0] == 0.f ? -INFINITY : m[0] + log2f(l[0]);
        lse[p.nq] = l[1] == 0.f ? -INFINITY : m[1] + log2f(l[1]);
    }
}

// Joins the key ranges of one row.
template <class E>
__global__ void __launch_bounds__(kMerge)
diff_merge_kernel(DiffProblem p)
{
    const int nrows = p.R * p.nq;
    const int64_t unit = blockIdx.x / unsigned(nrows);
    const int r = int(blockIdx.x - unit * nrows);
    const int w = int(unit / p.G), kvh = int(unit % p.G);
    const Row row = row_of(p, kvh, r);
    const float *part = p.partial + (unit * p.splits * nrows + r) * p.partial_row;
    const int64_t step = int64_t(nrows) * p.partial_row;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    for (int a = 0; a < 2; ++a) {
        for (int s = 0; s < p.splits; ++s)
            m[a] = fmaxf(m[a], part[s * step + 2 * p.dv4 + 2 * a]);
        for (int s = 0; s < p.splits; ++s)
            if (part[s * step + 2 * p.dv4 + 2 * a] != -INFINITY)
                l[a] += part[s * step + 2 * p.dv4 + 2 * a + 1] *
                        fast_exp2(part[s * step + 2 * p.dv4 + 2 * a] - m[a]);
    }
    const float lam = p.lambda[row.head];
    typename E::T *o = at_out<E>(p.o, w, row.head, row.token);
    typename E::T *o2 = p.o2 ? static_cast<typename E::T *>(p.o2) +
                                   ((int64_t(w) * p.H + row.head) * p.nq + row.token) * p.dv
                             : nullptr;
    for (int col = threadIdx.x; col < p.dv; col += kMerge) {
        float x[2] = {0.f, 0.f};
        for (int a = 0; a < 2; ++a) {
            for (int s = 0; s < p.splits; ++s) {
                const float ms = part[s * step + 2 * p.dv4 + 2 * a];
                if (ms != -INFINITY)
                    x[a] = fmaf(part[s * step + a * p.dv4 + col], fast_exp2(ms - m[a]), x[a]);
            }
            x[a] = l[a] == 0.f ? 0.f : x[a] / l[a];
        }
        E::store(o, col, x[0] - lam * x[1]);
        if (o2)
            E::store(o2, col, x[1]);
    }
    if (p.lse && threadIdx.x < 2) {
        const int a = threadIdx.x;
        p.lse[(int64_t(w) * 2 * p.H + 2 * row.head + a) * p.nq + row.token] =
            l[a] == 0.f ? -INFINITY : m[a] + log2f(l[a]);
    }
}

// ---- backward -----------------------------------------------------------------

// Sum of the products of two rows' elements, eight at a time.
__device__ inline float dot8(const Frag<BF16> &a, const Frag<BF16> &b)
{
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        s = fmaf(float(a.x[j]), float(b.x[j]), s);
    return s;
}

__device__ inline float dot8(const Frag<F32> &a, const Frag<F32> &b)
{
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        s = fmaf(a.x[j], b.x[j], s);
    return s;
}

// dQ, and per row D_1, D_2 and -dlam.  Rows as in the forward pass.  D_a comes from
// the outputs, D_2 = dO . O_2 and D_1 = dO . (O + lam O_2), or, where the forward pass
// kept no O_2 (few keys), from a first walk over the keys; there it is exact, so that a
// row with a single key has a gradient of zero and not the rounding of its output.
template <class E, int DK, int DV, int NW>
__global__ void __launch_bounds__(64 * NW)
diff_dq_kernel(DiffProblem p)
{
    using T = typename E::T;
    constexpr int KT = 32;
    constexpr int PK = pitch_of<E>(DK), PV = pitch_of<E>(DV);
    __shared__ alignas(16) T ks[2][KT * PK];
    __shared__ alignas(16) T vs[KT * PV];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5, c = lane & 31;
    const int64_t b = xcd_order(blockIdx.x, gridDim.x);
    const int tile = int(b % p.tiles);
    const int64_t unit = b / p.tiles;
    const int w = int(unit / p.G), kvh = int(unit % p.G);
    const int nrows = p.R * p.nq;
    const int r0 = tile * 32 * NW, r = r0 + wave * 32 + c;
    const bool live = r < nrows;
    const Row row = row_of(p, kvh, live ? r : r0);
    const int len = window_len(p, w);
    const int limit = live ? key_limit(p, len, row.token) : 0;
    const int r1 = min(r0 + 32 * NW, nrows) - 1;
    const int kend = tile_limit(p, len, r0, r1);
    const float lam = p.lambda[row.head];

    Frag<E> q[2][DK / 16], go[DV / 16];
    float L[2], D[2] = {0.f, 0.f};
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        const T *src = at<E>(p.q, w, 2 * row.head + a, row.token);
#pragma unroll
        for (int i = 0; i < DK / 16; ++i)
            q[a][i] = as_frag<E>(load_chunk<E>(src + 16 * i + 8 * g,
                                               live ? p.d - 16 * i - 8 * g : 0, p.vec_q));
        L[a] = p.lse[(int64_t(w) * 2 * p.H + 2 * row.head + a) * p.nq + row.token];
    }
    {
        const T *src = at<E>(p.go, w, row.head, row.token);
        const T *o = at<E>(p.o, w, row.head, row.token);
        const T *o2 = static_cast<const T *>(p.o2) +
                      ((int64_t(w) * p.H + row.head) * p.nq + row.token) * p.dv;
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < DV / 16; ++i) {
            const int col = 16 * i + 8 * g, n = live ? p.dv - col : 0;
            go[i] = as_frag<E>(load_chunk<E>(src + col, n, p.vec_go));
            if (p.o2) {
                dot += dot8(go[i], as_frag<E>(load_chunk<E>(o + col, n, p.vec_o)));
                D[1] += dot8(go[i], as_frag<E>(load_chunk<E>(o2 + col, n, p.vec_o2)));
            }
        }
        D[0] = fmaf(lam, D[1], dot);
#pragma unroll
        for (int a = 0; a < 2; ++a)
            D[a] += other_half(D[a]);
    }
    f16v acc[2][DK / 32] = {};
    float glam = 0.f;
    for (int sweep = p.o2 ? 1 : 0; sweep < 2; ++sweep) {
        float sum[2] = {0.f, 0.f};
        for (int k0 = 0; k0 < kend; k0 += KT) {
            __syncthreads();
            const int valid = kend - k0;
            stage<E, DK, KT>(ks[0], PK, at<E>(p.k, w, 2 * kvh, k0), p.k.token, valid, p.d,
                             p.vec_k);
            stage<E, DK, KT>(ks[1], PK, at<E>(p.k, w, 2 * kvh + 1, k0), p.k.token, valid, p.d,
                             p.vec_k);
            stage<E, DV, KT>(vs, PV, at<E>(p.v, w, kvh, k0), p.v.token, valid, p.dv, p.vec_v);
            __syncthreads();
            if (!__any(k0 < limit))
                continue;
            f16v s[2] = {}, x = {};
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int i = 0; i < DK / 16; ++i)
                    s[a] = mma(row_frag<E>(ks[a], PK, i), q[a][i], s[a]);
#pragma unroll
            for (int i = 0; i < DV / 16; ++i)
                x = mma(row_frag<E>(vs, PV, i), go[i], x);
            const bool masked = !__all(k0 + KT <= limit);
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int t = 0; t < 16; ++t) {
                    s[a][t] = fast_exp2(fmaf(s[a][t], p.scale2, -L[a]));
                    if (masked)
                        s[a][t] = k0 + reg_row(t, g) < limit ? s[a][t] : 0.f;
                }
            if (sweep == 0) {
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int t = 0; t < 16; ++t)
                        sum[a] = fmaf(s[a][t], x[t], sum[a]);
                continue;
            }
#pragma unroll
            for (int t = 0; t < 16; ++t) {
                glam = fmaf(s[1][t], x[t], glam);
                s[0][t] = s[0][t] * (x[t] - D[0]);
                s[1][t] = -lam * s[1][t] * (x[t] - D[1]);
            }
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const Frag<E> ds = frag_of(s[a], h, E());
#pragma unroll
                    for (int i = 0; i < DK / 32; ++i)
                        acc[a][i] = mma(col_frag<E>(ks[a], PK, h, 32 * i), ds, acc[a][i]);
                }
        }
        if (sweep == 0) {
#pragma unroll
            for (int a = 0; a < 2; ++a)
                D[a] = sum[a] + other_half(sum[a]);
        }
    }
    glam += other_half(glam);
    if (!live)
        return;
    if (g == 0) {
        const int64_t at_row = unit * nrows + r;
        p.rows_d1[at_row] = D[0];
        p.rows_d2[at_row] = D[1];
        p.rows_lam[at_row] = glam;
    }
    // A softmax over one key is constant: its gradient is zero, not the rounding of D.
    const float scale = limit == 1 ? 0.f : p.scale;
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        T *dst = at_out<E>(p.gq, w, 2 * row.head + a, row.token);
#pragma unroll
        for (int i = 0; i < DK / 32; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t)
                store4<E>(dst, 32 * i + 8 * t + 4 * g, p.d, p.vec_gq, scale * acc[a][i][4 * t],
                          scale * acc[a][i][4 * t + 1], scale * acc[a][i][4 * t + 2],
                          scale * acc[a][i][4 * t + 3]);
    }
}

// dK and dV: a wave owns 32 keys and walks over the unit's rows, so that the heads
// that share the keys are summed in registers.  Keys at or behind the window's
// length get zeros.
template <class E, int DK, int DV, int NW>
__global__ void __launch_bounds__(64 * NW)
diff_dkv_kernel(DiffProblem p)
{
    using T = typename E::T;
    constexpr int QT = 32;
    constexpr int PK = pitch_of<E>(DK), PV = pitch_of<E>(DV);
    __shared__ alignas(16) T qs[2][QT * PK];
    __shared__ alignas(16) T gs[QT * PV];
    __shared__ alignas(16) float stat[5][QT];   // L_1, L_2, D_1, D_2, lam
    __shared__ int lim[QT];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5, c = lane & 31;
    const int64_t b = xcd_order(blockIdx.x, gridDim.x);
    const int tile = int(b % p.ktiles);
    const int64_t unit = b / p.ktiles;
    const int w = int(unit / p.G), kvh = int(unit % p.G);
    const int nrows = p.R * p.nq;
    const int kb = tile * 32 * NW, kw = kb + wave * 32, key = kw + c;
    const int len = window_len(p, w);
    const bool live = key < len;

    Frag<E> k[2][DK / 16], v[DV / 16];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        const T *src = at<E>(p.k, w, 2 * kvh + a, live ? key : 0);
#pragma unroll
        for (int i = 0; i < DK / 16; ++i)
            k[a][i] = as_frag<E>(load_chunk<E>(src + 16 * i + 8 * g,
                                               live ? p.d - 16 * i - 8 * g : 0, p.vec_k));
    }
    {
        const T *src = at<E>(p.v, w, kvh, live ? key : 0);
#pragma unroll
        for (int i = 0; i < DV / 16; ++i)
            v[i] = as_frag<E>(load_chunk<E>(src + 16 * i + 8 * g,
                                            live ? p.dv - 16 * i - 8 * g : 0, p.vec_v));
    }
    f16v gk[2][DK / 32] = {}, gv[DV / 32] = {};
    for (int r0 = 0; r0 < nrows && kb < len; r0 += QT) {
        if (tile_limit(p, len, r0, min(r0 + QT, nrows) - 1) <= kb)
            continue;   // no row of this tile sees a key of this workgroup
        __syncthreads();
        for (int i = threadIdx.x; i < QT * (DK / 8); i += 64 * NW) {
            const int rr = i / (DK / 8), ch = i % (DK / 8);
            const bool in = r0 + rr < nrows;
            const Row row = row_of(p, kvh, in ? r0 + rr : r0);
#pragma unroll
            for (int a = 0; a < 2; ++a)
                *reinterpret_cast<Chunk<E> *>(qs[a] + rr * PK + 8 * ch) =
                    load_chunk<E>(at<E>(p.q, w, 2 * row.head + a, row.token) + 8 * ch,
                                  in ? p.d - 8 * ch : 0, p.vec_q);
        }
        for (int i = threadIdx.x; i < QT * (DV / 8); i += 64 * NW) {
            const int rr = i / (DV / 8), ch = i % (DV / 8);
            const bool in = r0 + rr < nrows;
            const Row row = row_of(p, kvh, in ? r0 + rr : r0);
            *reinterpret_cast<Chunk<E> *>(gs + rr * PV + 8 * ch) =
                load_chunk<E>(at<E>(p.go, w, row.head, row.token) + 8 * ch,
                              in ? p.dv - 8 * ch : 0, p.vec_go);
        }
        if (threadIdx.x < QT) {
            const int rr = r0 + threadIdx.x;
            const bool in = rr < nrows;
            const Row row = row_of(p, kvh, in ? rr : r0);
            const int n = in ? key_limit(p, len, row.token) : 0;
            const float *lse = p.lse + (int64_t(w) * 2 * p.H + 2 * row.head) * p.nq + row.token;
            // A row that sees no key has probabilities exp2(-inf) = 0.
            stat[0][threadIdx.x] = n > 0 ? lse[0] : INFINITY;
            stat[1][threadIdx.x] = n > 0 ? lse[p.nq] : INFINITY;
            stat[2][threadIdx.x] = in ? p.rows_d1[unit * nrows + rr] : 0.f;
            stat[3][threadIdx.x] = in ? p.rows_d2[unit * nrows + rr] : 0.f;
            stat[4][threadIdx.x] = p.lambda[row.head];
            lim[threadIdx.x] = n;
        }
        __syncthreads();
        if (!__any(kw < lim[c]))
            continue;
        const bool masked = !__all(kw + 32 <= lim[c]);
        f16v s[2] = {}, x = {};
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int i = 0; i < DK / 16; ++i)
                s[a] = mma(row_frag<E>(qs[a], PK, i), k[a][i], s[a]);
#pragma unroll
        for (int i = 0; i < DV / 16; ++i)
            x = mma(row_frag<E>(gs, PV, i), v[i], x);
        f16v pd;
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            const int rr = reg_row(t, g);
            float p1 = fast_exp2(fmaf(s[0][t], p.scale2, -stat[0][rr]));
            float p2 = fast_exp2(fmaf(s[1][t], p.scale2, -stat[1][rr]));
            if (masked) {
                const bool see = key < lim[rr];
                p1 = see ? p1 : 0.f;
                p2 = see ? p2 : 0.f;
            }
            p2 *= stat[4][rr];
            pd[t] = p1 - p2;
            s[0][t] = p1 * (x[t] - stat[2][rr]);
            s[1][t] = -p2 * (x[t] - stat[3][rr]);
            if (masked && lim[rr] == 1)   // constant: as in the dQ kernel
                s[0][t] = s[1][t] = 0.f;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const Frag<E> f = frag_of(pd, h, E());
#pragma unroll
            for (int i = 0; i < DV / 32; ++i)
                gv[i] = mma(col_frag<E>(gs, PV, h, 32 * i), f, gv[i]);
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const Frag<E> ds = frag_of(s[a], h, E());
#pragma unroll
                for (int i = 0; i < DK / 32; ++i)
                    gk[a][i] = mma(col_frag<E>(qs[a], PK, h, 32 * i), ds, gk[a][i]);
            }
        }
    }
    if (key >= p.nk)
        return;
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        T *dst = at_out<E>(p.gk, w, 2 * kvh + a, key);
#pragma unroll
        for (int i = 0; i < DK / 32; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t)
                store4<E>(dst, 32 * i + 8 * t + 4 * g, p.d, p.vec_gk,
                          live ? p.scale * gk[a][i][4 * t] : 0.f,
                          live ? p.scale * gk[a][i][4 * t + 1] : 0.f,
                          live ? p.scale * gk[a][i][4 * t + 2] : 0.f,
                          live ? p.scale * gk[a][i][4 * t + 3] : 0.f);
    }
    T *dst = at_out<E>(p.gv, w, kvh, key);
#pragma unroll
    for (int i = 0; i < DV / 32; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t)
            store4<E>(dst, 32 * i + 8 * t + 4 * g, p.dv, p.vec_gv, live ? gv[i][4 * t] : 0.f,
                      live ? gv[i][4 * t + 1] : 0.f, live ? gv[i][4 * t + 2] : 0.f,
                      live ? gv[i][4 * t + 3] : 0.f);
}

// dlam of one head: its rows over all windows.
__global__ void __launch_bounds__(1024)
diff_dlam_kernel(const float *__restrict__ rows, int W, int H, int nq, float *__restrict__ out)
{
    __shared__ float lds[16];
    const int h = blockIdx.x;
    const int64_t n = int64_t(W) * nq;
    float s = 0.f;
    for (int64_t i = threadIdx.x; i < n; i += 1024) {
        const int64_t w = i / nq;
        s += rows[(w * H + h) * nq + (i - w * nq)];
    }
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0)
        lds[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.f;
        for (int i = 0; i < 16; ++i)
            s += lds[i];
        out[h] = -s;
    }
}

// ---- dispatch -----------------------------------------------------------------

// Bytes of one load that every row of a tensor allows: 16, 4 or the element's.
int view_vec(const DiffView &v, int width, int bytes)
{
    const int64_t n = (v.window | v.head | v.token | width) * bytes;
    const uintptr_t a = uintptr_t(v.data);
    return (a % 16 == 0 && n % 16 == 0) ? 16 : (a % 4 == 0 && n % 4 == 0) ? 4 : bytes;
}

// Whether groups of four elements may be stored at once.
bool store_vec(const DiffView &v, int width, int bytes)
{
    return uintptr_t(v.data) % (4 * bytes) == 0 && ((v.window | v.head | v.token | width) % 4) == 0;
}

int ceil_div(int64_t a, int64_t b) { return int((a + b - 1) / b); }

// Waves to a workgroup: as many as there are tiles of 32 rows (or keys), at most four.
int waves_for(int64_t rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : 4; }

// Key ranges that a forward call is split into: enough workgroups for the 256 CUs
// twice over, of at least 256 keys each.
int splits_for(int64_t blocks, int nk)
{
    const int most = ceil_div(nk, 256);
    const int64_t want = (512 + blocks - 1) / blocks;
    return int(want < most ? want : most);
}

struct Plan {
    int waves, tiles, splits, chunk;
    int64_t blocks;
};

Plan forward_plan(const DiffProblem &p)
{
    Plan f;
    const int64_t rows = int64_t(p.R) * p.nq;
    f.waves = waves_for(rows);
    f.tiles = ceil_div(rows, 32 * f.waves);
    const int64_t units = int64_t(p.W) * p.G;
    f.splits = splits_for(units * f.tiles, p.nk);
    f.chunk = ceil_div(ceil_div(p.nk, f.splits), 64) * 64;
    f.splits = ceil_div(p.nk, f.chunk);
    f.blocks = units * f.tiles * f.splits;
    return f;
}

template <class E, int DK, int DV, int NW>
void run_forward(const DiffProblem &p, int64_t blocks, hipStream_t s)
{
    diff_forward_kernel<E, DK, DV, NW><<<dim3(unsigned(blocks)), 64 * NW, 0, s>>>(p);
}

template <class E, int DK, int DV>
void forward_waves(const DiffProblem &p, const Plan &f, hipStream_t s)
{
    if (f.waves == 1)
        run_forward<E, DK, DV, 1>(p, f.blocks, s);
    else if (f.waves == 2)
        run_forward<E, DK, DV, 2>(p, f.blocks, s);
    else
        run_forward<E, DK, DV, 4>(p, f.blocks, s);
}

template <class E, int DK, int DV, int NW>
void run_backward(const DiffProblem &p, bool keys, int64_t blocks, hipStream_t s)
{
    if (keys)
        diff_dkv_kernel<E, DK, DV, NW><<<dim3(unsigned(blocks)), 64 * NW, 0, s>>>(p);
    else
        diff_dq_kernel<E, DK, DV, NW><<<dim3(unsigned(blocks)), 64 * NW, 0, s>>>(p);
}

template <class E, int DK, int DV>
void backward_waves(const DiffProblem &p, bool keys, int waves, int64_t blocks, hipStream_t s)
{
    if (waves == 1)
        run_backward<E, DK, DV, 1>(p, keys, blocks, s);
    else if (waves == 2)
        run_backward<E, DK, DV, 2>(p, keys, blocks, s);
    else
        run_backward<E, DK, DV, 4>(p, keys, blocks, s);
}

// Widths are padded to 32 (queries, keys) and 64 (values) or to 64 and 128.
bool narrow(const DiffProblem &p) { return p.d <= 32 && p.dv <= 64; }

template <class E>
void forward_any(const DiffProblem &p, const Plan &f, hipStream_t s)
{
    if (narrow(p))
        forward_waves<E, 32, 64>(p, f, s);
    else
        forward_waves<E, 64, 128>(p, f, s);
}

template <class E>
void backward_any(const DiffProblem &p, bool keys, int waves, int64_t blocks, hipStream_t s)
{
    if (narrow(p))
        backward_waves<E, 32, 64>(p, keys, waves, blocks, s);
    else
        backward_waves<E, 64, 128>(p, keys, waves, blocks, s);
}

int64_t rows_bytes(const DiffProblem &p)
{
    return (int64_t(p.W) * p.H * p.nq * 4 + 255) / 256 * 256;
}

}  // namespace

bool diff_grid_fits(const DiffProblem &p)
{
    const int64_t rows = int64_t(p.R) * p.nq, units = int64_t(p.W) * p.G;
    // The largest grids: one wave to 32 rows or keys over one split, and the merge's rows.
    const int64_t most = units * ((rows + 31) / 32 + (p.nk + 31) / 32) + units * rows;
    return rows < (int64_t(1) << 30) && most < (int64_t(1) << 24);
}

size_t diff_forward_workspace(const DiffProblem &p)
{
    const Plan f = forward_plan(p);
    const int64_t row = 2 * ((p.dv + 3) / 4 * 4) + 4;
    return f.splits > 1
               ? size_t(int64_t(p.W) * p.G * f.splits * p.R * p.nq * row) * sizeof(float)
               : 0;
}

size_t diff_backward_workspace(const DiffProblem &p) { return size_t(3 * rows_bytes(p)); }

static void set_vectors(DiffProblem *p)
{
    const int e = p->dtype == 0 ? 4 : 2;
    p->vec_q = view_vec(p->q, p->d, e);
    p->vec_k = view_vec(p->k, p->d, e);
    p->vec_v = view_vec(p->v, p->dv, e);
}

hipError_t launch_diff_forward(DiffProblem p, void *workspace, hipStream_t s)
{
    const int e = p.dtype == 0 ? 4 : 2;
    const Plan f = forward_plan(p);
    set_vectors(&p);
    p.vec_o = store_vec(p.o, p.dv, e);
    p.vec_o2 = store_vec(DiffView{p.o2, p.dv, p.dv, p.dv}, p.dv, e);
    p.tiles = f.tiles;
    p.splits = f.splits;
    p.chunk = f.chunk;
    p.partial = static_cast<float *>(workspace);
    p.dv4 = (p.dv + 3) / 4 * 4;
    p.partial_row = 2 * p.dv4 + 4;
    p.dtype == 0 ? forward_any<F32>(p, f, s) : forward_any<BF16>(p, f, s);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess || f.splits == 1)
        return err;
    const dim3 grid(unsigned(int64_t(p.W) * p.G * p.R * p.nq));
    if (p.dtype == 0)
        diff_merge_kernel<F32><<<grid, kMerge, 0, s>>>(p);
    else
        diff_merge_kernel<BF16><<<grid, kMerge, 0, s>>>(p);
    return hipGetLastError();
}

hipError_t launch_diff_backward(DiffProblem p, void *workspace, float *glam, hipStream_t s)
{
    const int e = p.dtype == 0 ? 4 : 2;
    set_vectors(&p);
    p.vec_go = view_vec(p.go, p.dv, e);
    p.vec_o = p.o2 ? view_vec(p.o, p.dv, e) : e;
    p.vec_o2 = view_vec(DiffView{p.o2, p.dv, p.dv, p.dv}, p.dv, e);
    p.vec_gq = store_vec(p.gq, p.d, e);
    p.vec_gk = store_vec(p.gk, p.d, e);
    p.vec_gv = store_vec(p.gv, p.dv, e);
    char *ws = static_cast<char *>(workspace);
    p.rows_d1 = reinterpret_cast<float *>(ws);
    p.rows_d2 = reinterpret_cast<float *>(ws + rows_bytes(p));
    p.rows_lam = reinterpret_cast<float *>(ws + 2 * rows_bytes(p));
    const int64_t rows = int64_t(p.R) * p.nq, units = int64_t(p.W) * p.G;
    if (units > 0) {
        const int wq = waves_for(rows), wk = waves_for(p.nk);
        p.tiles = ceil_div(rows, 32 * wq);
        p.ktiles = ceil_div(p.nk, 32 * wk);
        for (const bool keys : {false, true}) {
            const int waves = keys ? wk : wq;
            const int64_t blocks = units * (keys ? p.ktiles : p.tiles);
            p.dtype == 0 ? backward_any<F32>(p, keys, waves, blocks, s)
                         : backward_any<BF16>(p, keys, waves, blocks, s);
            const hipError_t err = hipGetLastError();
            if (err != hipSuccess)
                return err;
        }
    }
    diff_dlam_kernel<<<p.H, 1024, 0, s>>>(p.rows_lam, p.W, p.H, p.nq, glam);
    return hipGetLastError();
}

}  // namespace nystra
