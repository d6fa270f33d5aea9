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
// bf16 runs it as one matrix instruction.  fp32 operands are carried as three bf16 terms
// (24 bits), whose six largest products make a product: 192 cycles against 512 of the eight
// fp32 instructions of depth two, and within 2^-22 of it.
#pragma once

#include <type_traits>

#include "device_common.hpp"
#include "internal.hpp"

namespace nystra {
namespace diff {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

template <class E>
struct Frag;

template <>
struct Frag<BF16> {
    bf8 x;
};

// x = h + m + l: h is x cut off at bf16, m and l are rounded to nearest even; exact down to
// |x| = 2^-110.  An infinity becomes NaN (its rest is inf - inf).
template <>
struct Frag<F32> {
    bf8 h, m, l;
};

__device__ inline f16v mma(const Frag<BF16> &a, const Frag<BF16> &b, f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.x, b.x, c, 0, 0, 0);
}

// The small products first; those left out (m l, l m, l l) are below 2^-22 of the whole.
__device__ inline f16v mma(const Frag<F32> &a, const Frag<F32> &b, f16v c)
{
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.l, b.h, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.h, b.l, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.m, b.m, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.m, b.h, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.h, b.m, c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.h, b.h, c, 0, 0, 0);
}

__device__ inline Frag<F32> split(const float (&x)[8])
{
    typedef float f8 __attribute__((ext_vector_type(8)));
    typedef uint32_t h8 __attribute__((ext_vector_type(4)));
    Frag<F32> f;
    h8 h;
    f8 r;
#pragma unroll
    for (int j = 0; j < 4; ++j)   // the upper halves of two
        h[j] = __builtin_amdgcn_perm(__float_as_uint(x[2 * j + 1]), __float_as_uint(x[2 * j]),
                                     0x07060302u);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        r[j] = x[j] - __uint_as_float(__float_as_uint(x[j]) & 0xffff0000u);
    f.h = __builtin_bit_cast(bf8, h);
    f.m = __builtin_convertvector(r, bf8);
    f.l = __builtin_convertvector(r - __builtin_convertvector(f.m, f8), bf8);
    return f;
}

// Eight consecutive elements as they lie in memory.
template <class E>
struct alignas(16) Chunk {
    uint32_t w[2 * E::bytes];
};

// 16 bytes from an address that is aligned to the element only.
template <class E>
struct __attribute__((packed, aligned(E::bytes))) Loose {
    uint32_t w[4];
};

// Eight elements of a row from p, of which the row has n (n may be <= 0 or above 8); the
// others, and all of them if the row is not `live`, are zero.  Every lane loads 16 bytes at a
// time, from the row's last ones where its own would reach past the row, and shifts those
// down, so that there are no branches and nothing is read outside the row.  WIDE: n is a
// multiple of eight and the address of 16 bytes.  `width`: the row's elements, of which
// fewer than 16 bytes are taken one by one.
template <class E, bool WIDE>
__device__ inline Chunk<E> load_chunk(const typename E::T *p, int n, bool live, int width)
{
    constexpr int per = 16 / E::bytes;
    Chunk<E> c;
#pragma unroll
    for (int h = 0; h < 8 / per; ++h) {
        const int left = n - h * per;   // elements of the row from here on
        uint32_t w[4];
        if (WIDE) {
            const uint4 u = *reinterpret_cast<const uint4 *>(p + min(0, left - per));
            w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
        } else if (width >= per) {
            const Loose<E> u =
                *reinterpret_cast<const Loose<E> *>(p + h * per + min(0, left - per));
#pragma unroll
            for (int j = 0; j < 4; ++j)
                w[j] = u.w[j];
            if (width % per != 0) {
                const int skip = max(0, per - left) * E::bytes;   // bytes, below 16 where live
                if (skip & 8)
                    w[0] = w[2], w[1] = w[3], w[2] = w[3] = 0u;
                if (skip & 4)
                    w[0] = w[1], w[1] = w[2], w[2] = w[3], w[3] = 0u;
                if (E::bytes == 2 && skip & 2)
                    w[0] = w[0] >> 16 | w[1] << 16, w[1] = w[1] >> 16 | w[2] << 16,
                    w[2] = w[2] >> 16 | w[3] << 16, w[3] >>= 16;
            }
        } else {
            w[0] = w[1] = w[2] = w[3] = 0u;
#pragma unroll 1   // rare and called in many places: small code
            for (int j = 0; j < per; ++j) {
                // The next element in from the top, the others down by one.
                const typename E::T *q = p + h * per + min(j, left - 1);
                if (E::bytes == 4) {
                    const uint32_t u = *reinterpret_cast<const uint32_t *>(q);
                    w[0] = w[1], w[1] = w[2], w[2] = w[3], w[3] = j < left ? u : 0u;
                } else {
                    const uint32_t u = *reinterpret_cast<const uint16_t *>(q);
                    w[0] = w[0] >> 16 | w[1] << 16, w[1] = w[1] >> 16 | w[2] << 16;
                    w[2] = w[2] >> 16 | w[3] << 16, w[3] = w[3] >> 16 | (j < left ? u << 16 : 0u);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            c.w[4 * h + j] = live && left > 0 ? w[j] : 0u;
    }
    return c;
}

__device__ inline Frag<BF16> as_frag(const Chunk<BF16> &c)
{
    return __builtin_bit_cast(Frag<BF16>, c);
}

__device__ inline Frag<F32> as_frag(const Chunk<F32> &c)
{
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        x[j] = __uint_as_float(c.w[j]);
    return split(x);
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
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        x[j] = s[8 * c + j];
    return split(x);
}

// LDS is addressed by byte offsets.
__device__ inline uint32_t lds_offset(void *p)
{
    return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void *)p));
}

template <class T>
__device__ inline __attribute__((address_space(3))) T *lds_at(uint32_t at)
{
    return (__attribute__((address_space(3))) T *)(uintptr_t(at));
}

__device__ inline void exchange(uint32_t &a, uint32_t &b)
{
    const uint32_t x = a;
    a = b;
    b = x;
}

// A tile of 32 rows of COLS elements in LDS, in chunks of eight elements, fp32 as one plane
// for each of its three terms.  Row fragments read the same chunk of eight rows at a time, the
// transposing reads below two neighbouring chunks of four rows; over the 64 banks of 4 bytes
// neither may meet a bank twice.  Rows lie without gaps (so that loads can go to LDS directly)
// with their chunks exchanged by a number from the row.  A tile starts at a multiple of 256
// bytes, so that its fragments follow from the first one's address by an exclusive or (one
// instruction and no register each).
template <class E, int COLS>
struct Tile {
    static constexpr int pitch = 2 * COLS;   // bytes
    static constexpr int kRow = COLS / 8;
    static constexpr uint32_t kPlane = 32 * pitch;
    static constexpr uint32_t kBytes = E::bytes == 2 ? kPlane : 3 * kPlane;

    __device__ static inline int swap(int row)
    {
        return COLS == 32 ? (row >> 2) & 3 : COLS == 64 ? row & 7 : (row & 7) << 1;
    }
    __device__ static inline uint32_t at(int row, int chunk)
    {
        return row * pitch + 16 * (chunk ^ swap(row));
    }
    __device__ static inline void store(uint32_t tile, int row, int chunk, const Chunk<E> &c)
    {
        const Frag<E> f = as_frag(c);
        const uint32_t to = tile + at(row, chunk);
        if constexpr (E::bytes == 2) {
            *lds_at<bf8>(to) = f.x;
        } else {
            *lds_at<bf8>(to) = f.h;
            *lds_at<bf8>(to + kPlane) = f.m;
            *lds_at<bf8>(to + 2 * kPlane) = f.l;
        }
    }
};

// Row fragments: row lane % 32 of the tile at `tile`, contraction indices (columns)
// 16 c + 8 g + j.  first_row() gives the address for c = 0.
template <class E, int COLS>
__device__ inline uint32_t first_row(uint32_t tile, unsigned lane = threadIdx.x & 63)
{
    return tile + Tile<E, COLS>::at(lane & 31, lane >> 5);
}

template <class E, int COLS>
__device__ inline Frag<E> row_frag(uint32_t first, int c)
{
    constexpr uint32_t plane = Tile<E, COLS>::kPlane;
    const uint32_t at = first ^ (32 * c);
    if constexpr (E::bytes == 2)
        return Frag<E>{*lds_at<bf8>(at)};
    else
        return Frag<E>{*lds_at<bf8>(at), *lds_at<bf8>(at + plane), *lds_at<bf8>(at + 2 * plane)};
}

// Column fragments: column 32 i + lane % 32, contraction indices (rows) in the order of a
// product's result, 16 c + 8 (j / 4) + 4 g + j % 4.  The transposing LDS read takes four rows
// of 16 columns from 16 lanes (lane p: row p / 4, columns 4 (p % 4) ..) and gives each lane
// its column of them.
template <class E, int COLS>
__device__ inline uint32_t first_col(uint32_t tile, unsigned lane = threadIdx.x & 63)
{
    const int col = (lane & 16) + 4 * (lane & 3);
    return tile + Tile<E, COLS>::at(4 * (lane >> 5) + ((lane & 15) >> 2), col >> 3) +
           2 * (col & 7);
}

template <int COLS>
__device__ inline bf8 col_plane(uint32_t first, int c, int i)
{
    constexpr int pitch = 2 * COLS;
    const uint32_t lo = (first ^ (64 * i)) + 16 * c * pitch;
    // Eight rows on, rows of four chunks have theirs exchanged by another number.
    const uint32_t hi = (COLS == 32 ? first ^ 32 : first ^ (64 * i)) + (16 * c + 8) * pitch;
    struct {
        s4 lo, hi;
    } v;
    v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<s4>(lo));
    v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_at<s4>(hi));
    return __builtin_bit_cast(bf8, v);
}

template <class E, int COLS>
__device__ inline Frag<E> col_frag(uint32_t first, int c, int i)
{
    constexpr uint32_t plane = Tile<E, COLS>::kPlane;
    if constexpr (E::bytes == 2)
        return Frag<E>{col_plane<COLS>(first, c, i)};
    else
        return Frag<E>{col_plane<COLS>(first, c, i), col_plane<COLS>(first + plane, c, i),
                       col_plane<COLS>(first + 2 * plane, c, i)};
}

// Walks tiles of together ROWS rows in chunks of eight elements over the NT threads of a
// workgroup: loaded into registers while the tile before it is worked on, stored to LDS
// when that is done.
template <class E, int COLS, int ROWS, int NT>
struct Stage {
    using L = Tile<E, COLS>;
    static constexpr int kAll = ROWS * L::kRow;
    static constexpr int kN = (kAll + NT - 1) / NT;
    Chunk<E> x[kN];

    // at(row) points to the first element of a row, live(row) says whether it is there.
    // Row 0 is always there.
    template <class At, class Live>
    __device__ inline void load(At at, Live live, int cols)
    {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int id = threadIdx.x + i * NT;
            const int row = id / L::kRow % ROWS, col = id % L::kRow * 8;
            const bool in = live(row);
            x[i] = load_chunk<E, false>(at(in ? row : 0) + col, cols - col, in, cols);
        }
    }

    __device__ inline void store(uint32_t lds) const
    {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int id = threadIdx.x + i * NT;
            if (kAll % NT == 0 || id < kAll)
                L::store(lds + id / L::kRow / 32 * L::kBytes, id / L::kRow % 32, id % L::kRow, x[i]);
        }
    }
};

// BYTES (16 or 4) from `base` plus each lane's offset to LDS, lane after lane from `lds` on,
// past the registers.  Nothing waits for it but arrived().  base and lds are the wave's.
// A vector memory instruction may read an SGPR that a VALU instruction wrote (a base from
// v_readfirstlane, or one that was kept in a vector register) five wait states later at the
// earliest, and m0 one after its writing; the compiler does not look into the statement for
// either.  Scalar instructions wait by themselves, and so do reads of what they wrote: base
// is copied by one, which is m0's wait state, too.
template <int BYTES>
__device__ inline void load_to_lds(const void *base, uint32_t offset, uint32_t lds)
{
    static_assert(BYTES == 16 || BYTES == 4, "one of the instruction's widths");
    uint32_t m0;
    const void *from;
    if constexpr (BYTES == 16)
        asm volatile("s_mov_b32 m0, %2\n\ts_mov_b64 %1, %4\n\tglobal_load_lds_dwordx4 %3, %1"
                     : "=&{m0}"(m0), "=&s"(from) : "s"(lds), "v"(offset), "s"(base) : "memory");
    else
        asm volatile("s_mov_b32 m0, %2\n\ts_mov_b64 %1, %4\n\tglobal_load_lds_dword %3, %1"
                     : "=&{m0}"(m0), "=&s"(from) : "s"(lds), "v"(offset), "s"(base) : "memory");
}

__device__ inline void arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// The thread's number, worked out anew by everything that follows from it here: for kernels
// that have no registers to keep such values in from one tile to the next (where they went to
// memory, their loads waited for the tile's).
__device__ inline unsigned thread_again()
{
    unsigned thread = threadIdx.x;
    asm volatile("" : "+v"(thread));
    return thread;
}

// The same tile by loads that go to LDS directly, for rows of whole and aligned groups of
// BYTES; at(row) is the row's offset from `base` in elements, below 2^30.  Every lane loads:
// rows that are not there must be given as another's (their products are masked), and columns
// from `cols` on hold the last group again (the other operand is zero there; times an infinity
// that is NaN.  Leaving them out: 1024 x 6 windows of 64 tokens of 30 / 60, both passes, 249
// instead of 243 us with the lanes switched off around each load, 269 with a branch).
template <int COLS, int ROWS, int NT, int BYTES, class At>
__device__ inline void direct_tile(uint32_t lds, const void *base, At at, int cols,
                                   unsigned thread = threadIdx.x)
{
    using L = Tile<BF16, COLS>;
    constexpr int kPer = 16 / BYTES, kRow = kPer * L::kRow, kWide = BYTES / 2;
    static_assert(ROWS * kRow % NT == 0, "whole waves");
    const uint32_t to = lds + 64 * BYTES * __builtin_amdgcn_readfirstlane(thread / 64);
#pragma unroll
    for (int i = 0; i < ROWS * kRow / NT; ++i) {
        const unsigned id = thread + i * NT;
        const int row = id / kRow, chunk = int(id % kRow / kPer) ^ L::swap(row);
        const int col = min(8 * chunk + kWide * int(id % kPer), cols - kWide);
        load_to_lds<BYTES>(base, 2 * uint32_t(at(row) + col), to + BYTES * i * NT);
    }
}

// The values of lanes c and c + 32, the same in both.
struct Halves {
    float lo, hi;
};

__device__ inline Halves halves(float x)
{
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return Halves{__builtin_bit_cast(float, unsigned(r[0])),
                  __builtin_bit_cast(float, unsigned(r[1]))};
}

__device__ inline float half_sum(float x)
{
    const Halves h = halves(x);
    return h.lo + h.hi;
}

__device__ inline float half_max(float x)
{
    const Halves h = halves(x);
    return fmaxf(h.lo, h.hi);
}

// r / n_q for 0 <= r < 2^30: with k = 31 + floor(log2 n_q) and M = ceil(2^k / n_q), M n_q
// exceeds 2^k by less than n_q < 2^(k - 30), so floor(r M / 2^k) is exact.
__device__ inline int div_nq(const DiffProblem &p, int r)
{
    return int((uint64_t(uint32_t(r)) * p.nq_mul) >> p.nq_shift);
}

// Position of a row of the unit: its query head and token.
struct Row {
    int head, token;
};

__device__ inline Row row_of(const DiffProblem &p, int g, int r)
{
    const int hh = div_nq(p, r);
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
    const int h1 = div_nq(p, r1);
    if (div_nq(p, r0) != h1)
        return key_limit(p, len, p.nq - 1);
    return key_limit(p, len, r1 - h1 * p.nq);
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

template <class E, bool ALIGNED>
__device__ inline void store_vec4(typename E::T *at, f4 x)
{
    typedef __bf16 b4 __attribute__((ext_vector_type(4)));
    using V = std::conditional_t<E::bytes == 4, f4, b4>;
    struct __attribute__((packed, aligned(E::bytes))) Any {
        V v;
    };
    const V v = __builtin_convertvector(x, V);   // bf16: to nearest even
    if constexpr (ALIGNED)
        *reinterpret_cast<V *>(at) = v;
    else
        reinterpret_cast<Any *>(at)->v = v;
}

// Four consecutive elements of an output row from column `col`, those below `n`; `vec`
// says that such groups are whole and aligned.  Others are stored whole at the elements'
// alignment, and only a row's last one by elements.
template <class E>
__device__ inline void store4(typename E::T *row, int col, int n, bool vec, f4 x)
{
    if (vec) {
        if (col < n)
            store_vec4<E, true>(row + col, x);
        return;
    }
    if (col + 4 <= n) {
        store_vec4<E, false>(row + col, x);
        return;
    }
#pragma unroll
    for (int j = 0; j < 3; ++j)
        if (col + j < n) {
            if constexpr (E::bytes == 4)
                row[col + j] = x[j];
            else
                reinterpret_cast<__bf16 *>(row)[col + j] = __bf16(x[j]);
        }
}

// A lane's part of the columns 32 i .. 32 i + 31 of its output row, times `scale`: in the order
// of a product's result, 32 i + 8 (r / 4) + 4 g + r % 4.
template <class E>
__device__ inline void store_block(typename E::T *row, int i, int g, int n, bool vec,
                                   const f16v &x, float scale = 1.f)
{
    f4 v[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[t][j] = scale * x[4 * t + j];
    if (vec && 32 * i + 32 <= n) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
            store_vec4<E, true>(row + 4 * g + 32 * i + 8 * t, v[t]);
    } else if (32 * i + 32 <= n) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
            store_vec4<E, false>(row + 4 * g + 32 * i + 8 * t, v[t]);
    } else {
#pragma unroll
        for (int t = 0; t < 4; ++t)
            store4<E>(row, 32 * i + 8 * t + 4 * g, n, vec, v[t]);
    }
}

// The exponents' base and the sum of a row's exponentials for its first map, in
// [W][2 H][n_q][2]; the second map's lie n_q behind.
__device__ inline float2 *sum_row(const DiffProblem &p, int w, const Row &row)
{
    return reinterpret_cast<float2 *>(p.sums) +
           (int64_t(w) * 2 * p.H + 2 * row.head) * p.nq + row.token;
}

// What is kept of a row for the backward pass, in fp32: the second map's output, and
// where O itself is rounded to bf16 the first one's, in [W][H][n_q][1 or 2][d_v].
template <class E>
__device__ inline float *map_row(const DiffProblem &p, int w, const Row &row)
{
    return p.maps + ((int64_t(w) * p.H + row.head) * p.nq + row.token) *
                        (E::bytes == 2 ? 2 * p.dv : p.dv);
}

// O from the two maps' outputs.  The difference is not fused with a product that gave its
// terms, so that equal maps cancel exactly.
__device__ inline float difference(float x, float lam, float y)
{
#pragma clang fp contract(off)
    return x - lam * y;
}

// The transposed tile's register r: its row.
__device__ inline int reg_row(int r, int g) { return 8 * (r >> 2) + 4 * g + (r & 3); }

// Scores of keys that a row does not see, in a tile of S^T.
__device__ inline void hide(f16v &s, int limit, int k0, int g)
{
#pragma unroll
    for (int r = 0; r < 16; ++r)
        s[r] = k0 + reg_row(r, g) < limit ? s[r] : -INFINITY;
}

// Online softmax of a 32 x 32 tile of S^T: s becomes exp2(scale2 s - m) and l the running
// sum of this lane's keys.  m, the exponents' base, follows the running maximum only when
// some row's has outgrown it by 2^8 (fp32 sums and bf16 terms keep their relative precision
// below that), and `grow(alpha)` then rescales what was summed: with every new maximum
// that would be in nearly every tile.
template <class Grow>
__device__ inline void softmax_step(f16v &s, float scale2, float &m, float &l, Grow grow)
{
    float t = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r)
        t = fmaxf(t, s[r]);
    t = half_max(t) * scale2;
    if (__any(t > m + 8.f)) {
        const float mn = fmaxf(m, t);
        // A row that has seen no key yet has nothing to rescale.
        const float alpha = mn == -INFINITY ? 1.f : fast_exp2(m - mn);
        l *= alpha;
        m = mn;
        grow(alpha);
    }
    const float base = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        s[r] = fast_exp2(fmaf(s[r], scale2, -base));
        sum += s[r];
    }
    l += sum;
}

// Which unit, tile and range a workgroup takes.  Even work: the workgroups of a unit run on
// one XCD (workgroups go to the eight of them in turn), so that its keys and values are
// fetched into one L2 only.  Uneven work (causal masks, lengths): the tiles with the most
// keys of all units first, over all XCDs.
struct Place {
    unsigned unit;
    int tile, split;
};

// All in 32 bits (a launch has fewer than 2^24 workgroups): a division of 64 bits is over a
// hundred instructions.
__device__ inline Place place(const DiffProblem &p, unsigned b, unsigned n, unsigned tiles,
                              unsigned splits, bool last_first)
{
    unsigned unit, tile, split;
    if (p.even) {
        const unsigned per = n / 8, full = per * 8;
        b = b < full ? (b % 8) * per + b / 8 : b;
        const unsigned rest = b / splits;
        split = b - rest * splits;
        unit = rest / tiles;
        tile = rest - unit * tiles;
    } else {
        const unsigned units = unsigned(p.W) * unsigned(p.G);
        const unsigned rest = b / units;
        unit = b - rest * units;
        tile = rest / splits;
        split = rest - tile * splits;
        if (last_first)
            tile = tiles - 1 - tile;
    }
    return Place{unit, int(tile), int(split)};
}

// Buffers of LDS for the tiles: two, or one where the next tile waits in registers and two
// would leave SIMDs empty: workgroups of one wave, and of two in fp32, whose tile of three
// terms takes up to 48 KB of a CU's 160.
template <class E, int NT, int DIRECT>
constexpr int buffers()
{
    return !DIRECT && (NT == 64 || (E::bytes == 4 && NT == 128)) ? 1 : 2;
}

// Keys and values of a unit, tile after tile of KT keys, into the LDS buffers in turn:
// fetch() starts on a tile, commit() ends it after the work on the one before, and ready()
// is the barrier behind which it may be read.
template <class E, int DK, int DV, int NT, int DIRECT>
struct KeyTiles {
    static constexpr int KT = 32;
    using T = typename E::T;
    using LK = Tile<E, DK>;
    using LV = Tile<E, DV>;
    // One buffer in LDS: the keys of both maps, then the values.
    static constexpr uint32_t kV = 2 * LK::kBytes, kBuffer = kV + LV::kBytes;
    static constexpr int kBuffers = buffers<E, NT, DIRECT>();
    Stage<E, DK, 2 * KT, NT> k;   // both maps, one under the other
    Stage<E, DV, KT, NT> v;

    __device__ inline void fetch(const DiffProblem &p, const T *k0, const T *v0, int key, int end,
                                 uint32_t to)
    {
        const int last = end - key - 1;
        k0 += key * p.k.token;
        v0 += key * p.v.token;
        if constexpr (DIRECT) {
            const int kh = int(p.k.head), kt = int(p.k.token), vt = int(p.v.token);
            direct_tile<DK, 2 * KT, NT, DIRECT>(
                to, k0, [&](int row) { return (row / KT) * kh + min(row % KT, last) * kt; },
                p.d);
            direct_tile<DV, KT, NT, DIRECT>(to + kV, v0,
                                            [&](int row) { return min(row, last) * vt; }, p.dv);
        } else {
            k.load([&](int row) { return k0 + (row / KT) * p.k.head + (row % KT) * p.k.token; },
                   [&](int row) { return row % KT <= last; }, p.d);
            v.load([&](int row) { return v0 + row * p.v.token; },
                   [&](int row) { return row <= last; }, p.dv);
        }
    }

    __device__ inline void commit(uint32_t to) const
    {
        if constexpr (!DIRECT) {
            k.store(to);
            v.store(to + kV);
        }
    }

    __device__ static inline void ready()
    {
        if constexpr (DIRECT)
            arrived();
        __syncthreads();
    }

    // Before commit(): where there is one buffer the work on it has to be done.
    __device__ static inline void vacate()
    {
        if constexpr (kBuffers == 1)
            __syncthreads();
    }
};

// Nothing is scheduled across: without it the operands of several products are fetched
// ahead of the first, which takes more registers than two waves to a SIMD leave.
__device__ inline void part() { __builtin_amdgcn_sched_barrier(0); }

// Waves to a SIMD that the kernels are compiled for: two, whose matrix instructions and
// exponentials run beside each other, or one for kernels with `more` to hold than 256
// registers: at full width, or fp32, whose operands take three terms; at full width fp32
// always.
template <class E, int DV>
constexpr int occupancy(bool more)
{
    return DV == 128 ? (E::bytes == 4 || more ? 1 : 2) : (E::bytes == 4 && more ? 1 : 2);
}

// ---- host side ----------------------------------------------------------------

// Whether every row of a tensor starts and ends on a multiple of `to` bytes.
inline bool aligned(const DiffView &v, int width, int bytes, int to)
{
    return uintptr_t(v.data) % to == 0 &&
           (v.window | v.head | v.token | width) * bytes % to == 0;
}

// Whether tiles can be loaded to LDS directly: bf16 rows of whole and aligned groups of
// `bytes`, and `span` elements, those of a tile or of a unit, within 32-bit offsets.
// 16 bytes where they fit; 4 otherwise, which still beat the way through registers: 256 x 6
// windows of 256 tokens of 30 / 60, dQ 168 instead of 221 us, dK, dV 172 instead of 215 us;
// 4 x 6 causal heads of 1024 tokens of 46 / 92, 57 instead of 103 us and 55 instead of 102 us.
inline bool direct(const DiffProblem &p, const DiffView &v, int width, int64_t span,
                   int bytes = 16)
{
    return p.dtype == 1 && aligned(v, width, 2, bytes) && span < (int64_t(1) << 30);
}

// Whether groups of four elements may be stored at once.
inline bool store_vec(const DiffView &v, int width, int bytes)
{
    return uintptr_t(v.data) % (4 * bytes) == 0 && ((v.window | v.head | v.token | width) % 4) == 0;
}

inline int ceil_div(int64_t a, int64_t b) { return int((a + b - 1) / b); }

inline int round4(int n) { return (n + 3) / 4 * 4; }

// Waves to a workgroup: as many as there are tiles of 32 rows (or keys), at most four.
inline int waves_for(int64_t rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : 4; }

// Widths are padded to 32 (queries, keys) and 64 (values) or to 64 and 128.
inline bool narrow(const DiffProblem &p) { return p.d <= 32 && p.dv <= 64; }

inline void set_common(DiffProblem *p)
{
    // With many units uneven work evens out, and each still has an L2 to itself.
    p->even = (p->causal == 0 && !p->kv_len) || int64_t(p->W) * p->G >= 512;
    p->nq_shift = 31 + (31 - __builtin_clz(unsigned(p->nq)));
    p->nq_mul = uint32_t(((uint64_t(1) << p->nq_shift) + p->nq - 1) / p->nq);
}

}  // namespace diff
}  // namespace nystra
