// Backward pass of differential attention, first half: dQ, row by row (the formulas stand
// in diff_common.hpp).
//
// Measured (sizes as in the forward pass): 4096 tokens 269 us, the matrix cores busy for
// 41 % of the time, 256 tokens 147 us, 23 %, both bound by two waves to a SIMD that wait for LDS
// and for each other's products; 777 tokens in fp32 146 us, one wave to a SIMD, 26 %.

#include "diff_common.hpp"

namespace nystra {
namespace {

using namespace diff;

// Sum of the products of eight elements and eight fp32 values.
template <class E>
__device__ inline float dot8(const Chunk<E> &a, const Chunk<F32> &b)
{
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t u = E::bytes == 4 ? a.w[j * E::bytes / 4]
                           : j & 1       ? a.w[j / 2] & 0xffff0000u
                                         : a.w[j / 2] << 16;
        s = fmaf(__uint_as_float(u), __uint_as_float(b.w[j]), s);
    }
    return s;
}

// dQ, and per row D_1, D_2 and -dlam.  Rows as in the forward pass.  The exponentials are
// the forward pass's, bit by bit, and their sums divide what is formed from them, so that
// every row's probabilities add up to one and dlam, a sum of both signs, keeps its digits.
//
// D_a comes from the maps' outputs, D_2 = dO . O_2 and D_1 = dO . O_1 (fp32: dO . O +
// lam D_2), which the forward pass keeps in fp32 (from outputs rounded to bf16, dQ was off
// by 0.0030 of its norm at 4096 keys where rounding it alone costs 0.0017), or, where it kept
// none (bf16 up to 256 keys), from a first walk over the keys: at 16 x 16 windows with heads
// of 32 / 64 that made the forward pass 120 -> 79 us and this one 139 -> 146 us, by 400 MB
// less of traffic; at 512 keys the walk would cost more than it saves, and fp32 with its six
// products always.  Forward and backward pass of 393216 rows with the walk and without:
// 64 keys of 32 / 64 193 and 302 us, of 64 / 128 (where the walk leaves one wave to a SIMD)
// 439 and 647; 128 keys 228 and 315, 507 and 628; 256 keys 313 and 360, 674 and 697; but of
// 44 / 88, which 4-byte loads bring, 524 and 596 at 128 keys, 734 and 695 at 256.
// DIRECT as in the forward pass.
template <class E, int DK, int DV, int NW, int DIRECT, bool KEPT>
__global__ void __launch_bounds__(64 * NW, (occupancy<E, DV>(!KEPT || E::bytes == 4)))
diff_dq_kernel(DiffProblem p)
{
    using T = typename E::T;
    using Tiles = KeyTiles<E, DK, DV, 64 * NW, DIRECT>;
    constexpr int KT = Tiles::KT;
    // The row's part of -dlam is dO . O_2 = D_2.  bf16 forms it here from the probabilities,
    // where O_2 came from their roundings (323 keys: dlam off by 1.5e-3 from O_2, 4.8e-7 so).
    // fp32 takes the kept O_2: the matrix instruction's sums round towards one side, which
    // dO . V carries into every row alike (777 keys: 1.5e-6 from dO . V, 1.6e-7 so).
    constexpr bool kSumLambda = KEPT && E::bytes == 2;
    __shared__ alignas(256) char lds[Tiles::kBuffers * Tiles::kBuffer];
    const uint32_t buf = lds_offset(lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5, c = lane & 31;
    const Place here = place(p, blockIdx.x, gridDim.x, p.tiles, p.splits, true);
    const int64_t unit = here.unit;
    const int w = int(here.unit / unsigned(p.G)), kvh = int(here.unit) - w * p.G;
    const int tile = here.tile;
    const int nrows = p.R * p.nq;
    const int r0 = tile * 32 * NW, r = r0 + wave * 32 + c;
    const bool live = r < nrows;
    const Row row = row_of(p, kvh, live ? r : r0);
    const int len = window_len(p, w);
    const int limit = live ? key_limit(p, len, row.token) : 0;
    // What a row without keys holds has no effect: it counts as zeros.
    const bool seeing = limit > 0;
    const int r1 = min(r0 + 32 * NW, nrows) - 1;
    const int kbegin = here.split * p.chunk;
    const int kend = min(tile_limit(p, len, r0, r1), kbegin + p.chunk);
    const float lam = p.lambda[row.head];
    const T *k0 = at<E>(p.k, w, 2 * kvh, 0), *v0 = at<E>(p.v, w, kvh, 0);

    Tiles tiles;
    if (kend > kbegin)
        tiles.fetch(p, k0, v0, kbegin, kend, buf);
    Frag<E> q[2][DK / 16], go[DV / 16];
    float base[2], inv[2], D[2] = {0.f, 0.f};
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        const T *src = at<E>(p.q, w, 2 * row.head + a, row.token);
#pragma unroll
        for (int i = 0; i < DK / 16; ++i)
            q[a][i] = as_frag(load_chunk<E, DIRECT == 16>(src + 16 * i + 8 * g,
                                                       p.d - 16 * i - 8 * g, seeing, p.d));
        const float2 sum = sum_row(p, w, row)[a * p.nq];
        base[a] = seeing ? sum.x : INFINITY;   // exp2(-inf) = 0 where no key is seen
        inv[a] = seeing && sum.y != 0.f ? 1.f / sum.y : 0.f;
    }
    const T *gosrc = at<E>(p.go, w, row.head, row.token);
#pragma unroll
    for (int i = 0; i < DV / 16; ++i)
        go[i] = as_frag(load_chunk<E, DIRECT == 16>(gosrc + 16 * i + 8 * g, p.dv - 16 * i - 8 * g,
                                                 seeing, p.dv));
    if constexpr (KEPT) {
        const float *o2 = map_row<E>(p, w, row);
        const float *o1 = E::bytes == 2 ? o2 + p.dv : at<F32>(p.o, w, row.head, row.token);
#pragma unroll 2   // more would hold more of the rows at once than there are registers
        for (int col = 8 * g; col < p.dv; col += 16) {
            const int n = p.dv - col;
            const Chunk<E> x = load_chunk<E, DIRECT == 16>(gosrc + col, n, seeing, p.dv);
            D[0] += dot8(x, load_chunk<F32, false>(o1 + col, n, seeing, p.dv));
            D[1] += dot8(x, load_chunk<F32, false>(o2 + col, n, seeing, p.dv));
        }
        if (E::bytes == 4)
            D[0] = fmaf(lam, D[1], D[0]);
#pragma unroll
        for (int a = 0; a < 2; ++a)
            D[a] = half_sum(D[a]);
    }
    const float w1 = inv[0], w2 = -lam * inv[1];
    f16v acc[2][DK / 32] = {};
    float glam = 0.f;   // bf16 with kept maps; D_2 where that is as exact
    if (kend > kbegin)
        tiles.commit(buf);
    // This tile's buffer and the next one's.
    uint32_t t = buf, other = buf + (Tiles::kBuffers - 1) * Tiles::kBuffer;
    for (int sweep = KEPT ? 1 : 0; sweep < 2; ++sweep) {
        float sum[2] = {0.f, 0.f};
        for (int key = kbegin; key < kend; key += KT) {
            Tiles::ready();
            const bool wrap = key + KT >= kend, more = !wrap || sweep == 0;
            if (more)
                tiles.fetch(p, k0, v0, wrap ? kbegin : key + KT, kend, other);
            if (__any(key < limit)) {
                const uint32_t krow = first_row<E, DK>(t), kcol = first_col<E, DK>(t);
                const uint32_t vrow = first_row<E, DV>(t + Tiles::kV);
                constexpr uint32_t kMap = Tiles::LK::kBytes;
                f16v s[2] = {}, x = {};
#pragma unroll
                for (int i = 0; i < DK / 16; ++i)
#pragma unroll
                    for (int a = 0; a < 2; ++a)
                        s[a] = mma(row_frag<E, DK>(krow + a * kMap, i), q[a][i], s[a]);
                part();
#pragma unroll
                for (int i = 0; i < DV / 16; ++i)
                    x = mma(row_frag<E, DV>(vrow, i), go[i], x);
                part();
                if (!__all(key + KT <= limit)) {
                    hide(s[0], limit, key, g);
                    hide(s[1], limit, key, g);
                }
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        s[a][i] = fast_exp2(fmaf(s[a][i], p.scale2, -base[a]));
                if (sweep == 0) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        sum[0] = fmaf(s[0][i], x[i], sum[0]);
                        sum[1] = fmaf(s[1][i], x[i], sum[1]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        // the sums of the exponentials divide the other factor
                        if (kSumLambda)
                            glam = fmaf(s[1][i], x[i], glam);
                        s[0][i] *= fmaf(w1, x[i], -w1 * D[0]);
                        s[1][i] *= fmaf(w2, x[i], -w2 * D[1]);
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int a = 0; a < 2; ++a) {
                            const Frag<E> ds = frag_of(s[a], h, E());
#pragma unroll
                            for (int i = 0; i < DK / 32; ++i)
                                acc[a][i] = mma(col_frag<E, DK>(kcol + a * kMap, h, i), ds, acc[a][i]);
                        }
                }
            }
            if (more) {
                Tiles::vacate();
                tiles.commit(other);
            }
            exchange(t, other);
        }
        if (sweep == 0) {
#pragma unroll
            for (int a = 0; a < 2; ++a)
                D[a] = half_sum(sum[a]) * inv[a];
        }
    }
    glam = kSumLambda ? half_sum(glam) * inv[1] : D[1];
    // What the dK, dV kernel needs of a row, also for those up to the end of the last tile
    // of 32.
    if (g == 0 && here.split == 0 && r < p.rows32) {
        p.row_stats[unit * p.rows32 + r] =
            seeing ? make_float4(base[0] - log2f(inv[0]), base[1] - log2f(inv[1]), D[0], D[1])
                   : make_float4(INFINITY, INFINITY, 0.f, 0.f);
        p.row_lambda[unit * p.rows32 + r] = lam;
    }
    if (!live)
        return;
    if (p.splits > 1) {
        float *out = p.partial + ((unit * p.splits + here.split) * nrows + r) * p.dq_row;
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int i = 0; i < DK / 32; ++i)
                store_block<F32>(out + a * p.d4, i, g, p.d4, true, acc[a][i]);
        if (g == 0)
            out[2 * p.d4] = kSumLambda || here.split == 0 ? glam : 0.f;
        return;
    }
    if (g == 0)
        p.rows_lam[unit * nrows + r] = glam;
    // A softmax over one key is constant: its gradient is zero, not the rounding of D.
    const float scale = limit == 1 ? 0.f : p.scale;
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        T *dst = at_out<E>(p.gq, w, 2 * row.head + a, row.token);
#pragma unroll
        for (int i = 0; i < DK / 32; ++i)
            store_block<E>(dst, i, g, p.d, p.vec_gq, acc[a][i], scale);
    }
}

// Adds up the key ranges of one row.
template <class E>
__global__ void __launch_bounds__(64) diff_dq_merge_kernel(DiffProblem p)
{
    const unsigned nrows = unsigned(p.R) * unsigned(p.nq);
    const int64_t unit = blockIdx.x / nrows;
    const int r = int(blockIdx.x - unit * nrows);
    const int w = int(unsigned(unit) / unsigned(p.G)), kvh = int(unit) - w * p.G;
    const Row row = row_of(p, kvh, r);
    const float scale = key_limit(p, window_len(p, w), row.token) == 1 ? 0.f : p.scale;
    const float *part = p.partial + (unit * p.splits * nrows + r) * p.dq_row;
    const int64_t step = int64_t(nrows) * p.dq_row;
    for (int col = threadIdx.x; col <= 2 * p.d4; col += 64) {
        float s = 0.f;
#pragma unroll 8
        for (int i = 0; i < p.splits; ++i)
            s += part[i * step + col];
        const int a = col >= p.d4, at_col = col - a * p.d4;
        if (col == 2 * p.d4)
            p.rows_lam[unit * nrows + r] = s;
        else if (at_col < p.d)
            E::store(at_out<E>(p.gq, w, 2 * row.head + a, row.token), at_col, scale * s);
    }
}

template <class E, int DK, int DV, int NW, int DIRECT>
void launch(const DiffProblem &p, int64_t blocks, hipStream_t s)
{
    const dim3 grid(unsigned(blocks), 1, 1);
    if constexpr (E::bytes == 2) {
        if (!p.maps) {
            diff_dq_kernel<E, DK, DV, NW, DIRECT, false><<<grid, 64 * NW, 0, s>>>(p);
            return;
        }
    }
    diff_dq_kernel<E, DK, DV, NW, DIRECT, true><<<grid, 64 * NW, 0, s>>>(p);
}

template <class E, int DK, int DV, int NW>
void run(const DiffProblem &p, int64_t blocks, hipStream_t s)
{
    if constexpr (E::bytes == 2) {
        if (direct(p, p.q, p.d, 0) && direct(p, p.go, p.dv, 0) &&
            direct(p, p.k, p.d, p.k.head + 32 * p.k.token) &&
            direct(p, p.v, p.dv, 32 * p.v.token))
            return launch<E, DK, DV, NW, 16>(p, blocks, s);
        if (direct(p, p.k, p.d, p.k.head + 32 * p.k.token, 4) &&
            direct(p, p.v, p.dv, 32 * p.v.token, 4))
            return launch<E, DK, DV, NW, 4>(p, blocks, s);
    }
    launch<E, DK, DV, NW, 0>(p, blocks, s);
}

template <class E>
void run_any(const DiffProblem &p, int waves, int64_t blocks, hipStream_t s)
{
    if (waves == 2)
        narrow(p) ? run<E, 32, 64, 2>(p, blocks, s) : run<E, 64, 128, 2>(p, blocks, s);
    else
        narrow(p) ? run<E, 32, 64, 4>(p, blocks, s) : run<E, 64, 128, 4>(p, blocks, s);
}

}  // namespace

hipError_t launch_diff_dq(const DiffProblem &p, int waves, int64_t blocks, hipStream_t s)
{
    p.dtype == 0 ? run_any<F32>(p, waves, blocks, s) : run_any<BF16>(p, waves, blocks, s);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess || p.splits == 1)
        return err;
    const dim3 rows(unsigned(int64_t(p.W) * p.G * p.R * p.nq));
    if (p.dtype == 0)
        diff_dq_merge_kernel<F32><<<rows, 64, 0, s>>>(p);
    else
        diff_dq_merge_kernel<BF16><<<rows, 64, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace nystra
