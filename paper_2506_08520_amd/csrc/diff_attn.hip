// Forward pass of differential attention (the formulas stand in diff_common.hpp).
//
// One walk over the keys with the running maximum and sum of both maps, whose outputs stay
// apart in registers (each has its own maximum).  Two or three waves to a SIMD (fp32 at full
// width: one): one's matrix instructions run beside the other's exponentials.  Keys are split over workgroups where
// there are few rows.  Measured: 2 x 8 heads of 4096 tokens of 64 / 128 in bf16 251 us, the
// matrix cores busy for 44 % of the time (the rest are exponentials and waits for LDS);
// 256 x 6 of 256 tokens of 32 / 64 79 us, 26 %; 1024 x 6 of 64 tokens of 30 / 60 50 us,
// bound by memory (203 MB, 4.1 TB/s) and by the latency of two tiles; 16 tokens of 16 heads
// over 4 x 8192 keys at most 42 us, bound by memory (169 MB, 4.0 TB/s), and 5 us for the
// merge; 5 x 8 causal heads of 777 tokens of 44 / 88 in fp32 110 and 13 us.
#include <algorithm>

#include "diff_common.hpp"

namespace nystra {
namespace {

using namespace diff;

constexpr int kMerge = 256;       // threads of the merge kernel: one row
constexpr int kFewSplits = 8;

// Waves to a SIMD that the kernel is compiled for.
// Narrow workgroups of two waves (up to 64 rows, the windows' form) whose tiles need no
// registers on their way: three, since all of them wait for the same two tiles.  Those with
// 16-byte loads fit by themselves; those with 4-byte loads keep five registers in memory for
// it: 1024 x 6 windows of 64 tokens of 14 / 28 take 34 instead of 41 us at two waves, of 22 / 44
// 45 instead of 50, of 30 / 60 54 instead of 56, of 49 tokens of 30 / 60 49 instead of 54.
// Single waves that stage their tiles in registers: one, for the token form (16 x 16 heads over
// 4 x 2048 keys of 31 / 62 in fp32 44 instead of 52 us at two; 6144 windows of 32 tokens of
// 31 / 61 in fp32 99 instead of 91, of 63 / 127 in bf16 126 instead of 111, of 16 tokens 77
// instead of 91).
template <class E, int DV, int NW, int DIRECT>
constexpr int forward_occupancy()
{
    if (NW == 1 && !DIRECT)
        return 1;
    if (NW == 2 && DV == 64)
        return DIRECT ? 3 : occupancy<E, DV>(true);
    return occupancy<E, DV>(false);
}

// DIRECT: the bytes of the loads that bring keys and values to LDS (16 or 4), or 0 where
// registers stage them.
template <class E, int DK, int DV, int NW, int DIRECT>
__global__ void __launch_bounds__(64 * NW, (forward_occupancy<E, DV, NW, DIRECT>()))
diff_forward_kernel(DiffProblem p)
{
    using T = typename E::T;
    using Tiles = KeyTiles<E, DK, DV, 64 * NW, DIRECT>;
    constexpr int KT = Tiles::KT;
    __shared__ alignas(256) char lds[Tiles::kBuffers * Tiles::kBuffer];
    const uint32_t buf = lds_offset(lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5, c = lane & 31;
    const Place here = place(p, blockIdx.x, gridDim.x, p.tiles, p.splits, true);
    const int64_t unit = here.unit;
    const int w = int(here.unit / unsigned(p.G)), kvh = int(here.unit) - w * p.G;
    const int tile = here.tile, split = here.split;
    const int nrows = p.R * p.nq;
    const int r0 = tile * 32 * NW, r = r0 + wave * 32 + c;
    const bool live = r < nrows;
    const Row row = row_of(p, kvh, live ? r : r0);
    const int len = window_len(p, w);
    const int r1 = min(r0 + 32 * NW, nrows) - 1;
    const int kbegin = split * p.chunk;
    const int kend = min(tile_limit(p, len, r0, r1), kbegin + p.chunk);
    const int limit = min(live ? key_limit(p, len, row.token) : 0, kend);
    const T *k0 = at<E>(p.k, w, 2 * kvh, 0), *v0 = at<E>(p.v, w, kvh, 0);

    Tiles tiles;
    if (kbegin < kend)
        tiles.fetch(p, k0, v0, kbegin, kend, buf);
    Frag<E> q[2][DK / 16];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        const T *src = at<E>(p.q, w, 2 * row.head + a, row.token);
#pragma unroll
        for (int i = 0; i < DK / 16; ++i)
            q[a][i] = as_frag(load_chunk<E, DIRECT == 16>(src + 16 * i + 8 * g,
                                                       p.d - 16 * i - 8 * g, live, p.d));
    }
    f16v acc[2][DV / 32] = {};
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    if (kbegin < kend)
        tiles.commit(buf);

    // This tile's buffer and the next one's.
    uint32_t t = buf, other = buf + (Tiles::kBuffers - 1) * Tiles::kBuffer;
    for (int key = kbegin; key < kend; key += KT) {
        Tiles::ready();
        const bool more = key + KT < kend;
        if (more)
            tiles.fetch(p, k0, v0, key + KT, kend, other);
        if (__any(key < limit)) {
            const uint32_t krow = first_row<E, DK>(t), vcol = first_col<E, DV>(t + Tiles::kV);
            f16v s[2] = {};
#pragma unroll
            for (int i = 0; i < DK / 16; ++i)
#pragma unroll
                for (int a = 0; a < 2; ++a)
                    s[a] = mma(row_frag<E, DK>(krow + a * Tiles::LK::kBytes, i), q[a][i], s[a]);
            part();
            if (!__all(key + KT <= limit)) {
                hide(s[0], limit, key, g);
                hide(s[1], limit, key, g);
            }
#pragma unroll
            for (int a = 0; a < 2; ++a)
                softmax_step(s[a], p.scale2, m[a], l[a], [&](float alpha) {
#pragma unroll
                    for (int i = 0; i < DV / 32; ++i)
                        acc[a][i] *= alpha;
                });
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Frag<E> p1 = frag_of(s[0], h, E()), p2 = frag_of(s[1], h, E());
#pragma unroll
                for (int i = 0; i < DV / 32; ++i) {
                    const Frag<E> v = col_frag<E, DV>(vcol, h, i);
                    acc[0][i] = mma(v, p1, acc[0][i]);
                    acc[1][i] = mma(v, p2, acc[1][i]);
                }
            }
        }
        if (more) {
            Tiles::vacate();
            tiles.commit(other);
        }
        exchange(t, other);
    }
#pragma unroll
    for (int a = 0; a < 2; ++a)
        l[a] = half_sum(l[a]);
    if (!live)
        return;
    if (p.splits > 1) {
        float *out = p.partial + ((unit * p.splits + split) * nrows + r) * p.partial_row;
#pragma unroll
        for (int a = 0; a < 2; ++a) {
#pragma unroll
            for (int i = 0; i < DV / 32; ++i)
                store_block<F32>(out + a * p.dv4, i, g, p.dv4, true, acc[a][i]);
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
    float *maps = p.maps ? map_row<E>(p, w, row) : nullptr;
    const bool maps4 = p.dv % 4 == 0;
#pragma unroll
    for (int i = 0; i < DV / 32; ++i) {
        f16v &x = acc[0][i], &y = acc[1][i], o16;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            x[r] *= inv1;
            y[r] *= inv2;
            o16[r] = difference(x[r], lam, y[r]);
        }
        store_block<E>(o, i, g, p.dv, p.store_o, o16);
        if (maps) {
            store_block<F32>(maps, i, g, p.dv, maps4, y);
            if (E::bytes == 2)
                store_block<F32>(maps + p.dv, i, g, p.dv, maps4, x);
        }
    }
    if (p.sums && g == 0) {
        float2 *sums = sum_row(p, w, row);
        sums[0] = make_float2(m[0], l[0]);
        sums[p.nq] = make_float2(m[1], l[1]);
    }
}

// Joins few key ranges, a thread to four columns of a row: each forms the weights itself.  A
// range without a key has a sum of zero; one whose scores are all NaN has no maximum either,
// but a sum of NaN, which has to reach the output.
template <class E>
__global__ void __launch_bounds__(kMerge)
diff_merge_few_kernel(DiffProblem p, int64_t items)
{
    const int64_t item = int64_t(blockIdx.x) * kMerge + threadIdx.x;
    if (item >= items)
        return;
    const int nrows = p.R * p.nq, groups = p.dv4 / 4;
    // below 2^24 rows of at most 32 groups
    const unsigned at_row = unsigned(item) / unsigned(groups);
    const int col = int(unsigned(item) - at_row * groups) * 4;
    const int64_t unit = at_row / unsigned(nrows);
    const int r = int(at_row - unsigned(unit) * nrows);
    const int w = int(unsigned(unit) / unsigned(p.G)), kvh = int(unit) - w * p.G;
    const Row row = row_of(p, kvh, r);
    const float *part = p.partial + (unit * p.splits * nrows + r) * p.partial_row;
    const int64_t step = int64_t(nrows) * p.partial_row;
    f4 ml[kFewSplits];
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int s = 0; s < kFewSplits; ++s) {
        const f4 none = {-INFINITY, 0.f, -INFINITY, 0.f};
        ml[s] = s < p.splits ? *reinterpret_cast<const f4 *>(part + s * step + 2 * p.dv4) : none;
        m[0] = fmaxf(m[0], ml[s][0]);
        m[1] = fmaxf(m[1], ml[s][2]);
    }
    f4 x[2] = {};
#pragma unroll
    for (int s = 0; s < kFewSplits; ++s)
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            if (ml[s][2 * a + 1] != 0.f) {
                const float e = fast_exp2(ml[s][2 * a] - m[a]);
                l[a] = fmaf(e, ml[s][2 * a + 1], l[a]);
                x[a] += e * *reinterpret_cast<const f4 *>(part + s * step + a * p.dv4 + col);
            }
        }
#pragma unroll
    for (int a = 0; a < 2; ++a)
        x[a] *= l[a] == 0.f ? 0.f : 1.f / l[a];
    const float lam = p.lambda[row.head];
    f4 o;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        o[j] = difference(x[0][j], lam, x[1][j]);
    store4<E>(at_out<E>(p.o, w, row.head, row.token), col, p.dv, p.store_o, o);
    if (p.maps) {
        float *maps = map_row<E>(p, w, row);
        store4<F32>(maps, col, p.dv, p.dv % 4 == 0, x[1]);
        if (E::bytes == 2)
            store4<F32>(maps + p.dv, col, p.dv, p.dv % 4 == 0, x[0]);
    }
    if (p.sums && col == 0) {
#pragma unroll
        for (int a = 0; a < 2; ++a)
            sum_row(p, w, row)[a * p.nq] = make_float2(m[a], l[a]);
    }
}

// Joins the key ranges of one row, a thread to a column of either map: as the softmax
// itself, one pass with a running maximum, kBatch ranges' values in flight at a time.
template <class E>
__global__ void __launch_bounds__(kMerge)
diff_merge_kernel(DiffProblem p)
{
    constexpr int kBatch = 16;
    __shared__ float out[2][128];
    const int nrows = p.R * p.nq;
    const int64_t unit = blockIdx.x / unsigned(nrows);
    const int r = int(blockIdx.x - unit * nrows);
    const int w = int(unsigned(unit) / unsigned(p.G)), kvh = int(unit) - w * p.G;
    const Row row = row_of(p, kvh, r);
    const float *part = p.partial + (unit * p.splits * nrows + r) * p.partial_row;
    const int64_t step = int64_t(nrows) * p.partial_row;
    const int i = threadIdx.x, a = i >= p.dv4;   // 2 dv4 <= kMerge columns
    if (i < 2 * p.dv4) {
        const float *ml = part + 2 * p.dv4 + 2 * a;
        float m = -INFINITY, l = 0.f, x = 0.f;
        for (int s0 = 0; s0 < p.splits; s0 += kBatch) {
            float mb[kBatch], lb[kBatch], xb[kBatch];
            float mn = m;
#pragma unroll
            for (int s = 0; s < kBatch; ++s) {
                const int64_t at = min(s0 + s, p.splits - 1) * step;
                mb[s] = ml[at];
                lb[s] = ml[at + 1];
                xb[s] = part[at + i];
            }
#pragma unroll
            for (int s = 0; s < kBatch; ++s)
                mn = fmaxf(mn, mb[s]);
            const float alpha = m == mn ? 1.f : fast_exp2(m - mn);
            l *= alpha;
            x *= alpha;
            m = mn;
#pragma unroll
            for (int s = 0; s < kBatch; ++s) {
                if (s0 + s < p.splits && lb[s] != 0.f) {   // as above
                    const float e = fast_exp2(mb[s] - m);
                    l = fmaf(e, lb[s], l);
                    x = fmaf(e, xb[s], x);
                }
            }
        }
        out[a][i - a * p.dv4] = l == 0.f ? 0.f : x / l;
        if (p.sums && i == a * p.dv4)
            sum_row(p, w, row)[a * p.nq] = make_float2(m, l);
    }
    __syncthreads();
    const float lam = p.lambda[row.head];
    typename E::T *o = at_out<E>(p.o, w, row.head, row.token);
    float *maps = p.maps ? map_row<E>(p, w, row) : nullptr;
    for (int col = threadIdx.x; col < p.dv; col += kMerge) {
        E::store(o, col, difference(out[0][col], lam, out[1][col]));
        if (maps) {
            maps[col] = out[1][col];
            if (E::bytes == 2)
                maps[p.dv + col] = out[0][col];
        }
    }
}

// ---- dispatch -----------------------------------------------------------------

struct Plan {
    int waves, tiles, splits, chunk;
    int64_t blocks;
};

// Key ranges: with few rows enough of them for eight waves on each of the 256 CUs, of at
// least one tile to a wave.  Workgroups of more waves are split only below one to a CU, or
// three under a causal mask, where the longest ones would be waited for.
Plan forward_plan(const DiffProblem &p)
{
    Plan f;
    const int64_t rows = int64_t(p.R) * p.nq;
    f.waves = waves_for(rows);
    f.tiles = ceil_div(rows, 32 * f.waves);
    const int64_t blocks = int64_t(p.W) * p.G * f.tiles;
    const int64_t want = f.waves == 1 ? (2048 + blocks - 1) / blocks
                                      : (p.causal == 0 ? 1 : 3) * 1024 / f.waves / blocks;
    const int64_t most = ceil_div(p.nk, 32 * f.waves);
    f.splits = int(std::max<int64_t>(std::min(want, most), 1));
    f.chunk = ceil_div(ceil_div(p.nk, f.splits), 32) * 32;
    f.splits = ceil_div(p.nk, f.chunk);
    f.blocks = blocks * f.splits;
    return f;
}

template <class E, int DK, int DV, int NW>
void run(const DiffProblem &p, const Plan &f, hipStream_t s)
{
    const dim3 grid(unsigned(f.blocks));
    if constexpr (E::bytes == 2) {
        if (direct(p, p.q, p.d, 0) && direct(p, p.k, p.d, p.k.head + 32 * p.k.token) &&
            direct(p, p.v, p.dv, 32 * p.v.token)) {
            diff_forward_kernel<E, DK, DV, NW, 16><<<grid, 64 * NW, 0, s>>>(p);
            return;
        }
        if (direct(p, p.k, p.d, p.k.head + 32 * p.k.token, 4) &&
            direct(p, p.v, p.dv, 32 * p.v.token, 4)) {
            diff_forward_kernel<E, DK, DV, NW, 4><<<grid, 64 * NW, 0, s>>>(p);
            return;
        }
    }
    diff_forward_kernel<E, DK, DV, NW, 0><<<grid, 64 * NW, 0, s>>>(p);
}

template <class E, int DK, int DV>
void run_waves(const DiffProblem &p, const Plan &f, hipStream_t s)
{
    if (f.waves == 1)
        run<E, DK, DV, 1>(p, f, s);
    else if (f.waves == 2)
        run<E, DK, DV, 2>(p, f, s);
    else
        run<E, DK, DV, 4>(p, f, s);
}

template <class E>
void run_any(const DiffProblem &p, const Plan &f, hipStream_t s)
{
    narrow(p) ? run_waves<E, 32, 64>(p, f, s) : run_waves<E, 64, 128>(p, f, s);
}

}  // namespace

bool diff_grid_fits(const DiffProblem &p)
{
    const int64_t rows = int64_t(p.R) * p.nq, units = int64_t(p.W) * p.G;
    // The largest grids: one wave to 32 rows or keys over one split, and the merges' rows
    // (the keys are merged for fewer than 512 workgroups of up to 128).
    const int64_t most = units * ((rows + 31) / 32 + (p.nk + 31) / 32) + units * rows;
    return rows < (int64_t(1) << 30) && most < (int64_t(1) << 24);
}

size_t diff_forward_workspace(const DiffProblem &p)
{
    const Plan f = forward_plan(p);
    const int64_t row = 2 * round4(p.dv) + 4;
    return f.splits > 1
               ? size_t(int64_t(p.W) * p.G * f.splits * p.R * p.nq * row) * sizeof(float)
               : 0;
}

hipError_t launch_diff_forward(DiffProblem p, void *workspace, hipStream_t s)
{
    const Plan f = forward_plan(p);
    set_common(&p);
    p.store_o = store_vec(p.o, p.dv, p.dtype == 0 ? 4 : 2);
    p.tiles = f.tiles;
    p.splits = f.splits;
    p.chunk = f.chunk;
    p.partial = static_cast<float *>(workspace);
    p.dv4 = round4(p.dv);
    p.partial_row = 2 * p.dv4 + 4;
    p.dtype == 0 ? run_any<F32>(p, f, s) : run_any<BF16>(p, f, s);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess || f.splits == 1)
        return err;
    const int64_t rows = int64_t(p.W) * p.G * p.R * p.nq;
    if (f.splits <= kFewSplits) {
        const int64_t items = rows * (p.dv4 / 4);
        const dim3 grid(unsigned((items + kMerge - 1) / kMerge));
        if (p.dtype == 0)
            diff_merge_few_kernel<F32><<<grid, kMerge, 0, s>>>(p, items);
        else
            diff_merge_few_kernel<BF16><<<grid, kMerge, 0, s>>>(p, items);
        return hipGetLastError();
    }
    const dim3 grid{unsigned(rows)};
    if (p.dtype == 0)
        diff_merge_kernel<F32><<<grid, kMerge, 0, s>>>(p);
    else
        diff_merge_kernel<BF16><<<grid, kMerge, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace nystra
