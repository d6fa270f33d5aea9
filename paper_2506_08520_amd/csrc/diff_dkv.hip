// Backward pass of differential attention, second half: dK, dV and dlam, key by key, and
// the calls of both halves (the formulas stand in diff_common.hpp).
//
// Measured (sizes as in the forward pass): 4096 tokens 444 us, the matrix cores busy for
// 32 % of the time (six products a tile, of which three meet operands by transposing
// reads of LDS), 256 tokens 147 us, 19 %, of which 311 MB of traffic alone would take 62 us;
// 777 tokens in fp32 145 us and 12 us for adding up the row ranges.
#include <algorithm>
#include <type_traits>

#include "diff_common.hpp"

namespace nystra {

// The first half; p.row_stats and p.rows_lam are its results besides dQ.
hipError_t launch_diff_dq(const DiffProblem &p, int waves, int64_t blocks, hipStream_t s);

namespace {

using namespace diff;

constexpr int kMerge = 64;   // threads of the merge kernel: one key

// dlam of one head: the sum over its rows in all windows, by one workgroup.  The other
// workgroups hide it with three heads and more; 393216 rows of 30 / 60 in windows of 64 take
// 177 us backward with six heads, 175 with three, but 326 with one.
template <int NT>
__device__ inline void sum_dlam(const DiffProblem &p, int h, float *out)
{
    __shared__ float lds[NT / 64];
    float s = 0.f;
    const int n = p.W * p.nq;   // below 2^24
#pragma unroll 8   // loads in flight: the rows are far more than the threads
    for (int i = threadIdx.x; i < n; i += NT) {
        const int w = div_nq(p, i);
        s += p.rows_lam[(int64_t(w) * p.H + h) * p.nq + (i - w * p.nq)];
    }
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0)
        lds[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.f;
        for (int i = 0; i < NT / 64; ++i)
            s += lds[i];
        out[h] = -s;
    }
}

// The factor of dK.  A softmax over one key is constant, as in the dQ kernel; with a causal
// mask the rows that see one key are taken out one by one.
__device__ inline float key_scale(const DiffProblem &p, int len)
{
    return p.causal == 0 && len == 1 ? 0.f : p.scale;
}

// dK and dV: a wave owns 32 keys and walks over the unit's rows, so that the heads
// that share the keys are summed in registers.  Keys at or behind the window's
// length get zeros.  With few workgroups the rows are split over p.rsplits of them, whose
// sums go to the workspace.  The first H workgroups add up dlam meanwhile.
// DIRECT as in the forward pass, for the queries and dO.
template <class E, int DK, int DV, int NW, int DIRECT>
__global__ void __launch_bounds__(64 * NW, (occupancy<E, DV>(E::bytes == 4)))
diff_dkv_kernel(DiffProblem p)
{
    using T = typename E::T;
    constexpr int QT = 32, NT = 64 * NW;
    using LQ = Tile<E, DK>;
    using LG = Tile<E, DV>;
    // The values' fragments stay in registers unless that halves the occupancy.
    constexpr bool kLdsV = E::bytes == 2 && DV == 128;
    // A buffer in LDS: the queries of both maps, dO, and per row L_1, L_2, D_1, D_2, lam
    // and the keys that it sees.
    constexpr uint32_t kMap = LQ::kBytes, kGo = 2 * kMap, kStat = kGo + LG::kBytes;
    constexpr uint32_t kLam = kStat + 16 * QT, kLim = kLam + 4 * QT;
    constexpr uint32_t kBuffer = (kLim + 4 * QT + 255) / 256 * 256;
    constexpr int kBuffers = buffers<E, NT, DIRECT>();
    __shared__ alignas(256) char lds[kBuffers * kBuffer + (kLdsV ? NW * LG::kBytes : 0)];
    const uint32_t buf = lds_offset(lds), vs = buf + kBuffers * kBuffer;
    if (int(blockIdx.x) < p.H) {
        sum_dlam<NT>(p, blockIdx.x, p.glam);
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 5, c = lane & 31;
    const Place here = place(p, blockIdx.x - p.H, gridDim.x - p.H, p.ktiles, p.rsplits, false);
    const int64_t unit = here.unit;
    const int w = int(here.unit / unsigned(p.G)), kvh = int(here.unit) - w * p.G;
    const int tile = here.tile, split = here.split;
    const int nrows = p.R * p.nq;
    const int kb = tile * 32 * NW, kw = kb + wave * 32, key = kw + c;
    const int len = window_len(p, w);
    const bool live = key < len;

    Frag<E> k[2][DK / 16], v[kLdsV ? 1 : DV / 16];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        const T *src = at<E>(p.k, w, 2 * kvh + a, live ? key : 0);
#pragma unroll
        for (int i = 0; i < DK / 16; ++i)
            k[a][i] = as_frag(load_chunk<E, DIRECT == 16>(src + 16 * i + 8 * g,
                                                       p.d - 16 * i - 8 * g, live, p.d));
    }
    if constexpr (kLdsV) {
        const T *v0 = at<E>(p.v, w, kvh, 0);
        constexpr int kChunks = NW * 32 * LG::kRow / NT;
#pragma unroll 4
        for (int i = 0; i < kChunks; ++i) {
            const int id = threadIdx.x + i * NT, row = id / LG::kRow, ch = id % LG::kRow;
            const bool in = kb + row < len;
            LG::store(vs + row / 32 * LG::kBytes, row % 32, ch,
                      load_chunk<E, DIRECT == 16>(v0 + (in ? kb + row : 0) * p.v.token + 8 * ch,
                                            p.dv - 8 * ch, in, p.dv));
        }
    } else {
        const T *src = at<E>(p.v, w, kvh, live ? key : 0);
#pragma unroll
        for (int i = 0; i < DV / 16; ++i)
            v[i] = as_frag(load_chunk<E, DIRECT == 16>(src + 16 * i + 8 * g, p.dv - 16 * i - 8 * g,
                                                    live, p.dv));
    }
    f16v gk[2][DK / 32] = {}, gv[DV / 32] = {};

    Stage<E, DK, 2 * QT, NT> sq;
    Stage<E, DV, QT, NT> sgo;
    f4 sstat;
    float slam;
    // Tiles of rows from `from` on, past those that see no key of this workgroup.
    const int rend = min(nrows, (split + 1) * p.rchunk);
    auto next = [&](int from) {
        while (from < rend && tile_limit(p, len, from, min(from + QT, nrows) - 1) <= kb)
            from += QT;
        return from;
    };
    using Off = std::conditional_t<DIRECT != 0, int, int64_t>;
    // A row's place from the unit's first: the heads that share the keys lie behind each
    // other, head after head.  The last row stands for those behind it, whose probabilities
    // are zero, and the first one that sees a key for those of its head in front of it.
    const T *q0 = at<E>(p.q, w, 2 * kvh * p.R, 0), *go0 = at<E>(p.go, w, kvh * p.R, 0);
    const int first = p.causal == 2 && len > 0 ? max(0, p.nq - len) : 0;
    auto place_of = [&](int r) {
        const Row row = row_of(p, 0, min(r, nrows - 1));
        return Row{row.head, max(row.token, first)};
    };
    auto q_row = [&](int r, int a) {
        const Row row = place_of(r);
        return (2 * row.head + a) * Off(p.q.head) + row.token * Off(p.q.token);
    };
    auto go_row = [&](int r) {
        const Row row = place_of(r);
        return row.head * Off(p.go.head) + row.token * Off(p.go.token);
    };
    auto fetch = [&](int r0, uint32_t t) {
        if constexpr (DIRECT) {
            direct_tile<DK, 2 * QT, NT, DIRECT>(
                t, q0, [&](int i) { return q_row(r0 + i % QT, i / QT); }, p.d,
                thread_again());
            direct_tile<DV, QT, NT, DIRECT>(
                t + kGo, go0, [&](int i) { return go_row(r0 + i); }, p.dv, thread_again());
        } else {
            sq.load([&](int i) { return q0 + q_row(r0 + i % QT, i / QT); },
                    [](int) { return true; }, p.d);
            sgo.load([&](int i) { return go0 + go_row(r0 + i); },
                     [](int) { return true; }, p.dv);
        }
        const float4 *stats = p.row_stats + unit * p.rows32 + r0;
        const float *lams = p.row_lambda + unit * p.rows32 + r0;
        if constexpr (DIRECT) {
            if (threadIdx.x < QT)
                load_to_lds<16>(stats, 16 * threadIdx.x, t + kStat);
            if (threadIdx.x < QT / 4)
                load_to_lds<16>(lams, 16 * threadIdx.x, t + kLam);
        } else if (threadIdx.x < QT) {
            sstat = *reinterpret_cast<const f4 *>(stats + threadIdx.x);
            slam = lams[threadIdx.x];
        }
    };
    auto commit = [&](int r0, uint32_t t) {
        if constexpr (!DIRECT) {
            sq.store(t);
            sgo.store(t + kGo);
        }
        if (threadIdx.x < QT) {
            if constexpr (!DIRECT) {
                *lds_at<f4>(t + kStat + 16 * threadIdx.x) = sstat;
                *lds_at<float>(t + kLam + 4 * threadIdx.x) = slam;
            }
            if (p.causal) {
                const int r = r0 + threadIdx.x;
                *lds_at<int>(t + kLim + 4 * threadIdx.x) =
                    r < nrows ? key_limit(p, len, row_of(p, kvh, r).token) : 0;
            }
        }
    };
    int r0 = kb < len ? next(split * p.rchunk) : rend;
    if (r0 < rend) {
        fetch(r0, buf);
        commit(r0, buf);
    }
    // This tile's buffer and the next one's.
    uint32_t t = buf, other = buf + (kBuffers - 1) * kBuffer;
    while (r0 < rend) {
        if constexpr (DIRECT)
            arrived();
        __syncthreads();
        const int r1 = next(r0 + QT);
        // Without a causal mask every row sees every key there is, and rows behind the last
        // have probabilities of zero.
        const int rowlim = p.causal ? *lds_at<int>(t + kLim + 4 * c) : len;
        const bool any = __any(kw < rowlim), masked = p.causal && !__all(kw + 32 <= rowlim);
        f16v s[2] = {}, x = {};
        if (any) {
            const unsigned at_lane = thread_again() & 63;
            const uint32_t qrow = first_row<E, DK>(t, at_lane);
            const uint32_t grow = first_row<E, DV>(t + kGo, at_lane);
#pragma unroll
            for (int i = 0; i < DK / 16; ++i)
#pragma unroll
                for (int a = 0; a < 2; ++a)
                    s[a] = mma(row_frag<E, DK>(qrow + a * kMap, i), k[a][i], s[a]);
            part();
#pragma unroll
            for (int i = 0; i < DV / 16; ++i) {
                if constexpr (kLdsV)
                    x = mma(row_frag<E, DV>(grow, i),
                            row_frag<E, DV>(first_row<E, DV>(vs + wave * LG::kBytes, at_lane), i), x);
                else
                    x = mma(row_frag<E, DV>(grow, i), v[i], x);
            }
            part();
        }
        // The next tile's loads, behind the first products: a register that the compiler
        // keeps in memory is waited for with all loads before it.
        if (r1 < rend)
            fetch(r1, other);
        if (any) {
            const unsigned at_lane = thread_again() & 63;
            const uint32_t qcol = first_col<E, DK>(t, at_lane);
            const uint32_t gcol = first_col<E, DV>(t + kGo, at_lane);
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const bool see = key < *lds_at<int>(t + kLim + 4 * reg_row(i, g));
                    s[0][i] = see ? s[0][i] : -INFINITY;
                    s[1][i] = see ? s[1][i] : -INFINITY;
                }
            }
            f16v pd;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f4 lam = *lds_at<f4>(t + kLam + 4 * (8 * j + 4 * g));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 4 * j + e;
                    const f4 st = *lds_at<f4>(t + kStat + 16 * reg_row(i, g));
                    const float p1 = fast_exp2(fmaf(s[0][i], p.scale2, -st.x));
                    const float p2 = lam[e] * fast_exp2(fmaf(s[1][i], p.scale2, -st.y));
                    pd[i] = p1 - p2;
                    s[0][i] = p1 * (x[i] - st.z);
                    s[1][i] = p2 * (st.w - x[i]);
                }
                part();
            }
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    // A factor, as in the dQ kernel: NaN stays.
                    const float keep =
                        *lds_at<int>(t + kLim + 4 * reg_row(i, g)) == 1 ? 0.f : 1.f;
                    s[0][i] *= keep;
                    s[1][i] *= keep;
                }
            }
            part();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Frag<E> f = frag_of(pd, h, E());
#pragma unroll
                for (int i = 0; i < DV / 32; ++i)
                    gv[i] = mma(col_frag<E, DV>(gcol, h, i), f, gv[i]);
#pragma unroll
                for (int a = 0; a < 2; ++a) {
                    const Frag<E> ds = frag_of(s[a], h, E());
#pragma unroll
                    for (int i = 0; i < DK / 32; ++i)
                        gk[a][i] = mma(col_frag<E, DK>(qcol + a * kMap, h, i), ds, gk[a][i]);
                }
            }
        }
        if (r1 < rend) {
            if (kBuffers == 1)
                __syncthreads();
            commit(r1, other);
        }
        exchange(t, other);
        r0 = r1;
    }
    if (key >= p.nk)
        return;
    if (p.rsplits > 1) {
        float *out = p.partial + ((unit * p.rsplits + split) * p.nk + key) * p.partial_row;
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int i = 0; i < DK / 32; ++i)
                store_block<F32>(out + a * p.d4, i, g, p.d4, true, gk[a][i]);
#pragma unroll
        for (int i = 0; i < DV / 32; ++i)
            store_block<F32>(out + 2 * p.d4, i, g, p.dv4, true, gv[i]);
        return;
    }
    // Keys behind the length, whose operands were zeros, have gradients of zero, but for NaN
    // that a query brought in.
    if (!live) {
#pragma unroll
        for (int i = 0; i < DV / 32; ++i)
            gv[i] = f16v{};
#pragma unroll
        for (int i = 0; i < DK / 32; ++i)
            gk[0][i] = gk[1][i] = f16v{};
    }
    const float scale = key_scale(p, len);
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int i = 0; i < DK / 32; ++i)
            store_block<E>(at_out<E>(p.gk, w, 2 * kvh + a, key), i, g, p.d, p.vec_gk, gk[a][i],
                           scale);
#pragma unroll
    for (int i = 0; i < DV / 32; ++i)
        store_block<E>(at_out<E>(p.gv, w, kvh, key), i, g, p.dv, p.vec_gv, gv[i]);
}

// Adds up the row ranges of one key.
template <class E>
__global__ void __launch_bounds__(kMerge)
diff_dkv_merge_kernel(DiffProblem p)
{
    const int64_t unit = blockIdx.x / unsigned(p.nk);
    const int key = int(blockIdx.x - unit * p.nk);
    const int w = int(unsigned(unit) / unsigned(p.G)), kvh = int(unit) - w * p.G;
    const int len = window_len(p, w);
    const bool live = key < len;
    const float scale = key_scale(p, len);
    const float *part = p.partial + (unit * p.rsplits * p.nk + key) * p.partial_row;
    const int64_t step = int64_t(p.nk) * p.partial_row;
    for (int col = threadIdx.x; col < 2 * p.d4 + p.dv4; col += kMerge) {
        float s = 0.f;
        if (live)
            for (int i = 0; i < p.rsplits; ++i)
                s += part[i * step + col];
        if (col < 2 * p.d4) {
            const int a = col >= p.d4, at_col = col - a * p.d4;
            if (at_col < p.d)
                E::store(at_out<E>(p.gk, w, 2 * kvh + a, key), at_col, scale * s);
        } else if (col - 2 * p.d4 < p.dv) {
            E::store(at_out<E>(p.gv, w, kvh, key), col - 2 * p.d4, s);
        }
    }
}

// No windows: the sum over nothing.
__global__ void diff_dlam_zero_kernel(int n, float *glam)
{
    for (int i = threadIdx.x; i < n; i += blockDim.x)
        glam[i] = 0.f;
}

// ---- dispatch -----------------------------------------------------------------

template <class E, int DK, int DV, int NW>
void run(const DiffProblem &p, int64_t blocks, hipStream_t s)
{
    const dim3 grid(unsigned(blocks + p.H));
    if constexpr (E::bytes == 2) {
        if (direct(p, p.k, p.d, 0) && direct(p, p.v, p.dv, 0) &&
            direct(p, p.q, p.d, 2 * p.R * p.q.head + p.nq * p.q.token) &&
            direct(p, p.go, p.dv, p.R * p.go.head + p.nq * p.go.token)) {
            diff_dkv_kernel<E, DK, DV, NW, 16><<<grid, 64 * NW, 0, s>>>(p);
            return;
        }
        if (direct(p, p.q, p.d, 2 * p.R * p.q.head + p.nq * p.q.token, 4) &&
            direct(p, p.go, p.dv, p.R * p.go.head + p.nq * p.go.token, 4)) {
            diff_dkv_kernel<E, DK, DV, NW, 4><<<grid, 64 * NW, 0, s>>>(p);
            return;
        }
    }
    diff_dkv_kernel<E, DK, DV, NW, 0><<<grid, 64 * NW, 0, s>>>(p);
}

template <class E>
void run_any(const DiffProblem &p, int waves, int64_t blocks, hipStream_t s)
{
    if (waves == 2)
        narrow(p) ? run<E, 32, 64, 2>(p, blocks, s) : run<E, 64, 128, 2>(p, blocks, s);
    else
        narrow(p) ? run<E, 32, 64, 4>(p, blocks, s) : run<E, 64, 128, 4>(p, blocks, s);
}

// Waves to a workgroup: two for up to 64 rows or keys, otherwise four.
int backward_waves(int64_t n) { return n <= 64 ? 2 : 4; }

int64_t round256(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// Row ranges of the dK, dV kernel: enough workgroups for the 256 CUs twice over, of at
// least four tiles each.
void plan_rows(DiffProblem *p, int waves)
{
    const int64_t rows = int64_t(p->R) * p->nq, units = int64_t(p->W) * p->G;
    p->rows32 = int64_t(ceil_div(rows, 32)) * 32;
    p->ktiles = ceil_div(p->nk, 32 * waves);
    const int64_t blocks = units * p->ktiles;
    const int most = ceil_div(rows, 128);
    const int64_t want = blocks > 0 ? (512 + blocks - 1) / blocks : 1;
    p->rsplits = int(want < most ? want : most);
    p->rchunk = ceil_div(ceil_div(rows, p->rsplits), 32) * 32;
    p->rsplits = ceil_div(rows, p->rchunk);
    p->d4 = round4(p->d);
    p->dv4 = round4(p->dv);
    p->partial_row = 2 * p->d4 + p->dv4;
}

// Key ranges of the dQ kernel, for few rows over many keys: enough workgroups for the 256
// CUs twice over, of at least four tiles each.  Only where the workgroups are half of the
// CUs at most: 8 queries over 8192 keys, forward and backward, take 70 instead of 321 us
// (fp32, twice as many, 140 instead of 1653 us), 8 heads of 2048 causal rows (128 workgroups) 185 instead of
// 206 us, but 14 heads of 2048 rows (224) 315 instead of 297 us; with one tile of rows to a
// unit, whose sums are small, all of them (180 of 2 queries over 1457 keys, fp32: 78 instead
// of 176 us for dQ, but 508 of 5 over 514 keys 188 instead of 168 us).  Up to 256 keys, where the
// kernel walks over them twice, there are none.
void plan_keys(DiffProblem *p, int waves)
{
    const int64_t rows = int64_t(p->R) * p->nq, units = int64_t(p->W) * p->G;
    p->tiles = ceil_div(rows, 32 * waves);
    p->dq_row = 2 * p->d4 + 4;
    p->splits = 1;
    p->chunk = p->nk;
    const int64_t blocks = units * p->tiles;
    if (p->nk <= NYSTRA_DIFF_SHORT_KEYS || blocks == 0 || blocks > (rows <= 32 ? 256 : 128))
        return;
    const int64_t most = ceil_div(p->nk, 128), want = (512 + blocks - 1) / blocks;
    p->splits = int(want < most ? want : most);
    p->chunk = ceil_div(ceil_div(p->nk, p->splits), 32) * 32;
    p->splits = ceil_div(p->nk, p->chunk);
}

// The workspace's parts: a record of each row and its lambda, dlam's rows, and, one after the
// other in the same place, dQ by key range and dK and dV by row range.
struct Parts {
    int64_t stats, lambda, lam, partial;
};

Parts parts_of(const DiffProblem &p)
{
    const int64_t units = int64_t(p.W) * p.G;
    return Parts{round256(units * p.rows32 * 16), round256(units * p.rows32 * 4),
                 round256(int64_t(p.W) * p.H * p.nq * 4),
                 std::max(p.rsplits > 1 ? units * p.rsplits * p.nk * p.partial_row * 4 : 0,
                          p.splits > 1 ? units * p.splits * p.R * p.nq * p.dq_row * 4 : 0)};
}

}  // namespace

size_t diff_backward_workspace(const DiffProblem &p)
{
    DiffProblem t = p;
    plan_rows(&t, backward_waves(p.nk));
    plan_keys(&t, backward_waves(int64_t(p.R) * p.nq));
    const Parts b = parts_of(t);
    return size_t(b.stats + b.lambda + b.lam + b.partial);
}

hipError_t launch_diff_backward(DiffProblem p, void *workspace, hipStream_t s)
{
    const int e = p.dtype == 0 ? 4 : 2;
    if (p.W == 0) {
        diff_dlam_zero_kernel<<<1, 256, 0, s>>>(p.H, p.glam);
        return hipGetLastError();
    }
    set_common(&p);
    p.vec_gq = store_vec(p.gq, p.d, e);
    p.vec_gk = store_vec(p.gk, p.d, e);
    p.vec_gv = store_vec(p.gv, p.dv, e);
    const int64_t rows = int64_t(p.R) * p.nq, units = int64_t(p.W) * p.G;
    const int wq = backward_waves(rows), wk = backward_waves(p.nk);
    plan_rows(&p, wk);
    plan_keys(&p, wq);
    const Parts b = parts_of(p);
    char *ws = static_cast<char *>(workspace);
    p.row_stats = reinterpret_cast<float4 *>(ws);
    p.row_lambda = reinterpret_cast<float *>(ws + b.stats);
    p.rows_lam = reinterpret_cast<float *>(ws + b.stats + b.lambda);
    p.partial = reinterpret_cast<float *>(ws + b.stats + b.lambda + b.lam);
    hipError_t err = launch_diff_dq(p, wq, units * p.tiles * p.splits, s);
    if (err != hipSuccess)
        return err;
    const int64_t blocks = units * p.ktiles * p.rsplits;
    p.dtype == 0 ? run_any<F32>(p, wk, blocks, s) : run_any<BF16>(p, wk, blocks, s);
    err = hipGetLastError();
    if (err != hipSuccess)
        return err;
    if (p.rsplits > 1) {
        const dim3 grid(unsigned(units * p.nk));
        if (p.dtype == 0)
            diff_dkv_merge_kernel<F32><<<grid, kMerge, 0, s>>>(p);
        else
            diff_dkv_merge_kernel<BF16><<<grid, kMerge, 0, s>>>(p);
    }
    return hipGetLastError();
}

}  // namespace nystra
