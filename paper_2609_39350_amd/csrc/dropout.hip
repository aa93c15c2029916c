// Dropout: out = residual + x / chance where the element is kept, residual where it is not; the gradient is the same of
// d_out, without a residual.
//
// Which are kept is a function of (seed, offset, the element's index), so no mask is stored: Philox4x32-10 (Salmon,
// Moraes, Dror, Shaw: Parallel random numbers, as easy as 1, 2, 3; 2011) of the counter (index / 8, offset) under the
// key seed gives 128 bits, 16 for each of 8 neighbours: element i of the 8 has half i % 2 (0: the low) of word i / 2, and
// is kept where that is at least the cut.  16 bits, because the ten rounds cost as much as moving 16 bytes does: with 32
// for each element the rounds would bound it, not HBM: they are most of the instructions that keep the vector units 50 %
// busy.  bf16, 32,768 x 7,168: onto a residual and backward 388 us for both (2.3 GB, 6.1 TB/s).
#include "operators.h"

namespace hapmoe {
namespace {

constexpr int kThreads = 256;

__device__ inline void philox(uint32_t w[4], uint64_t key)
{
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t a = (uint64_t)w[0] * 0xD2511F53u, b = (uint64_t)w[2] * 0xCD9E8D57u;
        w[0] = (uint32_t)(b >> 32) ^ w[1] ^ k0;
        w[1] = (uint32_t)b;
        w[2] = (uint32_t)(a >> 32) ^ w[3] ^ k1;
        w[3] = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

// The 8 elements from 8 * g on.  FLAT: the matrices are one row, of whole aligned vectors; else each 8 have their row and
// column, and are whole vectors of any alignment where the row does not end among them (3,001 x 1,023 of fp32, both
// passes: 31 us element by element, 17 by vectors).
template <typename T, bool FLAT>
__global__ __launch_bounds__(kThreads) void k_dropout(const T *__restrict__ x, int64_t x_stride, int64_t n,
                                                      int64_t columns, const T *__restrict__ residual,
                                                      int64_t residual_stride, uint32_t cut, float factor, uint64_t seed,
                                                      uint64_t offset, const int64_t *__restrict__ counter,
                                                      T *__restrict__ out)
{
    const int64_t first = workgroup() * kThreads, g = first + threadIdx.x;
    if (g * 8 >= n) return;
    if (counter) offset += (uint64_t)*counter;
    uint32_t w[4] = {(uint32_t)g, (uint32_t)(g >> 32), (uint32_t)offset, (uint32_t)(offset >> 32)};
    philox(w, seed);
    auto kept = [&](int i) { return (i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffff) >= cut; };
    if constexpr (FLAT) {
        const Vec8<T> v = *reinterpret_cast<const Vec8<T> *>(x + g * 8);
        Vec8<T> r = {}, o;
        if (residual) r = *reinterpret_cast<const Vec8<T> *>(residual + g * 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) o.v[i] = from_f32<T>((kept(i) ? to_f32(v.v[i]) * factor : 0.0f) + to_f32(r.v[i]));
        *reinterpret_cast<Vec8<T> *>(out + g * 8) = o;
    } else {
        // the workgroup's first element's row by one division, the thread's from there in 32 bits
        const int64_t at = first * 8;
        const int64_t row0 = at >> 32 ? at / columns : (int64_t)((uint32_t)at / (uint32_t)columns);
        const uint32_t from = (uint32_t)(at - row0 * columns) + threadIdx.x * 8, rows = from / (uint32_t)columns;
        int64_t row = row0 + rows;
        int column = (int)(from - rows * (uint32_t)columns);
        if (column + 8 <= columns) {
            const Words<T> v = load_words(x + row * x_stride + column);
            Words<T> r = {};
            if (residual) r = load_words(residual + row * residual_stride + column);
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = (kept(i) ? element<T>(v, i) * factor : 0.0f) + element<T>(r, i);
            store_words(out + g * 8, words_of<T>(o));
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (g * 8 + i >= n) break;
            float v = kept(i) ? to_f32(x[row * x_stride + column]) * factor : 0.0f;
            if (residual) v += to_f32(residual[row * residual_stride + column]);
            out[g * 8 + i] = from_f32<T>(v);
            if (++column == columns) column = 0, ++row;
        }
    }
}

}  // namespace

hipError_t launch_dropout(const void *x, int type, int64_t x_stride, int64_t rows, int64_t columns,
                          const void *residual, int64_t residual_stride, double p, uint64_t seed, uint64_t offset,
                          const int64_t *counter, void *out, hipStream_t s)
{
    const uint32_t cut = (uint32_t)(p * 65536.0 + 0.5);   // elements are dropped with a chance of cut / 65536
    const float factor = cut < 65536 ? (float)(65536.0 / (65536 - cut)) : 0.0f;
    const int64_t n = rows * columns;
    auto launch = [&](auto t) {
        using T = decltype(t);
        const int64_t bytes = sizeof(T) * 8;
        const bool flat = n % 8 == 0 && (rows <= 1 || (x_stride == columns && (!residual || residual_stride == columns))) &&
                          aligned(x, bytes) && aligned(out, bytes) && aligned(residual, bytes);
        hipLaunchKernelGGL((flat ? k_dropout<T, true> : k_dropout<T, false>), many(ceil_div(n, 8 * kThreads)),
                           dim3(kThreads), 0, s, static_cast<const T *>(x), x_stride, n, columns,
                           static_cast<const T *>(residual), residual_stride, cut, factor, seed, offset, counter,
                           static_cast<T *>(out));
        return hipGetLastError();
    };
    if (type == HAPMOE_F32) return launch(float());
    if (type == HAPMOE_BF16) return launch(bf16());
    return launch(f16());
}

}  // namespace hapmoe
