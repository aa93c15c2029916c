// The sum of a token's expert outputs under its weights, and its gradient.
// Bound by HBM: every row of y is read once (backward: and written once), 16
// bytes a lane; a workgroup a token and 2,048 columns, so that the sum has a fixed
// order and no atomics.  bf16, 8 choices, hidden 4,096: 4,096 tokens 60 us (5.1 TB/s),
// backward 110 us (5.5 TB/s).  16 tokens of 7,168: 4.2 us, a launch and two dependent
// loads.
#include <type_traits>

#include "operators.h"

namespace hapmoe {
namespace {

constexpr int kThreads = 256;

// out[t], 8 * kThreads elements of it a workgroup.  The rows are added in the order of j.
template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void k_combine(const T *__restrict__ y, int64_t rows, int64_t tokens, int top_k,
                                                      int64_t hidden,
                                                      const int32_t *__restrict__ place,
                                                      const float *__restrict__ weight, T *__restrict__ out)
{
    const int64_t t = workgroup();   // rows are read past the caches: 98 us in place of 110 at 470 MB, the same at 59
    const int64_t h = ((int64_t)blockIdx.y * kThreads + threadIdx.x) * (VEC ? 8 : 1);
    if (h >= hidden || t >= tokens) return;
    float sum[VEC ? 8 : 1] = {};
#pragma unroll 8
    for (int j = 0; j < top_k; ++j) {
        const int p = place[t * top_k + j];
        if ((uint32_t)p >= (uint64_t)rows) continue;
        const float w = weight ? weight[t * top_k + j] : 1.0f;
        if constexpr (VEC) {
            const Vec8<T> r = load_once(y + p * hidden + h);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += w * to_f32(r.v[i]);
        } else {
            sum[0] += w * to_f32(y[p * hidden + h]);
        }
    }
    if constexpr (VEC) {
        Vec8<T> r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[i] = from_f32<T>(sum[i]);
        *reinterpret_cast<Vec8<T> *>(out + t * hidden + h) = r;
    } else {
        out[t * hidden + h] = from_f32<T>(sum[0]);
    }
}

// A wave a (token, choice): it reads d_out[t] (which the token's other choices read too, from the cache) and its row
// of y once, and writes the row of d_y where slot names this choice there, as place and slot of the router do.  Where they
// do not agree each still has its own: d_weight[r] goes by place, and row r of d_y, by slot, has the wave of row r as its
// writer, which also clears it where no choice has it.  Knowing whether they agree costs one more
// dependent load: 106 us against 103 at 268 MB of y, nothing at 59 and 459.  ONCE: 1, y goes past the caches, 2, d_y too.  us
// at 59, 268, 470 MB of y (bf16): 22.1, 118.6, 203 (0), 24.4, 102.2, 205 (1), 25.5, 111, 190 (2).
template <typename T, bool VEC, int ONCE>
__global__ __launch_bounds__(kThreads) void k_combine_backward(
    const T *__restrict__ d_out, const T *__restrict__ y, int64_t rows, int top_k, int64_t hidden,
    const int32_t *__restrict__ slot, const int32_t *__restrict__ place, const float *__restrict__ weight,
    T *__restrict__ d_y, float *__restrict__ d_weight)
{
    constexpr int kStep = VEC ? 8 : 1;
    const int lane = threadIdx.x & 63;
    const int64_t r = workgroup() * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (r >= rows) return;
    const int p = place[r], s = slot[r];
    const float w = weight[r];
    const bool has = (uint32_t)p < (uint64_t)rows, taken = (uint32_t)s < (uint64_t)rows;
    const int back = slot[has ? p : 0], forth = place[taken ? s : 0];   // both on their way at once
    const bool writes = has && back == r, left = !taken || forth != r;
    float dot = 0.0f;
    auto pass = [&](auto write) {
        const T *g = d_out + (int)r / top_k * hidden, *row = y + p * hidden;
        T *to = d_y + p * hidden;
#pragma unroll 2
        for (int64_t h = lane * kStep; h < hidden; h += 64 * kStep) {
            if constexpr (VEC) {
                const Vec8<T> a = *reinterpret_cast<const Vec8<T> *>(g + h);
                const Vec8<T> b = ONCE ? load_once(row + h) : *reinterpret_cast<const Vec8<T> *>(row + h);
                Vec8<T> c;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    dot += to_f32(a.v[i]) * to_f32(b.v[i]);
                    c.v[i] = from_f32<T>(w * to_f32(a.v[i]));
                }
                if constexpr (!decltype(write)::value)
                    continue;
                else if constexpr (ONCE == 2)
                    store_once(to + h, c);
                else
                    *reinterpret_cast<Vec8<T> *>(to + h) = c;
            } else {
                dot += to_f32(g[h]) * to_f32(row[h]);
                if constexpr (decltype(write)::value) to[h] = from_f32<T>(w * to_f32(g[h]));
            }
        }
    };
    if (writes)
        pass(std::true_type());
    else if (has)
        pass(std::false_type());
    dot = wave_reduce(dot, Sum());
    if (lane == 0) d_weight[r] = dot;
    if (left) {
        const T *g = taken ? d_out + s / top_k * hidden : nullptr;
        const float other = taken ? weight[s] : 0.0f;
        for (int64_t h = lane; h < hidden; h += 64) d_y[r * hidden + h] = from_f32<T>(taken ? other * to_f32(g[h]) : 0.0f);
    }
}

template <typename T>
bool vectors(int64_t hidden, const void *a, const void *b, const void *c)
{
    const int64_t n = sizeof(T) * 8;
    return hidden % 8 == 0 && aligned(a, n) && aligned(b, n) && aligned(c, n);
}

template <typename T>
hipError_t combine(const void *y, int64_t rows, int64_t tokens, int top_k, int64_t hidden, const int32_t *place,
                   const float *weight, void *out, hipStream_t s)
{
    const bool vec = vectors<T>(hidden, y, out, out);
    hipLaunchKernelGGL((vec ? k_combine<T, true> : k_combine<T, false>),
                       many(tokens, (unsigned)ceil_div(hidden, kThreads * (vec ? 8 : 1))), dim3(kThreads), 0, s,
                       static_cast<const T *>(y), rows, tokens, top_k, hidden, place, weight, static_cast<T *>(out));
    return hipGetLastError();
}

template <typename T>
hipError_t combine_backward(const void *d_out, const void *y, int64_t tokens, int top_k, int64_t hidden,
                            const int32_t *slot, const int32_t *place, const float *weight, void *d_y,
                            float *d_weight, hipStream_t s)
{
    const bool vec = vectors<T>(hidden, d_out, y, d_y);
    const int64_t rows = tokens * top_k;
    const int64_t bytes = rows * hidden * (int64_t)sizeof(T);
    auto *kernel = !vec                   ? k_combine_backward<T, false, 0>
                   : bytes < (128 << 20) ? k_combine_backward<T, true, 0>
                   : bytes < (384 << 20) ? k_combine_backward<T, true, 1>
                                         : k_combine_backward<T, true, 2>;
    hipLaunchKernelGGL(kernel, many(ceil_div(rows, kThreads / 64)), dim3(kThreads), 0, s,
                       static_cast<const T *>(d_out), static_cast<const T *>(y), rows, top_k, hidden, slot, place,
                       weight, static_cast<T *>(d_y), d_weight);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_combine(const void *y, int type, int64_t rows, int64_t tokens, int top_k, int64_t hidden,
                          const int32_t *place, const float *weight, void *out, hipStream_t s)
{
    auto *f = type == HAPMOE_F32 ? combine<float> : type == HAPMOE_BF16 ? combine<bf16> : combine<f16>;
    return f(y, rows, tokens, top_k, hidden, place, weight, out, s);
}

hipError_t launch_combine_backward(const void *d_out, const void *y, int type, int64_t tokens, int top_k,
                                   int64_t hidden, const int32_t *slot, const int32_t *place, const float *weight,
                                   void *d_y, float *d_weight, hipStream_t s)
{
    auto *f = type == HAPMOE_F32    ? combine_backward<float>
              : type == HAPMOE_BF16 ? combine_backward<bf16>
                                    : combine_backward<f16>;
    return f(d_out, y, tokens, top_k, hidden, slot, place, weight, d_y, d_weight, s);
}

}  // namespace hapmoe
