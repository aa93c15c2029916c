// Layer norm of rows and its gradients.
//   y = (x - mean) rstd w + b,  rstd = 1 / sqrt(mean((x - mean)^2) + eps);  not centred: mean is 0
//   d_x = rstd (g - mean(g) - xhat mean(g xhat)) + add,  g = d_y w,  xhat = (x - mean) rstd;  not centred: no mean(g)
//   d_w = sum over rows of d_y xhat,  d_b = sum over rows of d_y
// The squares are of the differences from the mean (a second look at the row), so that a row far from 0 loses nothing.
#include "operators.h"

namespace hapmoe {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// Of the workgroup, in every thread.  sh: one place a wave.
__device__ inline float workgroup_sum(float v, float *sh)
{
    v = wave_reduce(v, Sum());
    __syncthreads();   // what was there is read
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += sh[w];
    return sum;
}

template <typename T, typename W, bool CENTER>
__global__ __launch_bounds__(kThreads) void k_norm(const T *__restrict__ x, int64_t stride, int64_t rows, int64_t hidden,
                                                   const W *__restrict__ weight, const W *__restrict__ bias, float eps,
                                                   float *__restrict__ mean, float *__restrict__ rstd, T *__restrict__ y)
{
    __shared__ float sh[kWaves];
    const int64_t r = workgroup();
    if (r >= rows) return;
    const T *const row = x + r * stride;
    float m = 0.0f, s = 0.0f;
    if (CENTER) {
        for (int64_t h = threadIdx.x; h < hidden; h += kThreads) s += to_f32(row[h]);
        m = workgroup_sum(s, sh) / (float)hidden;
        s = 0.0f;
    }
    for (int64_t h = threadIdx.x; h < hidden; h += kThreads) {
        const float d = to_f32(row[h]) - m;
        s += d * d;
    }
    const float rs = 1.0f / sqrtf(workgroup_sum(s, sh) / (float)hidden + eps);
    for (int64_t h = threadIdx.x; h < hidden; h += kThreads)
        y[r * hidden + h] = from_f32<T>((to_f32(row[h]) - m) * rs * to_f32(weight[h]) + (bias ? to_f32(bias[h]) : 0.0f));
    if (threadIdx.x == 0) {
        if (CENTER) mean[r] = m;
        rstd[r] = rs;
    }
}

template <typename T, typename W, bool CENTER>
__global__ __launch_bounds__(kThreads) void k_norm_backward(
    const T *__restrict__ d_y, int64_t d_y_stride, const T *__restrict__ x, int64_t x_stride, int64_t rows,
    int64_t hidden, const W *__restrict__ weight, const float *__restrict__ mean, const float *__restrict__ rstd,
    const T *__restrict__ add, int64_t add_stride, T *__restrict__ d_x)
{
    __shared__ float sh[kWaves];
    const int64_t r = workgroup();
    if (r >= rows) return;
    const T *const row = x + r * x_stride, *const g_row = d_y + r * d_y_stride;
    const float m = CENTER ? mean[r] : 0.0f, rs = rstd[r];
    float a = 0.0f, b = 0.0f;
    for (int64_t h = threadIdx.x; h < hidden; h += kThreads) {
        const float g = to_f32(g_row[h]) * to_f32(weight[h]);
        a += g;
        b += g * ((to_f32(row[h]) - m) * rs);
    }
    a = CENTER ? workgroup_sum(a, sh) / (float)hidden : 0.0f;
    b = workgroup_sum(b, sh) / (float)hidden;
    for (int64_t h = threadIdx.x; h < hidden; h += kThreads) {
        const float g = to_f32(g_row[h]) * to_f32(weight[h]), hat = (to_f32(row[h]) - m) * rs;
        const float d = rs * (g - a - hat * b);
        d_x[r * hidden + h] = from_f32<T>(add ? to_f32(add[r * add_stride + h]) + d : d);
    }
}

// Sums of the rows of a part: part[blockIdx.y][2][hidden].
template <typename T, bool CENTER>
__global__ __launch_bounds__(kThreads) void k_norm_weight(const T *__restrict__ d_y, int64_t d_y_stride,
                                                          const T *__restrict__ x, int64_t x_stride, int64_t rows,
                                                          int64_t hidden, const float *__restrict__ mean,
                                                          const float *__restrict__ rstd, int64_t each,
                                                          float *__restrict__ part)
{
    const int64_t h = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (h >= hidden) return;
    const int64_t lo = blockIdx.y * each, hi = lo + each < rows ? lo + each : rows;
    float w = 0.0f, b = 0.0f;
    for (int64_t r = lo; r < hi; ++r) {
        const float g = to_f32(d_y[r * d_y_stride + h]);
        w += g * ((to_f32(x[r * x_stride + h]) - (CENTER ? mean[r] : 0.0f)) * rstd[r]);
        b += g;
    }
    part[(blockIdx.y * 2) * hidden + h] = w;
    part[(blockIdx.y * 2 + 1) * hidden + h] = b;
}

__global__ __launch_bounds__(kThreads) void k_norm_join(const float *__restrict__ part, int parts, int64_t hidden,
                                                        float *__restrict__ d_weight, float *__restrict__ d_bias)
{
    const int64_t h = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (h >= hidden) return;
    float w = 0.0f, b = 0.0f;
    for (int p = 0; p < parts; ++p) {
        w += part[(2 * (int64_t)p) * hidden + h];
        b += part[(2 * (int64_t)p + 1) * hidden + h];
    }
    d_weight[h] = w;
    if (d_bias) d_bias[h] = b;
}

int parts_of(int64_t rows) { return rows < 256 ? (int)rows : 256; }

template <typename F>
hipError_t by_types(int type, int weight_type, F f)
{
    if (type == HAPMOE_F32) return f(float(), float());
    if (type == HAPMOE_BF16) return weight_type == HAPMOE_F32 ? f(bf16(), float()) : f(bf16(), bf16());
    return weight_type == HAPMOE_F32 ? f(f16(), float()) : f(f16(), f16());
}

}  // namespace

int64_t layer_norm_ws_bytes(int64_t rows, int64_t hidden) { return parts_of(rows) * 2 * hidden * 4; }

hipError_t launch_layer_norm(const LayerNorm &a, hipStream_t s)
{
    return by_types(a.type, a.weight_type, [&](auto t, auto w) {
        using T = decltype(t);
        using W = decltype(w);
        hipLaunchKernelGGL((a.mean ? k_norm<T, W, true> : k_norm<T, W, false>), many(a.rows), dim3(kThreads), 0, s,
                           static_cast<const T *>(a.x), a.x_stride, a.rows, a.hidden, static_cast<const W *>(a.weight),
                           static_cast<const W *>(a.bias), a.eps, a.mean, a.rstd, static_cast<T *>(a.out));
        return hipGetLastError();
    });
}

hipError_t launch_layer_norm_backward(const LayerNorm &a, hipStream_t s)
{
    return by_types(a.type, a.weight_type, [&](auto t, auto w) {
        using T = decltype(t);
        using W = decltype(w);
        const T *d_y = static_cast<const T *>(a.d_y), *x = static_cast<const T *>(a.x);
        float *part = static_cast<float *>(a.ws);
        if (a.rows > 0)
            hipLaunchKernelGGL((a.mean ? k_norm_backward<T, W, true> : k_norm_backward<T, W, false>), many(a.rows),
                               dim3(kThreads), 0, s, d_y, a.d_y_stride, x, a.x_stride, a.rows, a.hidden,
                               static_cast<const W *>(a.weight), a.mean, a.rstd, static_cast<const T *>(a.add),
                               a.add_stride, static_cast<T *>(a.out));
        const int parts = parts_of(a.rows);
        const unsigned columns = (unsigned)ceil_div(a.hidden, kThreads);
        if (parts > 0)
            hipLaunchKernelGGL((a.mean ? k_norm_weight<T, true> : k_norm_weight<T, false>), dim3(columns, parts),
                               dim3(kThreads), 0, s, d_y, a.d_y_stride, x, a.x_stride, a.rows, a.hidden, a.mean, a.rstd,
                               ceil_div(a.rows, parts), part);
        hipLaunchKernelGGL(k_norm_join, dim3(columns), dim3(kThreads), 0, s, part, parts, a.hidden, a.d_weight,
                           a.d_bias);
        return hipGetLastError();
    });
}

}  // namespace hapmoe
