// Layer norm of rows and its gradients.
//   y = (x - mean) rstd w + b,  rstd = 1 / sqrt(mean((x - mean)^2) + eps);  not centred: mean is 0
//   d_x = rstd (g - mean(g) - xhat mean(g xhat)) + add,  g = d_y w,  xhat = (x - mean) rstd;  not centred: no mean(g)
//   d_w = sum over rows of d_y xhat,  d_b = sum over rows of d_y
// The squares are of the differences from the mean (a second look at the row, in registers), so that a row far from 0
// loses no more than the mean's own rounding.
//
// Bound by HBM: each row is read once and held, 16-bit elements two a register, the next one's loads on their way under
// the sums.  A wave has a row of up to 1,024 elements, a workgroup a longer one, two vectors of 8 a thread (four a thread:
// 8,192 x 16,384 slower by 6 % forward and half backward).  us, bf16, backward with add and the parts' sums (4 to 7):
// 32,768 x 4,096: forward 90 to 100 (5.4 to 5.9 TB/s), backward 206 to 220 (4.9 to 5.2); 16,384 x 7,168 91 and 172 (5.4);
// 8,192 x 16,384 99 and 236 (4.6 TB/s: no room to hold two rows).  fp32, where 128 registers do not hold a row's two
// matrices and both sums, and 32 to 68 bytes a thread go to scratch (16-bit rows that end in part of a vector 8): 4,096 x
// 16,384 98 and 243 (4.4 TB/s), 4,096 x 12,288 75 and 244 (3.3).  Longer rows are read two and three times, an element a
// thread at once: bf16, 4,096 x 20,480 209 and 417.  Vectors of any alignment; a row that is no multiple of 8 ends in one
// that overlaps the one before.
#include "operators.h"

namespace hapmoe {
namespace {

constexpr int kThreads = 256;

// Over the THREADS threads that share a row, in each of them.  sh: one place a wave, in turn one of two, so that a wave
// that is ahead by one sum writes where none reads.
template <int THREADS, int N>
__device__ inline void row_sum(float *v, float (*sh)[N], int turn)
{
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = wave_reduce(v[n], Sum());
    if constexpr (THREADS > 64) {
        constexpr int kWaves = THREADS / 64;
        sh += turn * kWaves;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) sh[threadIdx.x >> 6][n] = v[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
#pragma unroll
            for (int n = 0; n < N; ++n) v[n] += sh[w][n];
    }
}

// A row by THREADS threads, NV vectors of 8 each: vector k = i * THREADS + t is thread t's i-th.  It starts at 8 k, or
// where less than 8 elements are left at the row's last 8: every load is whole, without a branch that would have to wait
// for what it loads.  The elements before skip(i) are other vectors' then; 8 or more: there are none.  FULL: the row has
// just these vectors.
template <int THREADS, int NV, bool FULL>
struct Part {
    int first[NV], over[NV];
    __device__ explicit Part(int hidden)
    {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int k = (i * THREADS + (int)threadIdx.x % THREADS) * 8;
            first[i] = FULL ? k : min(k, hidden - 8);
            over[i] = k - first[i];
        }
    }
    __device__ int skip(int i) const { return FULL ? 0 : over[i]; }
    template <typename T>
    __device__ void load(Words<T> *r, const T *row) const
    {
#pragma unroll
        for (int i = 0; i < NV; ++i) r[i] = load_words(row + first[i]);
    }
    // the i-th's elements of a vector of any of the types
    __device__ void load(float *v, int i, const void *p, int type) const
    {
        int at = first[i];
        asm volatile("" : "+v"(at));   // where it is loaded again for every row it is not to be kept instead
        auto convert = [&](auto t) {
            using T = decltype(t);
            const Words<T> w = load_words(static_cast<const T *>(p) + at);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = element<T>(w, j);
        };
        if (type == HAPMOE_F32)
            convert(float());
        else if (type == HAPMOE_BF16)
            convert(bf16());
        else
            convert(f16());
    }
    template <typename T>
    __device__ void store(T *row, int i, const float *v) const
    {
        if (skip(i) == 0) {
            store_words(row + first[i], words_of<T>(v));
        } else {
#pragma unroll
            for (int j = 1; j < 8; ++j)
                if (j >= skip(i)) row[first[i] + j] = from_f32<T>(v[j]);
        }
    }
};

// Rows of a workgroup: 1, or one a wave where a wave has a row.  Rows go on by the grid; the next one's loads are on their
// way while one is summed.
template <typename T, int THREADS, int NV, bool FULL>
__global__ __launch_bounds__(THREADS > 256 ? THREADS : 256) void k_norm(
    const T *__restrict__ x, int64_t stride, int64_t rows, int hidden, const void *__restrict__ weight,
    const void *__restrict__ bias, int weight_type, float eps, float *__restrict__ mean, float *__restrict__ rstd,
    T *__restrict__ y)
{
    constexpr int kRows = THREADS < 256 ? 256 / THREADS : 1;
    __shared__ float sh[2 * THREADS / 64][1];
    const Part<THREADS, NV, FULL> p(hidden);
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / THREADS;
    if (r >= rows) return;
    Words<T> next[NV];
    p.load(next, x + r * stride);
    float w[NV][8], b[NV][8] = {};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        p.load(w[i], i, weight, weight_type);
        if (bias) p.load(b[i], i, bias, weight_type);
    }
    for (int turn = 0; r < rows; r += step, turn ^= 1) {
        float v[NV][8];
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = j >= p.skip(i) ? element<T>(next[i], j) : 0.0f;
        if (r + step < rows) p.load(next, x + (r + step) * stride);
        float m = 0.0f, s = 0.0f;
        if (mean) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) m += v[i][j];
            row_sum<THREADS, 1>(&m, sh, 0);
            m /= (float)hidden;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = j >= p.skip(i) ? v[i][j] - m : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s = __builtin_fmaf(v[i][j], v[i][j], s);
        row_sum<THREADS, 1>(&s, sh, mean ? 1 : turn);
        const float rs = 1.0f / sqrtf(s / (float)hidden + eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = __builtin_fmaf(v[i][j] * rs, w[i][j], b[i][j]);
            p.store(y + r * hidden, i, v[i]);
        }
        if (threadIdx.x % THREADS == 0) {
            if (mean) mean[r] = m;
            rstd[r] = rs;
        }
    }
}

// Keeps the compiler from holding what it computed of w, in 32 bits for every element.
template <typename V>
__device__ inline void forget(V &w)
{
#pragma unroll
    for (unsigned i = 0; i < sizeof(V) / 4; ++i) {
        uint32_t x = w[i];
        asm volatile("" : "+v"(x));
        w[i] = x;
    }
}

// What the gradient reads of a row.
template <typename T, int NV, bool ADD>
struct Rows {
    Words<T> x[NV], g[NV], more[ADD ? NV : 1];
    float mean, rstd;
};

// The same rows' gradients, and in the thread of a column its sums for the weight and the bias:
// part[blockIdx.x][2][hidden].  All of the next row is on its way while one is summed, but where 1,024 threads have 128
// registers each, which the sums take half of: there a row is loaded when its turn comes, and the weight twice.
template <typename T, int THREADS, int NV, bool FULL, bool ADD>
__global__ __launch_bounds__(THREADS > 256 ? THREADS : 256) void k_norm_backward(
    const T *__restrict__ d_y, int64_t d_y_stride, const T *__restrict__ x, int64_t x_stride, int64_t rows, int hidden,
    const void *__restrict__ weight, int weight_type, const float *__restrict__ mean, const float *__restrict__ rstd,
    const T *__restrict__ add, int64_t add_stride, T *__restrict__ d_x, float *__restrict__ part)
{
    constexpr int kRows = THREADS < 256 ? 256 / THREADS : 1;
    constexpr bool kAhead = THREADS < 1024;
    __shared__ float sh[2 * THREADS / 64][2];
    __shared__ float joined[kRows > 1 ? kRows * THREADS * NV * 8 : 1];
    const Part<THREADS, NV, FULL> p(hidden);
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / THREADS;
    Rows<T, NV, ADD> next, now;
    float w[kAhead ? NV : 1][8], sum_w[NV][8] = {}, sum_b[NV][8] = {};
    auto load = [&](int64_t row) {
        p.load(next.x, x + row * x_stride);
        p.load(next.g, d_y + row * d_y_stride);
        if constexpr (ADD && kAhead) p.load(next.more, add + row * add_stride);
        next.mean = mean ? mean[row] : 0.0f;
        next.rstd = rstd[row];
    };
    if (kAhead && r < rows) load(r);
    auto weights = [&](int i) { p.load(w[kAhead ? i : 0], i, weight, weight_type); };
    if constexpr (kAhead)
#pragma unroll
        for (int i = 0; i < NV; ++i) weights(i);
    for (int turn = 0; r < rows; r += step, turn ^= 1) {
        if constexpr (!kAhead) load(r);
        now = next;
        if (kAhead && r + step < rows) load(r + step);
        const float m = now.mean, rs = now.rstd;
        float s[2] = {};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if constexpr (!kAhead) weights(i);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = j >= p.skip(i) ? element<T>(now.g[i], j) : 0.0f;
                const float hat = (element<T>(now.x[i], j) - m) * rs, g = d * w[kAhead ? i : 0][j];
                sum_w[i][j] = __builtin_fmaf(d, hat, sum_w[i][j]);
                sum_b[i][j] += d;
                s[0] += g;
                s[1] = __builtin_fmaf(g, hat, s[1]);
            }
            forget(now.g[i]);
            forget(now.x[i]);
        }
        row_sum<THREADS, 2>(s, sh, turn);
        const float a = mean ? s[0] / (float)hidden : 0.0f, b = s[1] / (float)hidden;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float o[8];
            if constexpr (!kAhead) {
                weights(i);
                if constexpr (ADD) now.more[i] = load_words(add + r * add_stride + p.first[i]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float g = element<T>(now.g[i], j) * w[kAhead ? i : 0][j], hat = (element<T>(now.x[i], j) - m) * rs;
                o[j] = rs * __builtin_fmaf(-hat, b, g - a);
                if constexpr (ADD) o[j] += element<T>(now.more[i], j);
            }
            p.store(d_x + r * hidden, i, o);
        }
    }
    float *const to = part + (int64_t)blockIdx.x * 2 * hidden;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float(*const sum)[8] = which ? sum_b : sum_w;
        if constexpr (kRows > 1) {   // the waves' sums, in their order
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    joined[((threadIdx.x / THREADS * NV + i) * 8 + j) * THREADS + threadIdx.x % THREADS] = sum[i][j];
            __syncthreads();
            if (threadIdx.x < THREADS) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
#pragma unroll
                        for (int k = 1; k < kRows; ++k)
                            sum[i][j] += joined[((k * NV + i) * 8 + j) * THREADS + threadIdx.x];
                    p.store(to + which * hidden, i, sum[i]);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) p.store(to + which * hidden, i, sum[i]);
        }
    }
}

// Rows of any length, read again from the caches.  A thread adds up to 2^16 elements of a long row one after another, so
// its sums S are in 64 bits: in 32 a row of 2^20 equal elements had a mean off by 4e-5 of it (bf16, 4,096 x 20,480: forward
// 208 us, 205 in 32 bits, backward 313, 312).  Of rows of less than 8 elements each thread has one at most: 32 bits, as
// 2^20 of 7 take 817 us forward, 997 in 64.
// Of the workgroup, in every thread; sh: one place a wave.
template <typename S>
__device__ inline S workgroup_sum(S v, S *sh)
{
    v = wave_reduce(v, Sum());
    __syncthreads();   // what was there is read
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    S sum = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) sum += sh[w];
    return sum;
}

__device__ inline float weight_at(const void *p, int type, int64_t h)
{
    return type == HAPMOE_F32    ? static_cast<const float *>(p)[h]
           : type == HAPMOE_BF16 ? to_f32(static_cast<const bf16 *>(p)[h])
                                 : to_f32(static_cast<const f16 *>(p)[h]);
}

template <typename T, typename S>
__global__ __launch_bounds__(kThreads) void k_norm_long(const T *__restrict__ x, int64_t stride, int64_t rows,
                                                        int64_t hidden, const void *__restrict__ weight,
                                                        const void *__restrict__ bias, int weight_type, float eps,
                                                        float *__restrict__ mean, float *__restrict__ rstd,
                                                        T *__restrict__ y)
{
    __shared__ S sh[kThreads / 64];
    const int64_t r = workgroup();
    if (r >= rows) return;
    const T *const row = x + r * stride;
    float m = 0.0f;
    S s = 0;
    if (mean) {
        for (int64_t h = threadIdx.x; h < hidden; h += kThreads) s += to_f32(row[h]);
        m = (float)(workgroup_sum(s, sh) / (S)hidden);
        s = 0;
    }
    for (int64_t h = threadIdx.x; h < hidden; h += kThreads) {
        const S d = to_f32(row[h]) - m;
        s += d * d;
    }
    const float rs = 1.0f / sqrtf((float)(workgroup_sum(s, sh) / (S)hidden) + eps);
    for (int64_t h = threadIdx.x; h < hidden; h += kThreads)
        y[r * hidden + h] = from_f32<T>((to_f32(row[h]) - m) * rs * weight_at(weight, weight_type, h) +
                                        (bias ? weight_at(bias, weight_type, h) : 0.0f));
    if (threadIdx.x == 0) {
        if (mean) mean[r] = m;
        rstd[r] = rs;
    }
}

template <typename T, typename S>
__global__ __launch_bounds__(kThreads) void k_norm_backward_long(
    const T *__restrict__ d_y, int64_t d_y_stride, const T *__restrict__ x, int64_t x_stride, int64_t rows,
    int64_t hidden, const void *__restrict__ weight, int weight_type, const float *__restrict__ mean,
    const float *__restrict__ rstd, const T *__restrict__ add, int64_t add_stride, T *__restrict__ d_x)
{
    __shared__ S sh[kThreads / 64];
    const int64_t r = workgroup();
    if (r >= rows) return;
    const T *const row = x + r * x_stride, *const g_row = d_y + r * d_y_stride;
    const float m = mean ? mean[r] : 0.0f, rs = rstd[r];
    S sum_g = 0, sum_hat = 0;
    for (int64_t h = threadIdx.x; h < hidden; h += kThreads) {
        const float g = to_f32(g_row[h]) * weight_at(weight, weight_type, h);
        sum_g += g;
        sum_hat += g * ((to_f32(row[h]) - m) * rs);
    }
    const float a = mean ? (float)(workgroup_sum(sum_g, sh) / (S)hidden) : 0.0f;
    const float b = (float)(workgroup_sum(sum_hat, sh) / (S)hidden);
    for (int64_t h = threadIdx.x; h < hidden; h += kThreads) {
        const float g = to_f32(g_row[h]) * weight_at(weight, weight_type, h), hat = (to_f32(row[h]) - m) * rs;
        const float d = rs * (g - a - hat * b);
        d_x[r * hidden + h] = from_f32<T>(add ? to_f32(add[r * add_stride + h]) + d : d);
    }
}

// Sums of the rows of a part: part[blockIdx.y][2][hidden].
template <typename T>
__global__ __launch_bounds__(kThreads) void k_norm_weight(const T *__restrict__ d_y, int64_t d_y_stride,
                                                          const T *__restrict__ x, int64_t x_stride, int64_t rows,
                                                          int64_t hidden, const float *__restrict__ mean,
                                                          const float *__restrict__ rstd, int64_t each,
                                                          float *__restrict__ part)
{
    const int64_t h = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (h >= hidden) return;
    const int64_t lo = blockIdx.y * each, hi = lo + each < rows ? lo + each : rows;
    double w = 0.0, b = 0.0;   // in 64 bits, as a part may have many rows: 2^11 of 2^20 short ones
    for (int64_t r = lo; r < hi; ++r) {
        const float g = to_f32(d_y[r * d_y_stride + h]);
        w += g * ((to_f32(x[r * x_stride + h]) - (mean ? mean[r] : 0.0f)) * rstd[r]);
        b += g;
    }
    part[(blockIdx.y * 2) * hidden + h] = (float)w;
    part[(blockIdx.y * 2 + 1) * hidden + h] = (float)b;
}

// Sums over the parts: a workgroup has 64 columns, each of its waves a run of the parts, then the waves in their order.
constexpr int kJoinThreads = 1024;
__global__ __launch_bounds__(kJoinThreads) void k_norm_join(const float *__restrict__ part, int parts, int64_t hidden,
                                                            float *__restrict__ d_weight, float *__restrict__ d_bias)
{
    constexpr int kWaves = kJoinThreads / 64, kAhead = 8;
    __shared__ float sh[kWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    float *const out = blockIdx.y ? d_bias : d_weight;
    const int run = (parts + kWaves - 1) / kWaves, lo = min(wave * run, parts), hi = min(lo + run, parts);
    float sum = 0.0f;
    if (c < hidden) {
        const float *from = part + blockIdx.y * hidden + c;
        for (int p = lo; p < hi; p += kAhead) {
            float v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) v[i] = p + i < hi ? from[(int64_t)(p + i) * 2 * hidden] : 0.0f;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) sum += v[i];
        }
    }
    sh[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && c < hidden) {
        sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += sh[w][lane];
        out[c] = sum;
    }
}

// How a row is shared: threads, vectors of 8 each; 0 threads: a row that is too long to be held, or shorter than one.
struct Share {
    int threads, vectors;
};
Share share_of(int64_t hidden)
{
    if (hidden < 8 || hidden > 16384) return {0, 0};
    if (hidden <= 512) return {64, 1};
    if (hidden <= 1024) return {64, 2};
    if (hidden <= 2048) return {256, 1};
    if (hidden <= 4096) return {256, 2};
    if (hidden <= 8192) return {512, 2};
    return {1024, 2};
}
template <typename F>
hipError_t by_share(Share sh, bool full, F f)
{
    using std::integral_constant;
    auto g = [&](auto threads, auto vectors) {
        return full ? f(threads, vectors, std::true_type()) : f(threads, vectors, std::false_type());
    };
    if (sh.threads == 64 && sh.vectors == 1) return g(integral_constant<int, 64>(), integral_constant<int, 1>());
    if (sh.threads == 64) return g(integral_constant<int, 64>(), integral_constant<int, 2>());
    if (sh.threads == 256 && sh.vectors == 1) return g(integral_constant<int, 256>(), integral_constant<int, 1>());
    if (sh.threads == 256) return g(integral_constant<int, 256>(), integral_constant<int, 2>());
    if (sh.threads == 512) return g(integral_constant<int, 512>(), integral_constant<int, 2>());
    return g(integral_constant<int, 1024>(), integral_constant<int, 2>());
}
bool is_full(Share sh, int64_t hidden) { return hidden == sh.threads * sh.vectors * 8; }
int64_t rows_at_once(Share sh) { return sh.threads < 256 ? 256 / sh.threads : 1; }
unsigned threads_of(Share sh) { return sh.threads < 256 ? 256 : sh.threads; }

// Workgroups of 256 threads a CU, or as many threads.  us, bf16, 32,768 x 4,096: forward by 4, 5, 6 100, 102, 102 (4,096 rows
// 15 by each), backward with add by 2, 3, 4 208, 218, 227 (30, 32, 35): more are more parts of the weight's sums.
constexpr int kForward = 4, kBackward = 2;
int64_t workgroups_of(Share sh, int64_t rows, int a_cu)
{
    const int64_t n = ceil_div(rows, rows_at_once(sh));
    const int each = a_cu * 256 / (int)threads_of(sh), most = 256 * (each > 0 ? each : 1);
    return n < most ? n : most;
}
// Workgroups of the gradient, each a part of the weight's sums.
int parts_of(int64_t rows, int64_t hidden)
{
    const Share sh = share_of(hidden);
    if (sh.threads) return (int)workgroups_of(sh, rows, kBackward);
    int64_t most = (int64_t)2048 * kThreads / hidden;   // of long rows few: the columns fill the card
    most = most < 1 ? 1 : most > 512 ? 512 : most;
    return (int)(rows < most ? rows : most);
}

template <typename F>
hipError_t by_type(int type, F f)
{
    if (type == HAPMOE_F32) return f(float());
    if (type == HAPMOE_BF16) return f(bf16());
    return f(f16());
}

}  // namespace

int64_t layer_norm_ws_bytes(int64_t rows, int64_t hidden) { return parts_of(rows, hidden) * 2 * hidden * 4; }

hipError_t launch_layer_norm(const LayerNorm &a, hipStream_t s)
{
    return by_type(a.type, [&](auto t) {
        using T = decltype(t);
        const T *x = static_cast<const T *>(a.x);
        const Share sh = share_of(a.hidden);
        if (!sh.threads) {
            hipLaunchKernelGGL((a.hidden < 8 ? k_norm_long<T, float> : k_norm_long<T, double>), many(a.rows), dim3(kThreads),
                               0, s, x, a.x_stride, a.rows, a.hidden, a.weight, a.bias, a.weight_type, a.eps, a.mean, a.rstd,
                               static_cast<T *>(a.out));
            return hipGetLastError();
        }
        return by_share(sh, is_full(sh, a.hidden), [&](auto threads, auto vectors, auto full) {
            hipLaunchKernelGGL((k_norm<T, decltype(threads)::value, decltype(vectors)::value, decltype(full)::value>),
                               dim3((unsigned)workgroups_of(sh, a.rows, kForward)), dim3(threads_of(sh)), 0, s, x,
                               a.x_stride, a.rows, (int)a.hidden, a.weight, a.bias, a.weight_type, a.eps, a.mean, a.rstd,
                               static_cast<T *>(a.out));
            return hipGetLastError();
        });
    });
}

hipError_t launch_layer_norm_backward(const LayerNorm &a, hipStream_t s)
{
    float *part = static_cast<float *>(a.ws);
    const int parts = parts_of(a.rows, a.hidden);
    const hipError_t e = by_type(a.type, [&](auto t) {
        using T = decltype(t);
        const T *d_y = static_cast<const T *>(a.d_y), *x = static_cast<const T *>(a.x);
        const T *add = static_cast<const T *>(a.add);
        T *d_x = static_cast<T *>(a.out);
        if (parts == 0) return hipSuccess;
        const Share sh = share_of(a.hidden);
        if (sh.threads)
            return by_share(sh, is_full(sh, a.hidden), [&](auto threads, auto vectors, auto full) {
                constexpr int THREADS = decltype(threads)::value, NV = decltype(vectors)::value;
                constexpr bool FULL = decltype(full)::value;
                hipLaunchKernelGGL((add ? k_norm_backward<T, THREADS, NV, FULL, true>
                                        : k_norm_backward<T, THREADS, NV, FULL, false>),
                                   dim3(parts), dim3(threads_of(sh)), 0, s, d_y, a.d_y_stride, x, a.x_stride, a.rows,
                                   (int)a.hidden, a.weight, a.weight_type, a.mean, a.rstd, add, a.add_stride, d_x, part);
                return hipGetLastError();
            });
        hipLaunchKernelGGL((a.hidden < 8 ? k_norm_backward_long<T, float> : k_norm_backward_long<T, double>), many(a.rows),
                           dim3(kThreads), 0, s, d_y, a.d_y_stride, x, a.x_stride, a.rows, a.hidden, a.weight,
                           a.weight_type, a.mean, a.rstd, add, a.add_stride, d_x);
        hipLaunchKernelGGL(k_norm_weight<T>, dim3((unsigned)ceil_div(a.hidden, kThreads), parts), dim3(kThreads), 0, s,
                           d_y, a.d_y_stride, x, a.x_stride, a.rows, a.hidden, a.mean, a.rstd, ceil_div(a.rows, parts),
                           part);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_norm_join, dim3((unsigned)ceil_div(a.hidden, 64), a.d_bias ? 2 : 1), dim3(kJoinThreads), 0, s,
                       part, parts, a.hidden, a.d_weight, a.d_bias);
    return hipGetLastError();
}

}  // namespace hapmoe
