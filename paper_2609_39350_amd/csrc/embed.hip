// Rows of a table by token, and the table's gradient.
//
// out[t] = scale table[token[t]], a row of zeros where the token is none of the table's.
//
// The gradient's row of a token is the sum over its places in the order of t, with no atomics.  A workgroup sorts up to
// 16,384 places by token in LDS: a stable counting sort, 9 bits of the token a pass; more places are several such
// segments, whose sums follow each other.  Then workgroups take equal chunks of the sorted places, whatever the tokens' shares: a
// token that lies within a chunk is written, one that goes on into the next leaves its sums in the workspace, and a last
// launch puts those together.
#include "operators.h"

namespace hapmoe {
namespace {

constexpr int kThreads = 256;
constexpr int kSegment = 16384;    // places of a sort: tokens, two orders and counts in 144 KB of LDS
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kSteps = kSegment / kSortThreads;
constexpr int kDigit = 9, kBins = 1 << kDigit;

template <typename I>
__device__ inline int64_t token_at(const void *token, int64_t t)
{
    return (int64_t) static_cast<const I *>(token)[t];
}

template <typename T, typename I, bool VEC>
__global__ __launch_bounds__(kThreads) void k_embed(const void *__restrict__ token, int64_t tokens,
                                                    const T *__restrict__ table, int64_t stride, int64_t vocab,
                                                    int64_t hidden, float scale, T *__restrict__ out)
{
    const int64_t t = workgroup(), h = ((int64_t)blockIdx.y * kThreads + threadIdx.x) * (VEC ? 8 : 1);
    if (t >= tokens || h >= hidden) return;
    const int64_t v = token_at<I>(token, t);
    const bool real = (uint64_t)v < (uint64_t)vocab;
    if constexpr (VEC) {
        Vec8<T> r = {};
        if (real) {
            r = *reinterpret_cast<const Vec8<T> *>(table + v * stride + h);
#pragma unroll
            for (int i = 0; i < 8; ++i) r.v[i] = from_f32<T>(to_f32(r.v[i]) * scale);
        }
        *reinterpret_cast<Vec8<T> *>(out + t * hidden + h) = r;
    } else {
        out[t * hidden + h] = from_f32<T>(real ? to_f32(table[v * stride + h]) * scale : 0.0f);
    }
}

// Segment blockIdx.x: sorted[i] = (token, place) for its places, the tokens ascending, the places of one ascending.
// Tokens that are none of the table's count as `vocab`.  bits: of vocab.
template <typename I>
__global__ __launch_bounds__(kSortThreads) void k_sort(const void *__restrict__ token, int64_t tokens, int64_t vocab,
                                                       int bits, int2 *__restrict__ sorted)
{
    __shared__ int key[kSegment];
    __shared__ uint16_t order[2][kSegment], count[kSortWaves][kBins];
    __shared__ int sh[kSortWaves];
    const int64_t first = (int64_t)blockIdx.x * kSegment;
    const int n = tokens - first < kSegment ? (int)(tokens - first) : kSegment;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < n; i += kSortThreads) {
        const int64_t v = token_at<I>(token, first + i);
        key[i] = (uint64_t)v < (uint64_t)vocab ? (int)v : (int)vocab;
        order[0][i] = (uint16_t)i;
    }
    const int run = (n + kSortThreads - 1) / kSortThreads * 64;   // a wave's
    const int lo = wave * run, hi = min(lo + run, n);
    int from = 0;
    for (int shift = 0; shift < bits; shift += kDigit, from ^= 1) {
        const int digits = min(kDigit, bits - shift);
        for (int i = threadIdx.x; i < kSortWaves * kBins; i += kSortThreads) (&count[0][0])[i] = 0;
        __syncthreads();
        int held[kSteps], rank[kSteps];   // place and digit, rank among the wave's of its digit
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int i = lo + s * 64 + lane;
            if (lo + s * 64 >= hi) break;
            const bool in = i < hi;
            const int place = in ? order[from][i] : 0;
            const int digit = in ? key[place] >> shift & ((1 << digits) - 1) : 0;
            uint64_t same = __ballot(in);
            for (int b = 0; b < digits; ++b) {
                const uint64_t on = __ballot(digit >> b & 1);
                same &= digit >> b & 1 ? on : ~on;
            }
            const uint64_t below = same & ((1ull << lane) - 1);
            held[s] = place | digit << 16;
            rank[s] = in ? count[wave][digit] + __popcll(below) : 0;
            // every lane's read is before the writes of each digit's lowest lane
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (in && below == 0) count[wave][digit] += (uint16_t)__popcll(same);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        // where each wave's places of a digit begin: those of lower digits, then of the waves before
        int total = 0, inc;
        if (threadIdx.x < kBins)
            for (int w = 0; w < kSortWaves; ++w) {
                const int c = count[w][threadIdx.x];
                count[w][threadIdx.x] = (uint16_t)total;
                total += c;
            }
        inc = total;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(inc, d, 64);
            if (lane >= d) inc += o;
        }
        if (lane == 63) sh[wave] = inc;
        __syncthreads();
        if (threadIdx.x < kBins) {
            int before = inc - total;
            for (int w = 0; w < wave; ++w) before += sh[w];
            for (int w = 0; w < kSortWaves; ++w) count[w][threadIdx.x] += (uint16_t)before;
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int i = lo + s * 64 + lane;
            if (i < hi) order[from ^ 1][count[wave][held[s] >> 16] + rank[s]] = (uint16_t)(held[s] & 0xffff);
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < n; i += kSortThreads) {
        const int place = order[from][i];
        sorted[first + i] = make_int2(key[place], (int)first + place);
    }
}

__global__ __launch_bounds__(kThreads) void k_zero(float *__restrict__ p, int64_t n)
{
    const int64_t i = (workgroup() * kThreads + threadIdx.x) * 4;
    if (i + 4 <= n && ((uintptr_t)p & 15) == 0) {
        *reinterpret_cast<float4 *>(p + i) = make_float4(0, 0, 0, 0);
    } else {
        for (int64_t j = i; j < i + 4 && j < n; ++j) p[j] = 0.0f;
    }
}

// A row of the gradient, or what is added to it.
template <int N>
__device__ inline void put(float *__restrict__ to, const float *sum, float scale, bool add)
{
#pragma unroll
    for (int i = 0; i < N; ++i) to[i] = (add ? to[i] : 0.0f) + sum[i] * scale;
}

// Chunk `workgroup` of a segment of n sorted places, N columns a thread.
template <typename T, int N>
__global__ __launch_bounds__(kThreads) void k_embed_sum(const T *__restrict__ d_out, int64_t stride, int64_t hidden,
                                                        const int2 *__restrict__ sorted, int n, int chunk, int vocab,
                                                        float scale, bool add, float *__restrict__ d_table,
                                                        float *__restrict__ part)
{
    const int64_t h = ((int64_t)blockIdx.y * kThreads + threadIdx.x) * N;
    if (h >= hidden) return;
    const int lo = blockIdx.x * chunk, hi = min(lo + chunk, n);
    float sum[N] = {};
    for (int i = lo; i < hi; ++i) {
        const int2 at = sorted[i];
        if (at.x == vocab) break;
        const T *const row = d_out + at.y * stride + h;
#pragma unroll
        for (int c = 0; c < N; ++c) sum[c] += to_f32(row[c]);
        const bool goes_on = i + 1 < n && sorted[i + 1].x == at.x;
        if (goes_on && i + 1 < hi) continue;
        const bool began = lo > 0 && sorted[lo - 1].x == at.x;
        if (began || goes_on) {
            float *const to = part + ((int64_t)blockIdx.x * 2 + (began ? 0 : 1)) * hidden + h;
#pragma unroll
            for (int c = 0; c < N; ++c) to[c] = sum[c];
        } else {
            put<N>(d_table + at.x * hidden + h, sum, scale, add);
        }
#pragma unroll
        for (int c = 0; c < N; ++c) sum[c] = 0.0f;
    }
}

// The token that begins in chunk `workgroup` and goes on: its sums there and in the chunks that follow.
template <int N>
__global__ __launch_bounds__(kThreads) void k_embed_join(int64_t hidden, const int2 *__restrict__ sorted, int n,
                                                         int chunk, int vocab, float scale, bool add,
                                                         const float *__restrict__ part, float *__restrict__ d_table)
{
    const int64_t h = ((int64_t)blockIdx.y * kThreads + threadIdx.x) * N;
    const int lo = blockIdx.x * chunk, hi = lo + chunk;
    if (h >= hidden || hi >= n) return;
    const int token = sorted[hi - 1].x;
    if (token == vocab || sorted[hi].x != token || (lo > 0 && sorted[lo - 1].x == token)) return;
    float sum[N];
    const float *from = part + ((int64_t)blockIdx.x * 2 + 1) * hidden + h;
#pragma unroll
    for (int c = 0; c < N; ++c) sum[c] = from[c];
    for (int i = hi; i < n && sorted[i].x == token; i += chunk) {
        from = part + (int64_t)(i / chunk) * 2 * hidden + h;
#pragma unroll
        for (int c = 0; c < N; ++c) sum[c] += from[c];
    }
    put<N>(d_table + token * hidden + h, sum, scale, add);
}

int chunk_of(int64_t tokens) { return tokens < 8192 ? 8 : 32; }
int64_t chunks_of(int64_t tokens) { return ceil_div(tokens < kSegment ? tokens : kSegment, chunk_of(tokens)); }

template <typename F>
hipError_t by_type(int type, F f)
{
    if (type == HAPMOE_F32) return f(float());
    if (type == HAPMOE_BF16) return f(bf16());
    return f(f16());
}

}  // namespace

int64_t embed_ws_bytes(int64_t tokens, int64_t hidden) { return ceil_div(tokens, 2) * 16 + chunks_of(tokens) * 2 * hidden * 4; }

hipError_t launch_embed(const void *token, bool wide, int64_t tokens, const void *table, int type, int64_t stride,
                        int64_t vocab, int64_t hidden, float scale, void *out, hipStream_t s)
{
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        const int64_t bytes = sizeof(T) * 8;
        const bool vec = hidden % 8 == 0 && stride % 8 == 0 && aligned(table, bytes) && aligned(out, bytes);
        auto *kernel = wide ? (vec ? k_embed<T, int64_t, true> : k_embed<T, int64_t, false>)
                            : (vec ? k_embed<T, int32_t, true> : k_embed<T, int32_t, false>);
        hipLaunchKernelGGL(kernel, many(tokens, (unsigned)ceil_div(hidden, kThreads * (vec ? 8 : 1))), dim3(kThreads), 0,
                           s, token, tokens, static_cast<const T *>(table), stride, vocab, hidden, scale,
                           static_cast<T *>(out));
        return hipGetLastError();
    });
}

hipError_t launch_embed_backward(const void *d_out, int type, int64_t stride, int64_t tokens, int64_t hidden,
                                 const void *token, bool wide, int64_t vocab, float scale, bool add, float *d_table,
                                 void *ws, hipStream_t s)
{
    if (!add)
        hipLaunchKernelGGL(k_zero, many(ceil_div(vocab * hidden, 4 * kThreads)), dim3(kThreads), 0, s, d_table,
                           vocab * hidden);
    if (tokens == 0) return hipGetLastError();
    int2 *sorted = static_cast<int2 *>(ws);
    float *part = reinterpret_cast<float *>(sorted + ceil_div(tokens, 2) * 2);
    int bits = 1;
    while (vocab >> bits) ++bits;
    hipLaunchKernelGGL((wide ? k_sort<int64_t> : k_sort<int32_t>), dim3((unsigned)ceil_div(tokens, kSegment)),
                       dim3(kSortThreads), 0, s, token, tokens, vocab, bits, sorted);
    const int chunk = chunk_of(tokens);
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        for (int64_t first = 0; first < tokens; first += kSegment) {
            const int n = (int)(tokens - first < kSegment ? tokens - first : kSegment);
            const dim3 grid((unsigned)ceil_div(n, chunk), (unsigned)ceil_div(hidden, kThreads));
            hipLaunchKernelGGL((k_embed_sum<T, 1>), grid, dim3(kThreads), 0, s, static_cast<const T *>(d_out), stride,
                               hidden, sorted + first, n, chunk, (int)vocab, scale, add || first > 0, d_table, part);
            hipLaunchKernelGGL((k_embed_join<1>), grid, dim3(kThreads), 0, s, hidden, sorted + first, n, chunk,
                               (int)vocab, scale, add || first > 0, part, d_table);
        }
        return hipGetLastError();
    });
}

}  // namespace hapmoe
