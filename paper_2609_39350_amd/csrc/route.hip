// The router: of every token's logits the top_k largest, their softmax weights,
// and the order that puts each expert's rows together; and its gradient.
//
// Sixteen lanes take a token (four tokens a wave): lane l holds the logits
// l * PER .. l * PER + PER - 1 in registers, so a choice is two reductions over
// a row of lanes (the largest logit, then the lowest index that has it), each
// four rotations without LDS, and the softmax's maximum and sum come of the same.
//
// The order is stable, so it needs every row's rank among the earlier rows of
// its expert.  A workgroup ranks its own tokens' rows: one wave takes 64 rows at
// a time, finds for each lane the lanes of the same expert by a ballot a bit of
// the expert's number, and keeps the counts so far in LDS.  A second kernel sums
// the workgroups' counts over the workgroups, a third adds the experts' offsets
// and writes both directions of the order.  Up to 64 tokens one workgroup does
// all of it in one launch, which is what a decoding step waits for.
#include "operators.h"

namespace hapmoe {
namespace {

constexpr int kThreads = 256;
constexpr int kPass = kThreads / 16;   // tokens of a workgroup at a time
constexpr int kOneLaunch = 64;         // tokens
constexpr int kPlaceRows = 1024;       // rows of a workgroup of the last kernel

// tokens of a workgroup
__host__ __device__ inline int group_tokens(int64_t tokens) { return tokens <= 64 * 512 ? 32 : 64; }

// A token's logits in the registers of 16 lanes; closed experts (-inf, NaN, past the end, keep = 0) are -inf.
template <typename T, int PER, bool VEC>
__device__ inline void load_logits(float *v, const T *__restrict__ row, int lane, int experts, bool keep)
{
    const int base = lane * PER;
    if constexpr (VEC) {
        constexpr int kStep = 16 / (int)sizeof(T) < PER ? 16 / (int)sizeof(T) : PER;
        struct alignas(kStep * sizeof(T)) Piece {
            T x[kStep];
        };
#pragma unroll
        for (int c = 0; c < PER; c += kStep) {
            const Piece p = *reinterpret_cast<const Piece *>(row + base + c);
#pragma unroll
            for (int i = 0; i < kStep; ++i) v[c + i] = to_f32(p.x[i]);
        }
    } else {
#pragma unroll
        for (int c = 0; c < PER; ++c) v[c] = base + c < experts ? to_f32(row[base + c]) : -INFINITY;
    }
#pragma unroll
    for (int c = 0; c < PER; ++c) v[c] = keep && v[c] > -INFINITY ? v[c] : -INFINITY;
}

// exp(x - top), 1 where x is the largest: also where both are infinite
__device__ inline float exp_from(float x, float top) { return x == top ? 1.0f : expf(x - top); }

template <int PER>
__device__ inline float softmax_sum(const float *v, float top)
{
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < PER; ++c) s += v[c] == -INFINITY ? 0.0f : exp_from(v[c], top);
    return row_reduce(s, Sum());
}

template <int PER>
__device__ inline float largest(const float *v)
{
    float m = v[0];
#pragma unroll
    for (int c = 1; c < PER; ++c) m = fmaxf(m, v[c]);
    return row_reduce(m, Max());
}

// For each lane the lanes of the wave whose `key` is the same; bits: of the keys.
__device__ inline uint64_t same_key(int key, int bits)
{
    uint64_t same = ~0ull;
    for (int b = 0; b < bits; ++b) {
        const uint64_t on = __ballot((key >> b) & 1);
        same &= (key >> b) & 1 ? on : ~on;
    }
    return same;
}

// Exclusive sums over count[0 .. experts) by the workgroup, in place; returns the total.  sh: one int a wave.
__device__ inline int scan_counts(int *count, int experts, int *sh)
{
    constexpr int kPer = HAPMOE_MAX_EXPERTS / kThreads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int own[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = threadIdx.x * kPer + i;
        own[i] = e < experts ? count[e] : 0;
        sum += own[i];
    }
    int inc = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(inc, d, 64);
        if (lane >= d) inc += o;
    }
    if (lane == 63) sh[wave] = inc;
    __syncthreads();
    int before = inc - sum, total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        before += w < wave ? sh[w] : 0;
        total += sh[w];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = threadIdx.x * kPer + i;
        if (e < experts) count[e] = before;
        before += own[i];
    }
    __syncthreads();
    return total;
}

// Choices, weights and ranks.  ALONE: the only workgroup, which finishes the order too; else rank goes to `place` and
// the workgroup's counts to hist[workgroup][experts].
template <typename T, int PER, bool VEC, bool ALONE>
__global__ __launch_bounds__(kThreads) void k_choose(const T *__restrict__ logits, int64_t stride, int64_t tokens,
                                                     int experts, int top_k, const uint8_t *__restrict__ keep,
                                                     int renormalize, int group, int bits, float *__restrict__ weight,
                                                     int32_t *__restrict__ expert, int32_t *__restrict__ place,
                                                     int32_t *__restrict__ hist, int32_t *__restrict__ count,
                                                     int32_t *__restrict__ offset, int32_t *__restrict__ slot)
{
    extern __shared__ int lds[];
    int *sums = lds;                              // [experts]
    int *chosen = lds + HAPMOE_MAX_EXPERTS;       // [group * top_k]
    __shared__ int sh[kThreads / 64];
    const int lane = threadIdx.x & 15;
    const int64_t first = (int64_t)blockIdx.x * group;
    const int here = tokens - first < group ? (int)(tokens - first) : group;
    for (int e = threadIdx.x; e < experts; e += kThreads) sums[e] = 0;
    for (int t0 = threadIdx.x >> 4; t0 < here; t0 += kPass) {
        const int64_t t = first + t0;
        float v[PER];
        load_logits<T, PER, VEC>(v, logits + t * stride, lane, experts, !keep || keep[t]);
        const float top = largest<PER>(v);
        float total = renormalize || top == -INFINITY ? 0.0f : softmax_sum<PER>(v, top);
        float won[2] = {-INFINITY, -INFINITY};   // choices lane and lane + 16
        int who[2] = {-1, -1};
        float m = top;
        for (int j = 0; j < top_k && m > -INFINITY; ++j) {
            int at = PER;
#pragma unroll
            for (int c = PER - 1; c >= 0; --c) at = v[c] == m ? c : at;
            const int best = row_reduce(at < PER ? lane * PER + at : INT32_MAX, Min());
#pragma unroll
            for (int c = 0; c < PER; ++c) v[c] = lane * PER + c == best ? -INFINITY : v[c];
            if (renormalize) total += exp_from(m, top);
            if (lane == (j & 15)) {
                won[0] = j < 16 ? m : won[0];
                who[0] = j < 16 ? best : who[0];
                won[1] = j < 16 ? won[1] : m;
                who[1] = j < 16 ? who[1] : best;
            }
            m = largest<PER>(v);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = lane + 16 * h;
            if (j < top_k) {
                weight[t * top_k + j] = who[h] < 0 ? 0.0f : exp_from(won[h], top) / total;
                expert[t * top_k + j] = who[h];
                chosen[t0 * top_k + j] = who[h];
            }
        }
    }
    __syncthreads();
    const int rows = here * top_k;
    int32_t *const mine = place + first * top_k;
    if (threadIdx.x < 64) {
        for (int r0 = 0; r0 < rows; r0 += 64) {
            const int r = r0 + (int)threadIdx.x;
            const int e = r < rows ? chosen[r] : -1;
            const uint64_t same = same_key(e + 1, bits);
            const uint64_t below = same & ((1ull << threadIdx.x) - 1);
            if (e >= 0) {
                const int rank = sums[e] + __popcll(below);
                if constexpr (ALONE)
                    chosen[r] = rank << 10 | e;   // rank < 2^11, e < 2^10
                else
                    mine[r] = rank;
            }
            // the counts before this round are read by every lane before the lowest of each expert adds to them
            __builtin_amdgcn_wave_barrier();
            if (e >= 0 && below == 0) sums[e] += __popcll(same);
            __builtin_amdgcn_wave_barrier();
        }
    }
    __syncthreads();
    if constexpr (!ALONE) {
        for (int e = threadIdx.x; e < experts; e += kThreads) hist[(int64_t)blockIdx.x * experts + e] = sums[e];
    } else {
        for (int e = threadIdx.x; e < experts; e += kThreads) count[e] = sums[e];
        const int total = scan_counts(sums, experts, sh);
        for (int e = threadIdx.x; e < experts; e += kThreads) offset[e] = sums[e];
        if (threadIdx.x == 0) offset[experts] = total;
        for (int r = threadIdx.x; r < rows; r += kThreads) {
            const int c = chosen[r];
            const int p = c < 0 ? -1 : sums[c & 1023] + (c >> 10);
            place[r] = p;
            if (p >= 0) slot[p] = r;
            if (r >= total) slot[r] = -1;
        }
    }
}

// hist[group][experts] -> the sums over the groups before, and count.  A workgroup takes 64 experts, wave w an equal
// run of the groups: its sum, the waves' sums before it, then the running sum.
constexpr int kScanWaves = 16;
__global__ __launch_bounds__(64 * kScanWaves) void k_scan_groups(int32_t *__restrict__ hist, int groups, int experts,
                                                                 int32_t *__restrict__ count)
{
    __shared__ int part[kScanWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int e = blockIdx.x * 64 + lane;
    const int run = (groups + kScanWaves - 1) / kScanWaves;
    const int lo = wave * run < groups ? wave * run : groups, hi = lo + run < groups ? lo + run : groups;
    int sum = 0;
    if (e < experts) {
#pragma unroll 16
        for (int g = lo; g < hi; ++g) sum += hist[(int64_t)g * experts + e];
    }
    part[wave][lane] = sum;
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kScanWaves; ++w) {
        before += w < wave ? part[w][lane] : 0;
        total += part[w][lane];
    }
    if (e >= experts) return;
    if (wave == 0) count[e] = total;
#pragma unroll 16
    for (int g = lo; g < hi; ++g) {
        const int64_t i = (int64_t)g * experts + e;
        const int h = hist[i];
        hist[i] = before;
        before += h;
    }
}

// rank within the group -> place and slot
__global__ __launch_bounds__(kThreads) void k_place(const int32_t *__restrict__ expert,
                                                    const int32_t *__restrict__ hist,
                                                    const int32_t *__restrict__ count, int64_t rows, int experts,
                                                    int group_rows, int32_t *__restrict__ offset,
                                                    int32_t *__restrict__ place, int32_t *__restrict__ slot)
{
    __shared__ int at[HAPMOE_MAX_EXPERTS];
    __shared__ int sh[kThreads / 64];
    for (int e = threadIdx.x; e < experts; e += kThreads) at[e] = count[e];
    __syncthreads();
    const int total = scan_counts(at, experts, sh);
    if (blockIdx.x == 0) {
        for (int e = threadIdx.x; e < experts; e += kThreads) offset[e] = at[e];
        if (threadIdx.x == 0) offset[experts] = total;
    }
    const int64_t r0 = (int64_t)blockIdx.x * kPlaceRows;
#pragma unroll
    for (int i = 0; i < kPlaceRows / kThreads; ++i) {
        const int64_t r = r0 + i * kThreads + threadIdx.x;
        if (r >= rows) break;
        const int e = expert[r];
        int p = -1;
        if (e >= 0) {
            p = at[e] + hist[r / group_rows * experts + e] + place[r];
            slot[p] = (int)r;
        }
        place[r] = p;
        if (r >= total) slot[r] = -1;
    }
}

// d_logits.  Over all experts d_i = p_i (g_i - sum_j g_j w_j), g 0 for experts not chosen: p again from the logits.
// Renormalised: w_j (g_j - sum g w) at the chosen, 0 elsewhere, and the logits are not read.
template <typename T, int PER, bool VEC>
__global__ __launch_bounds__(kThreads) void k_route_backward(
    const T *__restrict__ logits, int64_t stride, int64_t tokens, int experts, int top_k,
    const uint8_t *__restrict__ keep, int renormalize, const int32_t *__restrict__ expert,
    const float *__restrict__ weight, const float *__restrict__ d_weight, T *__restrict__ d_logits)
{
    const int lane = threadIdx.x & 15;
    const int64_t t = (int64_t)blockIdx.x * kPass + (threadIdx.x >> 4);
    if (t >= tokens) return;
    int who[2];
    float gw[2], g[2], w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int j = lane + 16 * h;
        who[h] = j < top_k ? expert[t * top_k + j] : -1;
        w[h] = who[h] >= 0 ? weight[t * top_k + j] : 0.0f;
        g[h] = who[h] >= 0 ? d_weight[t * top_k + j] : 0.0f;
        gw[h] = g[h] * w[h];
    }
    const float mean = row_reduce(gw[0] + gw[1], Sum());
    float d[PER];
    if (renormalize) {
#pragma unroll
        for (int c = 0; c < PER; ++c) d[c] = 0.0f;
    } else {
        load_logits<T, PER, VEC>(d, logits + t * stride, lane, experts, !keep || keep[t]);
        const float top = largest<PER>(d);
        const float total = top == -INFINITY ? 1.0f : softmax_sum<PER>(d, top);
#pragma unroll
        for (int c = 0; c < PER; ++c) d[c] = d[c] == -INFINITY ? 0.0f : exp_from(d[c], top) / total * -mean;
    }
    const int row = threadIdx.x & 48;   // first lane of the row within the wave
    for (int j = 0; j < top_k; ++j) {
        const int h = j >> 4;
        const int e = __shfl(h ? who[1] : who[0], row + (j & 15), 64);
        const float add = __shfl(h ? w[1] * (renormalize ? g[1] - mean : g[1])
                                   : w[0] * (renormalize ? g[0] - mean : g[0]),
                                 row + (j & 15), 64);
#pragma unroll
        for (int c = 0; c < PER; ++c) d[c] += lane * PER + c == e ? add : 0.0f;
    }
    T *out = d_logits + t * experts + lane * PER;
    if constexpr (VEC) {
        constexpr int kStep = 16 / (int)sizeof(T) < PER ? 16 / (int)sizeof(T) : PER;
        struct alignas(kStep * sizeof(T)) Piece {
            T x[kStep];
        };
#pragma unroll
        for (int c = 0; c < PER; c += kStep) {
            Piece p;
#pragma unroll
            for (int i = 0; i < kStep; ++i) p.x[i] = from_f32<T>(d[c + i]);
            *reinterpret_cast<Piece *>(out + c) = p;
        }
    } else {
#pragma unroll
        for (int c = 0; c < PER; ++c)
            if (lane * PER + c < experts) out[c] = from_f32<T>(d[c]);
    }
}

// a call's PER for its experts, and whether whole vectors can be loaded
template <typename F>
hipError_t by_experts(int experts, F f)
{
    if (experts <= 64) return f(std::integral_constant<int, 4>());
    if (experts <= 128) return f(std::integral_constant<int, 8>());
    if (experts <= 256) return f(std::integral_constant<int, 16>());
    if (experts <= 512) return f(std::integral_constant<int, 32>());
    return f(std::integral_constant<int, 64>());
}
template <typename F>
hipError_t by_type(int type, F f)
{
    if (type == HAPMOE_F32) return f(float());
    if (type == HAPMOE_BF16) return f(bf16());
    return f(f16());
}

}  // namespace

int64_t route_ws_bytes(int64_t tokens, int experts, int top_k)
{
    (void)top_k;
    if (tokens <= kOneLaunch) return 0;
    return ceil_div(tokens, group_tokens(tokens)) * experts * 4;
}

hipError_t launch_route(const void *logits, int type, int64_t stride, int64_t tokens, int experts, int top_k,
                        const uint8_t *keep, bool renormalize, float *weight, int32_t *expert, int32_t *count,
                        int32_t *offset, int32_t *slot, int32_t *place, void *ws, hipStream_t s)
{
    const bool alone = tokens <= kOneLaunch;
    const int group = alone ? kOneLaunch : group_tokens(tokens);
    const int64_t groups = alone ? 1 : ceil_div(tokens, group);
    int32_t *hist = static_cast<int32_t *>(ws);
    int bits = 1;
    while ((1 << bits) <= experts) ++bits;   // of the keys 0 .. experts
    const int rows_here = (int)(tokens < group ? tokens : group) * top_k;
    const size_t lds = (HAPMOE_MAX_EXPERTS + (size_t)rows_here) * 4;
    hipError_t e = by_type(type, [&](auto t) {
        using T = decltype(t);
        return by_experts(experts, [&](auto per) {
            constexpr int PER = decltype(per)::value;
            const bool vec = experts == 16 * PER && aligned(logits, 16) && stride * (int64_t)sizeof(T) % 16 == 0;
            auto *kernel = alone ? (vec ? k_choose<T, PER, true, true> : k_choose<T, PER, false, true>)
                                 : (vec ? k_choose<T, PER, true, false> : k_choose<T, PER, false, false>);
            hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(kThreads), lds, s, static_cast<const T *>(logits),
                               stride, tokens, experts, top_k, keep, renormalize ? 1 : 0, group, bits, weight, expert,
                               place, hist, count, offset, slot);
            return hipGetLastError();
        });
    });
    if (e != hipSuccess || alone) return e;
    hipLaunchKernelGGL(k_scan_groups, dim3((unsigned)ceil_div(experts, 64)), dim3(64 * kScanWaves), 0, s, hist,
                       (int)groups, experts, count);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const int64_t rows = tokens * top_k;
    hipLaunchKernelGGL(k_place, dim3((unsigned)ceil_div(rows, kPlaceRows)), dim3(kThreads), 0, s, expert, hist, count,
                       rows, experts, group * top_k, offset, place, slot);
    return hipGetLastError();
}

hipError_t launch_route_backward(const void *logits, int type, int64_t stride, int64_t tokens, int experts, int top_k,
                                 const uint8_t *keep, bool renormalize, const int32_t *expert, const float *weight,
                                 const float *d_weight, void *d_logits, hipStream_t s)
{
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        return by_experts(experts, [&](auto per) {
            constexpr int PER = decltype(per)::value;
            const bool vec = experts == 16 * PER && aligned(logits, 16) && aligned(d_logits, 16) &&
                             stride * (int64_t)sizeof(T) % 16 == 0;
            hipLaunchKernelGGL((vec ? k_route_backward<T, PER, true> : k_route_backward<T, PER, false>),
                               dim3((unsigned)ceil_div(tokens, kPass)), dim3(kThreads), 0, s,
                               static_cast<const T *>(logits), stride, tokens, experts, top_k, keep,
                               renormalize ? 1 : 0, expert, weight, d_weight, static_cast<T *>(d_logits));
            return hipGetLastError();
        });
    });
}

}  // namespace hapmoe
