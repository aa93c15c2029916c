// The router: of every token's logits the top_k largest, their softmax weights,
// and the order that puts each expert's rows together; and its gradient.
//
// Sixteen lanes take a token (four tokens a wave): lane l holds the logits
// l * PER .. l * PER + PER - 1 in registers, so a choice is two reductions over
// a row of lanes (the largest logit, then the lowest index that has it), each
// four rotations without LDS, and the softmax's maximum and sum come of the same.
//
// The order is stable, so it needs every row's rank among the earlier rows of
// its expert.  A workgroup ranks its own tokens' rows: a wave takes 64 rows at a
// time, finds for each lane the lanes of the same expert by a ballot a bit of the
// expert's number, and keeps its counts so far in LDS.  A second kernel sums
// the workgroups' counts over the workgroups, a third adds the experts' offsets
// and writes both directions of the order.  Up to 64 tokens one workgroup does
// all of it in one launch, which is what a decoding step waits for.
#include "operators.h"

namespace hapmoe {
namespace {

constexpr int kThreads = 256;
constexpr int kChoose = 512;           // threads of the first kernel
constexpr int kPass = kThreads / 16;   // tokens of a workgroup of the gradient
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

// exp(x - top), 1 where x is the largest: also where both are infinite.  2^t with t = x log2(e) in two parts, so that the
// error is that of the instruction (one unit) and not t's rounding; 0 below 2^-126.
__device__ inline float exp_from(float x, float top)
{
    const float d = fmaxf(x - top, -200.0f);
    const float t = d * 1.44269504f, rest = __builtin_fmaf(d, 1.44269504f, -t) + d * 1.92596303e-8f;
    const float y = __builtin_amdgcn_exp2f(t);
    return x == top ? 1.0f : __builtin_fmaf(y, rest * 0.693147181f, y);
}

// Logits as whole numbers of the same order (both zeros equal), kClosed below all of them: the maxima need no care for
// NaN, and the lane rotations go into them.
constexpr int kClosed = INT32_MIN;
__device__ inline int key_of(float x)
{
    const int b = __builtin_bit_cast(int, x + 0.0f);
    return x == -INFINITY ? kClosed : b ^ (b >> 31 & 0x7fffffff);
}
__device__ inline float logit_of(int key) { return __builtin_bit_cast(float, key ^ (key >> 31 & 0x7fffffff)); }

template <int PER>
__device__ inline float softmax_sum(const float *v, float top)
{
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < PER; ++c) s += v[c] == -INFINITY ? 0.0f : exp_from(v[c], top);
    return row_reduce(s, Sum());
}

template <typename V, int PER>
__device__ inline V largest(const V *v)
{
    V m = v[0];
#pragma unroll
    for (int c = 1; c < PER; ++c) m = Max()(m, v[c]);
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
template <int THREADS>
__device__ inline int scan_counts(int *count, int experts, int *sh)
{
    constexpr int kPer = HAPMOE_MAX_EXPERTS / THREADS;
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
    for (int w = 0; w < THREADS / 64; ++w) {
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
__global__ __launch_bounds__(kChoose) void k_choose(const T *__restrict__ logits, int64_t stride, int64_t tokens,
                                                     int experts, int top_k, const uint8_t *__restrict__ keep,
                                                     int renormalize, int group, int bits, float *__restrict__ weight,
                                                     int32_t *__restrict__ expert, int32_t *__restrict__ place,
                                                     int32_t *__restrict__ hist, int32_t *__restrict__ count,
                                                     int32_t *__restrict__ offset, int32_t *__restrict__ slot)
{
    constexpr int kWaves = kChoose / 64;
    extern __shared__ int lds[];
    int *sums = lds;                         // [kWaves][experts]
    int *chosen = lds + kWaves * experts;    // [group * top_k]
    __shared__ int sh[kWaves];
    const int lane = threadIdx.x & 15;
    const int64_t first = workgroup() * group;
    if (first >= tokens && first > 0) return;
    const int here = tokens - first < group ? (int)(tokens - first) : group;
    for (int e = threadIdx.x; e < kWaves * experts; e += kChoose) sums[e] = 0;
    for (int t0 = threadIdx.x >> 4; t0 < here; t0 += kChoose / 16) {
        const int64_t t = first + t0;
        float x[PER];
        int v[PER];
        load_logits<T, PER, VEC>(x, logits + t * stride, lane, experts, !keep || keep[t]);
#pragma unroll
        for (int c = 0; c < PER; ++c) v[c] = key_of(x[c]);
        int m = largest<int, PER>(v);
        const float top = logit_of(m);
        float total = renormalize || m == kClosed ? 0.0f : softmax_sum<PER>(x, top);
        int won[2] = {kClosed, kClosed};   // choices lane and lane + 16
        int who[2] = {-1, -1};
        for (int j = 0; j < top_k && m != kClosed; ++j) {
            int at = PER;
#pragma unroll
            for (int c = PER - 1; c >= 0; --c) at = v[c] == m ? c : at;
            const int best = row_reduce(at < PER ? lane * PER + at : INT32_MAX, Min());
            const int mine = best - lane * PER;
#pragma unroll
            for (int c = 0; c < PER; ++c) v[c] = c == mine ? kClosed : v[c];
            if (renormalize) total += exp_from(logit_of(m), top);
            if (lane == (j & 15)) {
                won[0] = j < 16 ? m : won[0];
                who[0] = j < 16 ? best : who[0];
                won[1] = j < 16 ? won[1] : m;
                who[1] = j < 16 ? who[1] : best;
            }
            m = largest<int, PER>(v);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = lane + 16 * h;
            if (j < top_k) {
                weight[t * top_k + j] = who[h] < 0 ? 0.0f : exp_from(logit_of(won[h]), top) / total;
                expert[t * top_k + j] = who[h];
                chosen[t0 * top_k + j] = who[h];
            }
        }
    }
    __syncthreads();
    // each wave ranks a run of the rows among its own
    const int rows = here * top_k, run = (rows + kChoose - 1) / kChoose * 64;
    const int wave = threadIdx.x >> 6, wave_lane = threadIdx.x & 63;
    const int lo = min(wave * run, rows), hi = min(lo + run, rows);
    int *const own = sums + wave * experts;
    int32_t *const mine = place + first * top_k;
    for (int r0 = lo; r0 < hi; r0 += 64) {
        const int r = r0 + wave_lane;
        const int e = r < hi ? chosen[r] : -1;
        const uint64_t same = same_key(e + 1, bits);
        const uint64_t below = same & ((1ull << wave_lane) - 1);
        if (e >= 0) chosen[r] = (own[e] + __popcll(below)) << 10 | e;   // rank < 2^11, e < 2^10
        // the counts before this round are read by every lane before the lowest of each expert adds to them
        __builtin_amdgcn_wave_barrier();
        if (e >= 0 && below == 0) own[e] += __popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // the counts of the waves before, and the whole
    for (int e = threadIdx.x; e < experts; e += kChoose) {
        int before = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const int n = sums[w * experts + e];
            sums[w * experts + e] = before;
            before += n;
        }
        if constexpr (ALONE)
            count[e] = before;
        else
            hist[workgroup() * experts + e] = before;
    }
    __syncthreads();
    if constexpr (ALONE) {
        // experts' offsets into the last wave's place, then the others' by them
        int *const at = chosen + rows;
        for (int e = threadIdx.x; e < experts; e += kChoose) at[e] = count[e];
        __syncthreads();
        const int total = scan_counts<kChoose>(at, experts, sh);
        for (int e = threadIdx.x; e < experts; e += kChoose) offset[e] = at[e];
        if (threadIdx.x == 0) offset[experts] = total;
        for (int r = threadIdx.x; r < rows; r += kChoose) {
            const int c = chosen[r], e = c & 1023;
            const int p = c < 0 ? -1 : at[e] + sums[r / run * experts + e] + (c >> 10);
            place[r] = p;
            if (p >= 0) slot[p] = r;
            if (r >= total) slot[r] = -1;
        }
    } else {
        for (int r = threadIdx.x; r < rows; r += kChoose) {
            const int c = chosen[r];
            mine[r] = c < 0 ? -1 : sums[r / run * experts + (c & 1023)] + (c >> 10);
        }
    }
}

// hist[group][experts] -> the sums over the groups before, and count.  A workgroup takes 16 experts, 16 lanes an equal
// run of the groups: its sum, the runs' sums before it, then the running sum.
constexpr int kScanThreads = 1024, kRuns = kScanThreads / 16;
__global__ __launch_bounds__(kScanThreads) void k_scan_groups(int32_t *__restrict__ hist, int groups, int experts,
                                                              int32_t *__restrict__ count)
{
    __shared__ int part[kRuns][16];
    const int lane = threadIdx.x & 15, run = threadIdx.x >> 4;
    const int e = blockIdx.x * 16 + lane;
    const int each = (groups + kRuns - 1) / kRuns;
    const int lo = min(run * each, groups), hi = min(lo + each, groups);
    int sum = 0;
    if (e < experts) {
#pragma unroll 8
        for (int g = lo; g < hi; ++g) sum += hist[(int64_t)g * experts + e];
    }
    part[run][lane] = sum;
    __syncthreads();
#pragma unroll
    for (int d = 1; d < kRuns; d <<= 1) {
        const int o = run >= d ? part[run - d][lane] : 0;
        __syncthreads();
        part[run][lane] += o;
        __syncthreads();
    }
    if (e >= experts) return;
    int before = part[run][lane] - sum;
    if (run == kRuns - 1) count[e] = before + sum;
#pragma unroll 8
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
    const int total = scan_counts<kThreads>(at, experts, sh);
    if (workgroup() == 0) {
        for (int e = threadIdx.x; e < experts; e += kThreads) offset[e] = at[e];
        if (threadIdx.x == 0) offset[experts] = total;
    }
    const int64_t r0 = workgroup() * kPlaceRows;
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
    // what the chosen add, [token][16 lanes' PER + 1]: a lane's are a row of their own, a row's banks shifted by one
    __shared__ float added[kPass * 16 * (PER + 1)];
    const int lane = threadIdx.x & 15;
    const int64_t t = workgroup() * kPass + (threadIdx.x >> 4);
    if (t >= tokens) return;
    float *const mine = added + threadIdx.x * (PER + 1), *const row = added + (threadIdx.x & ~15u) * (PER + 1);
#pragma unroll
    for (int c = 0; c < PER; ++c) mine[c] = 0.0f;
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
        const float top = largest<float, PER>(d);
        const float total = top == -INFINITY ? 1.0f : softmax_sum<PER>(d, top);
#pragma unroll
        for (int c = 0; c < PER; ++c) d[c] = d[c] == -INFINITY ? 0.0f : exp_from(d[c], top) / total * -mean;
    }
    // a token's choices are 16 lanes of one wave, and all different
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (who[h] >= 0 && who[h] < 16 * PER) row[who[h] / PER * (PER + 1) + who[h] % PER] = w[h] * (renormalize ? g[h] - mean : g[h]);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int c = 0; c < PER; ++c) d[c] += mine[c];
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
    const size_t lds = ((kChoose / 64 + (alone ? 1 : 0)) * (size_t)experts + rows_here) * 4;
    hipError_t e = by_type(type, [&](auto t) {
        using T = decltype(t);
        return by_experts(experts, [&](auto per) {
            constexpr int PER = decltype(per)::value;
            const bool vec = experts == 16 * PER && aligned(logits, 16) && stride * (int64_t)sizeof(T) % 16 == 0;
            auto *kernel = alone ? (vec ? k_choose<T, PER, true, true> : k_choose<T, PER, false, true>)
                                 : (vec ? k_choose<T, PER, true, false> : k_choose<T, PER, false, false>);
            hipLaunchKernelGGL(kernel, many(groups), dim3(kChoose), lds, s, static_cast<const T *>(logits),
                               stride, tokens, experts, top_k, keep, renormalize ? 1 : 0, group, bits, weight, expert,
                               place, hist, count, offset, slot);
            return hipGetLastError();
        });
    });
    if (e != hipSuccess || alone) return e;
    hipLaunchKernelGGL(k_scan_groups, dim3((unsigned)ceil_div(experts, 16)), dim3(kScanThreads), 0, s, hist,
                       (int)groups, experts, count);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const int64_t rows = tokens * top_k;
    hipLaunchKernelGGL(k_place, many(ceil_div(rows, kPlaceRows)), dim3(kThreads), 0, s, expert, hist, count,
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
                               many(ceil_div(tokens, kPass)), dim3(kThreads), 0, s,
                               static_cast<const T *>(logits), stride, tokens, experts, top_k, keep,
                               renormalize ? 1 : 0, expert, weight, d_weight, static_cast<T *>(d_logits));
            return hipGetLastError();
        });
    });
}

}  // namespace hapmoe
