// What the two routers share: a token's logits in the lanes that take it, the exponential, and the stable order of the
// rows by expert.
#pragma once

#include <type_traits>

#include "operators.h"

namespace hapmoe {

// Launches of the order after k_choose: hist [groups][experts] of group_rows rows each, expert and place [rows].
hipError_t launch_route_order(const int32_t *expert, int32_t *hist, int64_t groups, int64_t rows, int experts,
                              int group_rows, int32_t *count, int32_t *offset, int32_t *place, int32_t *slot,
                              hipStream_t s);

#ifdef __HIPCC__
namespace {

// Up to this many tokens one launch: us by one, by three: 8 experts, top 2: 64 tokens 6.0, 9.3, 128 7.9, 9.3; 256 experts, top
// 8: 64 tokens 9.6, 12.4, 128 15.3, 14.0, 256 26.7, 14.2.  The balanced router, whose workgroup has no more than 64: 64
// experts, 8 of them: 32 tokens 7.4, 11.9, 64 10.0, 12.7; 256 experts, 8 of 4 of 8 groups: 9.7, 14.4, 14.4, 15.0; of 1,024
// experts, 4 of them, three launches would be the better from 48 on: 33.9, 38.0, 48 tokens 46.9, 38.0, 64 59.9, 38.7.
constexpr int kOneLaunch = 64;

// Tokens of a workgroup.  us by 32, by 64: 256 experts, top 8: 16,384 tokens 18.7, 19.6, 32,768 25.9, 24.5, 65,536 38.6, 34.0;
// 8 experts 13.8, 13.9, 15.7, 15.3, 21.7, 18.4; 1,024 experts, top 4, 32,768 tokens 49, 58: for those 32,768 are by 32 too.
// The balanced router's choices and order: 64 experts, 8 of them, 4,096 tokens 17.9, 20.3, 16,384 20.5, 20.6, 32,768 27.3,
// 25.2, 65,536 43.2, 36.2; 256 experts, 8 of 4 of 8 groups, 18.5, 22.8, 24.2, 25.7, 39.4, 36.6, 61.1, 53.4; 1,024, 4 of
// them, 45.4, 71.6, 56.1, 78.8, 69.3, 92.6, 138.7, 114.9.
__host__ __device__ inline int group_tokens(int64_t tokens) { return tokens <= 64 * 512 ? 32 : 64; }

// Neighbouring elements of a lane: those that it loads and stores at once where vectors are aligned; where they are not
// it has the same, so that sums have the same order.
template <typename T, int PER>
constexpr int kStep = 16 / (int)sizeof(T) < PER ? 16 / (int)sizeof(T) : PER;
template <typename T, int N>
struct alignas(N * sizeof(T)) Piece {
    T x[N];
};
// The expert whose logit is a lane's c-th: lanes take turns at steps of a row, so that loads and stores are whole lines, or
// each has a RUN of PER, for the lowest of equal logits.
template <int STEP, int PER, bool RUN>
__device__ inline int expert_at(int lane, int c)
{
    return RUN ? lane * PER + c : (c / STEP * 16 + lane) * STEP + c % STEP;
}

// A token's logits in the registers of 16 lanes; closed experts (-inf, NaN, past the end, keep = 0) are -inf.
template <typename T, int PER, bool VEC, bool RUN>
__device__ inline void load_logits(float *v, const T *__restrict__ row, int lane, int experts, bool keep)
{
    constexpr int kN = kStep<T, PER>;
#pragma unroll
    for (int c = 0; c < PER; c += kN) {
        const int e = expert_at<kN, PER, RUN>(lane, c);
        if constexpr (VEC) {
            const auto p = *reinterpret_cast<const Piece<T, kN> *>(row + e);
#pragma unroll
            for (int i = 0; i < kN; ++i) v[c + i] = to_f32(p.x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i) v[c + i] = e + i < experts ? to_f32(row[e + i]) : -INFINITY;
        }
    }
#pragma unroll
    for (int c = 0; c < PER; ++c) v[c] = keep && v[c] > -INFINITY ? v[c] : -INFINITY;
}

// threads of the first kernel: 32 KB of keys where they are in LDS, so that four workgroups share a CU
constexpr int choose_threads(int per) { return per <= 16 ? 512 : 8192 / per; }
// Where a lane's keys are in LDS too.  Taking a choice out of registers costs every lane a look at all of its PER keys,
// three times; out of LDS the 16 lanes look at the chosen lane's keys together, once.
constexpr bool keys_in_lds(int per) { return per >= 16; }
constexpr int key_row(int per) { return 16 * per + 16; }   // a token's keys, the tokens' banks shifted

// exp(x - top), 1 where x is the largest: also where both are infinite.  2^t with t = x log2(e) in two parts, so that the
// error is that of the instruction (one unit) and not t's rounding; 0 below 2^-126.
__device__ inline float exp_from(float x, float top)
{
    const float d = fmaxf(x - top, -200.0f);
    const float t = d * 1.44269504f, rest = __builtin_fmaf(d, 1.92596303e-8f, __builtin_fmaf(d, 1.44269504f, -t));
    const float y = __builtin_amdgcn_exp2f(t);
    return x == top ? 1.0f : __builtin_fmaf(y, rest * 0.693147181f, y);
}

// 1 / (1 + exp(-x)), and of -x what is left of 1, each to its own precision
__device__ inline float sigmoid_of(float x)
{
    const float e = exp_from(-fabsf(x), 0.0f);
    return (x >= 0.0f ? 1.0f : e) / (1.0f + e);
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

// v to exp(v - top), 0 where closed (top is not), and their sum
template <int PER>
__device__ inline float softmax(float *v, float top)
{
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < PER; ++c) s += v[c] = exp_from(v[c], top);
    return row_reduce(s, Sum());
}

template <typename V, int PER>
__device__ inline V lane_largest(const V *v)
{
    V m = v[0];
#pragma unroll
    for (int c = 1; c < PER; ++c) m = Max()(m, v[c]);
    return m;
}

// The lowest lane of this lane's row of 16 where yes; 31 if none.
__device__ inline int first_of_row(bool yes)
{
    return __ffs((int)((uint32_t)(__ballot(yes) >> (threadIdx.x & 48)) & 0xffff) | INT32_MIN) - 1;
}

// LDS written by lanes of a wave and read by others of it: its accesses are done in order, the compiler has to keep it.
__device__ inline void wave_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
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

// The order of a workgroup's rows by its `here` tokens' choices, chosen[here * top_k].  sums: [waves][experts] zeros, and
// if ALONE experts more.  ALONE: the only workgroup, which finishes the order too; else ranks go to `place` and the
// workgroup's counts to hist[workgroup][experts].
template <int THREADS, bool ALONE>
__device__ inline void order_rows(int *chosen, int *sums, int *sh, int here, int top_k, int64_t first, int experts,
                                  int bits, int32_t *__restrict__ place, int32_t *__restrict__ hist,
                                  int32_t *__restrict__ count, int32_t *__restrict__ offset, int32_t *__restrict__ slot)
{
    constexpr int kWaves = THREADS / 64;
    // each wave ranks a run of the rows among its own
    const int rows = here * top_k, run = (rows + THREADS - 1) / THREADS * 64;
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
        wave_order();
        if (e >= 0 && below == 0) own[e] += __popcll(same);
        wave_order();
    }
    __syncthreads();
    // the counts of the waves before, and the whole
    for (int e = threadIdx.x; e < experts; e += THREADS) {
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
        int *const at = sums + kWaves * experts;
        for (int e = threadIdx.x; e < experts; e += THREADS) at[e] = count[e];
        __syncthreads();
        const int total = scan_counts<THREADS>(at, experts, sh);
        for (int e = threadIdx.x; e < experts; e += THREADS) offset[e] = at[e];
        if (threadIdx.x == 0) offset[experts] = total;
        for (int r = threadIdx.x; r < rows; r += THREADS) {
            const int c = chosen[r], e = c & 1023;
            const int p = c < 0 ? -1 : at[e] + sums[r / run * experts + e] + (c >> 10);
            place[r] = p;
            if (p >= 0) slot[p] = r;
            if (r >= total) slot[r] = -1;
        }
    } else {
        for (int r = threadIdx.x; r < rows; r += THREADS) {
            const int c = chosen[r];
            mine[r] = c < 0 ? -1 : sums[r / run * experts + (c & 1023)] + (c >> 10);
        }
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
#endif

}  // namespace hapmoe
