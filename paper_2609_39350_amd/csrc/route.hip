// The router: of every token's logits the top_k largest, their softmax weights,
// and the order that puts each expert's rows together; and its gradient.
//
// Sixteen lanes take a token (four tokens a wave), its logits in their registers.
// A choice is the largest key over a row of lanes, four rotations without LDS,
// then the lowest index that has it; the softmax's maximum and sum come of the
// same.  From 129 experts on the keys are in LDS too and a choice looks again
// at the chosen lane's alone.
//
// The order is stable, so it needs every row's rank among the earlier rows of
// its expert.  A workgroup ranks its own tokens' rows: a wave takes 64 rows at a
// time, finds for each lane the lanes of the same expert by a ballot a bit of the
// expert's number, and keeps its counts so far in LDS.  A second kernel sums
// the workgroups' counts over the workgroups, a third adds the experts' offsets
// and writes both directions of the order.  Up to 64 tokens one workgroup does
// all of it in one launch, which is what a decoding step waits for.
//
// 32,768 tokens, 256 fp32 logits, top 8: choices 16.6 us (instruction issue; 7 of
// them would be the reading; 21.4 with all keys in registers), the groups' sums 4.7,
// the order 6.9, the gradient 12.4 (its 67 MB at 5.4 TB/s).  4 tokens of 64: 4.7 us.
#include "router.h"

namespace hapmoe {
namespace {

constexpr int kThreads = 256;
constexpr int kPass = kThreads / 16;   // tokens of a workgroup of the gradient
constexpr int kPlaceRows = 1024;       // rows of a workgroup of the last kernel

// Choices, weights and ranks.  ALONE: the only workgroup, which finishes the order too; else rank goes to `place` and
// the workgroup's counts to hist[workgroup][experts].
template <typename T, int PER, bool VEC, bool ALONE>
__global__ __launch_bounds__(choose_threads(PER)) void k_choose(
    const T *__restrict__ logits, int64_t stride, int64_t tokens, int experts, int top_k,
    const uint8_t *__restrict__ keep, int renormalize, int group, int bits, float *__restrict__ weight,
    int32_t *__restrict__ expert, int32_t *__restrict__ place, int32_t *__restrict__ hist, int32_t *__restrict__ count,
    int32_t *__restrict__ offset, int32_t *__restrict__ slot)
{
    constexpr int kChoose = choose_threads(PER), kWaves = kChoose / 64;
    constexpr bool kInLds = keys_in_lds(PER);
    extern __shared__ __attribute__((aligned(16))) int lds[];
    const int64_t first = workgroup() * group;
    if (first >= tokens && first > 0) return;
    const int here = tokens - first < group ? (int)(tokens - first) : group;
    int *const chosen = lds;                              // [here * top_k], whole vectors
    int *const sums = lds + ((here * top_k + 3) & ~3);    // [kWaves][experts]; before that the tokens' keys
    __shared__ int sh[kWaves];
    const int lane = threadIdx.x & 15;
    if constexpr (!kInLds)
        for (int e = threadIdx.x; e < kWaves * experts; e += kChoose) sums[e] = 0;
    for (int t0 = threadIdx.x >> 4; t0 < here; t0 += kChoose / 16) {
        const int64_t t = first + t0;
        float x[PER];
        int v[PER];
        load_logits<T, PER, VEC, true>(x, logits + t * stride, lane, experts, !keep || keep[t]);
#pragma unroll
        for (int c = 0; c < PER; ++c) v[c] = key_of(x[c]);
        int *const row = sums + (threadIdx.x >> 4) * key_row(PER);
        if constexpr (kInLds) {
            wave_order();   // the keys of the token before are read
#pragma unroll
            for (int c = 0; c < PER; c += 4)
                *reinterpret_cast<int4 *>(row + lane * PER + c) = make_int4(v[c], v[c + 1], v[c + 2], v[c + 3]);
            wave_order();
        }
        int own = lane_largest<int, PER>(v);   // the largest of the lane's keys that are left
        int m = row_reduce(own, Max());
        const float top = logit_of(m);
        float total = renormalize || m == kClosed ? 0.0f : softmax<PER>(x, top);
        int won[2] = {kClosed, kClosed};   // choices lane and lane + 16
        int who[2] = {-1, -1};
        for (int j = 0; j < top_k && m != kClosed; ++j) {
            int best;
            if constexpr (kInLds) {
                const int from = first_of_row(own == m);
                int k[PER / 16], at = 0;
#pragma unroll
                for (int q = 0; q < PER / 16; ++q) k[q] = row[from * PER + 16 * q + lane];
#pragma unroll
                for (int q = PER / 16 - 1; q >= 0; --q) {
                    const int l = first_of_row(k[q] == m);
                    at = l < 16 ? 16 * q + l : at;
                }
                best = from * PER + at;
#pragma unroll
                for (int q = 0; q < PER / 16; ++q) k[q] = at == 16 * q + lane ? kClosed : k[q];
                if (lane == 0) row[best] = kClosed;
                wave_order();
                const int left = row_reduce(lane_largest<int, PER / 16>(k), Max());
                own = lane == from ? left : own;
            } else {
                int at = PER;
#pragma unroll
                for (int c = PER - 1; c >= 0; --c) at = v[c] == m ? c : at;
                best = row_reduce(at < PER ? lane * PER + at : INT32_MAX, Min());
                const int mine = best - lane * PER;
#pragma unroll
                for (int c = 0; c < PER; ++c) v[c] = c == mine ? kClosed : v[c];
                own = lane_largest<int, PER>(v);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                won[h] = lane + 16 * h == j ? m : won[h];
                who[h] = lane + 16 * h == j ? best : who[h];
            }
            m = row_reduce(own, Max());
        }
        float share[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) share[h] = who[h] < 0 ? 0.0f : exp_from(logit_of(won[h]), top);
        if (renormalize) total = row_reduce(share[0] + share[1], Sum());
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = lane + 16 * h;
            if (j < top_k) {
                weight[t * top_k + j] = who[h] < 0 ? 0.0f : share[h] / total;
                expert[t * top_k + j] = who[h];
                chosen[t0 * top_k + j] = who[h];
            }
        }
    }
    if constexpr (kInLds) {
        __syncthreads();
        for (int e = threadIdx.x; e < kWaves * experts; e += kChoose) sums[e] = 0;
    }
    __syncthreads();
    order_rows<kChoose, ALONE>(chosen, sums, sh, here, top_k, first, experts, bits, place, hist, count, offset, slot);
}

// hist[group][experts] -> the sums over the groups before, and count.  A workgroup takes 16 experts, 16 lanes an equal
// run of the groups: its sum, the runs' sums before it, then the running sum.
constexpr int kScanThreads = 1024, kScanExperts = 16, kRuns = kScanThreads / kScanExperts;
__global__ __launch_bounds__(kScanThreads) void k_scan_groups(int32_t *__restrict__ hist, int groups, int experts,
                                                              int32_t *__restrict__ count)
{
    constexpr int kKept = 16;   // counts in registers: a run that is no longer is loaded once
    __shared__ int part[kScanThreads / 64][kScanExperts];
    const int mine = threadIdx.x % kScanExperts, run = threadIdx.x / kScanExperts;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int e = blockIdx.x * kScanExperts + mine;
    const int each = (groups + kRuns - 1) / kRuns;
    const int lo = min(run * each, groups), hi = e < experts ? min(lo + each, groups) : lo;
    int32_t *const own = hist + e;
    int kept[kKept], sum = 0;
    auto load = [&](int g0) {
#pragma unroll
        for (int i = 0; i < kKept; ++i) kept[i] = g0 + i < hi ? own[(int64_t)(g0 + i) * experts] : 0;
    };
    for (int g = lo; g < hi; g += kKept) {
        load(g);
#pragma unroll
        for (int i = 0; i < kKept; ++i) sum += kept[i];
    }
    int before = sum;
#pragma unroll
    for (int d = kScanExperts; d < 64; d <<= 1) {
        const int o = __shfl_up(before, d, 64);
        before += lane >= d ? o : 0;
    }
    if (lane >= 64 - kScanExperts) part[wave][mine] = before;
    __syncthreads();
    before -= sum;
#pragma unroll
    for (int w = 0; w < kScanThreads / 64; ++w) before += w < wave ? part[w][mine] : 0;
    if (e < experts && run == kRuns - 1) count[e] = before + sum;
    for (int g = lo; g < hi; g += kKept) {
        if (each > kKept) load(g);
#pragma unroll
        for (int i = 0; i < kKept; ++i) {
            if (g + i < hi) own[(int64_t)(g + i) * experts] = before;
            before += kept[i];
        }
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
// BALANCED: weights that were multiplied by a scale (the renormalised form's sum is of shares w_j / scale), and where the
// scores are sigmoids w_j (g_j - the same sum, if renormalised) (1 - s_j) at the chosen.
template <typename T, int PER, bool VEC, bool BALANCED>
__global__ __launch_bounds__(kThreads) void k_route_backward(
    const T *__restrict__ logits, int64_t stride, int64_t tokens, int experts, int top_k,
    const uint8_t *__restrict__ keep, int renormalize, const int32_t *__restrict__ expert,
    const float *__restrict__ weight, const float *__restrict__ d_weight, T *__restrict__ d_logits, int sigmoid, float scale)
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
        // a choice by itself has a share of 1, not of 1 but for a rounding: its gradient is 0
        const float share = BALANCED && renormalize ? w[h] / scale : w[h];
        gw[h] = g[h] * share;
    }
    float mean = row_reduce(gw[0] + gw[1], Sum());
    if (BALANCED && sigmoid && !renormalize) mean = 0.0f;
    float d[PER];
    if (renormalize || (BALANCED && sigmoid)) {
#pragma unroll
        for (int c = 0; c < PER; ++c) d[c] = 0.0f;
    } else {
        load_logits<T, PER, VEC, false>(d, logits + t * stride, lane, experts, !keep || keep[t]);
        const float top = row_reduce(lane_largest<float, PER>(d), Max());
        const float total = top == -INFINITY ? 1.0f : softmax<PER>(d, top), scale = -mean / total;
#pragma unroll
        for (int c = 0; c < PER; ++c) d[c] = top == -INFINITY ? 0.0f : d[c] * scale;
    }
    constexpr int kN = kStep<T, PER>;
    auto place_of = [](int e) { return e / kN % 16 * (PER + 1) + e / (16 * kN) * kN + e % kN; };
    // a token's choices are 16 lanes of one wave, and all different
    wave_order();
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (who[h] >= 0 && who[h] < 16 * PER) {
            float add = w[h] * (renormalize ? g[h] - mean : g[h]);
            if constexpr (BALANCED)
                if (sigmoid) add = who[h] < experts ? add * sigmoid_of(-to_f32(logits[t * stride + who[h]])) : 0.0f;
            row[place_of(who[h])] = add;
        }
    wave_order();
#pragma unroll
    for (int c = 0; c < PER; ++c) d[c] += mine[c];
    T *const out = d_logits + t * experts;
#pragma unroll
    for (int c = 0; c < PER; c += kN) {
        const int e = expert_at<kN, PER, false>(lane, c);
        if constexpr (VEC) {
            Piece<T, kN> p;
#pragma unroll
            for (int i = 0; i < kN; ++i) p.x[i] = from_f32<T>(d[c + i]);
            *reinterpret_cast<Piece<T, kN> *>(out + e) = p;
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i)
                if (e + i < experts) out[e + i] = from_f32<T>(d[c + i]);
        }
    }
}

}  // namespace

int64_t route_ws_bytes(int64_t tokens, int experts, int top_k)
{
    (void)top_k;
    if (tokens <= kOneLaunch) return 0;
    return ceil_div(tokens, group_tokens(tokens)) * experts * 4;
}

hipError_t launch_route_order(const int32_t *expert, int32_t *hist, int64_t groups, int64_t rows, int experts,
                              int group_rows, int32_t *count, int32_t *offset, int32_t *place, int32_t *slot,
                              hipStream_t s)
{
    hipLaunchKernelGGL(k_scan_groups, dim3((unsigned)ceil_div(experts, kScanExperts)), dim3(kScanThreads), 0, s, hist,
                       (int)groups, experts, count);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_place, many(ceil_div(rows, kPlaceRows)), dim3(kThreads), 0, s, expert, hist, count,
                       rows, experts, group_rows, offset, place, slot);
    return hipGetLastError();
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
    hipError_t e = by_type(type, [&](auto t) {
        using T = decltype(t);
        return by_experts(experts, [&](auto per) {
            constexpr int PER = decltype(per)::value;
            constexpr int kChoose = choose_threads(PER);
            const bool vec = experts == 16 * PER && aligned(logits, 16) && stride * (int64_t)sizeof(T) % 16 == 0;
            const int sums = (kChoose / 64 + (alone ? 1 : 0)) * experts, keys = kChoose / 16 * key_row(PER);
            const size_t lds = (((rows_here + 3) & ~3) + (keys_in_lds(PER) && keys > sums ? keys : sums)) * sizeof(int);
            auto *kernel = alone ? (vec ? k_choose<T, PER, true, true> : k_choose<T, PER, false, true>)
                                 : (vec ? k_choose<T, PER, true, false> : k_choose<T, PER, false, false>);
            hipLaunchKernelGGL(kernel, many(groups), dim3(kChoose), lds, s, static_cast<const T *>(logits),
                               stride, tokens, experts, top_k, keep, renormalize ? 1 : 0, group, bits, weight, expert,
                               place, hist, count, offset, slot);
            return hipGetLastError();
        });
    });
    if (e != hipSuccess || alone) return e;
    return launch_route_order(expert, hist, groups, tokens * top_k, experts, group * top_k, count, offset, place, slot, s);
}

namespace {
template <bool BALANCED>
hipError_t route_backward(const void *logits, int type, int64_t stride, int64_t tokens, int experts, int top_k,
                          const uint8_t *keep, bool renormalize, const int32_t *expert, const float *weight,
                          const float *d_weight, void *d_logits, bool sigmoid, float scale, hipStream_t s)
{
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        return by_experts(experts, [&](auto per) {
            constexpr int PER = decltype(per)::value;
            const bool vec = experts == 16 * PER && aligned(logits, 16) && aligned(d_logits, 16) &&
                             stride * (int64_t)sizeof(T) % 16 == 0;
            hipLaunchKernelGGL((vec ? k_route_backward<T, PER, true, BALANCED> : k_route_backward<T, PER, false, BALANCED>),
                               many(ceil_div(tokens, kPass)), dim3(kThreads), 0, s,
                               static_cast<const T *>(logits), stride, tokens, experts, top_k, keep,
                               renormalize ? 1 : 0, expert, weight, d_weight, static_cast<T *>(d_logits),
                               sigmoid ? 1 : 0, scale);
            return hipGetLastError();
        });
    });
}
}  // namespace

hipError_t launch_route_backward(const void *logits, int type, int64_t stride, int64_t tokens, int experts, int top_k,
                                 const uint8_t *keep, bool renormalize, const int32_t *expert, const float *weight,
                                 const float *d_weight, void *d_logits, hipStream_t s)
{
    return route_backward<false>(logits, type, stride, tokens, experts, top_k, keep, renormalize, expert, weight,
                                 d_weight, d_logits, false, 1.0f, s);
}

hipError_t launch_route_balanced_backward(const void *logits, int type, int64_t stride, int64_t tokens, int experts,
                                          int top_k, bool sigmoid, const uint8_t *keep, bool renormalize, float scale,
                                          const int32_t *expert, const float *weight, const float *d_weight,
                                          void *d_logits, hipStream_t s)
{
    return route_backward<true>(logits, type, stride, tokens, experts, top_k, keep, renormalize, expert, weight,
                                d_weight, d_logits, sigmoid, scale, s);
}

}  // namespace hapmoe
