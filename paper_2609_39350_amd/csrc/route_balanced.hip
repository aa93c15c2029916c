// The router with a balanced choice: scores s = sigmoid(x) or softmax(x), a bias that enters the choice alone, the
// best groups of experts, the best experts of those; weights from the scores without the bias.
//
// The choice is that of the exact scores: with a bias no order of the logits tells it, and two sums s + bias can be
// nearer to each other than fp32 resolves.  So they are computed in 64 bits.
#include "router.h"

namespace hapmoe {
namespace {

constexpr int kChooseThreads = 512;

__device__ inline double wave_max(double v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v = fmax(v, __shfl_xor(v, d, 64));
    return v;
}
__device__ inline double wave_sum(double v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    return v;
}
__device__ inline float wave_max(float v) { return wave_reduce(v, Max()); }

struct Choice {
    float x;     // the logit
    int expert;  // -1: none
};

// One token by a wave, its choice j in lane j; lane's experts are lane * N .. lane * N + N.  total: of exp(x - top).
template <typename T, int N>
__device__ inline Choice choose_exactly(const T *__restrict__ row, const float *__restrict__ bias, int experts,
                                        int top_k, bool sigmoid, int groups, int top_groups, int group_best, bool keep,
                                        float &top, float &total)
{
    const int lane = threadIdx.x & 63;
    float x[N];
    double c[N];
    top = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = lane * N + i;
        x[i] = keep && e < experts ? to_f32(row[e]) : -INFINITY;
        x[i] = x[i] > -INFINITY ? x[i] : -INFINITY;
        top = fmaxf(top, x[i]);
    }
    top = wave_max(top);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (sigmoid)
            c[i] = 1.0 / (1.0 + exp(-(double)x[i]));
        else
            sum += c[i] = x[i] == top ? 1.0 : exp((double)x[i] - (double)top);   // top closed: not read below
    }
    if (!sigmoid) {
        sum = wave_sum(sum);
        total = (float)sum;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (!sigmoid) c[i] /= sum;
        const int e = lane * N + i;
        if (bias && e < experts) c[i] += (double)bias[e];
        // closed to the choice: closed by its logit, or by a bias of -inf or NaN
        c[i] = x[i] > -INFINITY && c[i] > -INFINITY ? c[i] : -INFINITY;
    }
    if (top_groups < groups) {
        const int each = experts / groups;
        double mine = -INFINITY;   // of group `lane`
        for (int g = 0; g < groups; ++g) {
            double first = -INFINITY;
            int at = -1;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int e = lane * N + i;
                if (e >= g * each && e < g * each + each && c[i] > first) first = c[i], at = i;
            }
            const double best = wave_max(first);
            double score = best;
            if (group_best > 1) {
                const uint64_t who = __ballot(first == best && at >= 0);
                const bool out = who != 0 && lane == __ffsll((unsigned long long)who) - 1;
                double next = -INFINITY;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int e = lane * N + i;
                    if (e >= g * each && e < g * each + each && !(out && i == at)) next = fmax(next, c[i]);
                }
                next = wave_max(next);
                if (next > -INFINITY) score += next;
            }
            if (lane == g) mine = score;
        }
        int before = 0;   // groups that go before this lane's
        for (int g = 0; g < groups; ++g) {
            const double other = __shfl(mine, g, 64);
            before += other > mine || (other == mine && g < lane);
        }
        const uint64_t taken = __ballot(lane < groups && before < top_groups);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = lane * N + i;
            if (e >= experts || !(taken >> (e / each) & 1)) c[i] = -INFINITY;
        }
    }
    if (!bias) {   // the scores' order is that of the logits
#pragma unroll
        for (int i = 0; i < N; ++i) c[i] = c[i] > -INFINITY ? (double)x[i] : -INFINITY;
    }
    Choice won = {-INFINITY, -1};
    for (int j = 0; j < top_k; ++j) {
        double own = c[0];
        float own_x = x[0];
        int at = 0;
#pragma unroll
        for (int i = 1; i < N; ++i) {
            const bool more = c[i] > own;
            own = more ? c[i] : own;
            own_x = more ? x[i] : own_x;
            at = more ? i : at;
        }
        const double best = wave_max(own);
        if (best == -INFINITY) break;
        const int from = __ffsll((unsigned long long)__ballot(own == best)) - 1;
        const int which = __shfl(at, from, 64);
        const float value = __shfl(own_x, from, 64);
        if (lane == j) won = {value, from * N + which};
        if (lane == from) {
#pragma unroll
            for (int i = 0; i < N; ++i) c[i] = i == which ? -INFINITY : c[i];
        }
    }
    return won;
}

template <typename T, int N, bool ALONE>
__global__ __launch_bounds__(kChooseThreads) void k_choose_balanced(
    const T *__restrict__ logits, int64_t stride, int64_t tokens, int experts, int top_k,
    const float *__restrict__ bias, int sigmoid, int groups, int top_groups, int group_best,
    const uint8_t *__restrict__ keep, int renormalize, float scale, int group, int bits, float *__restrict__ weight,
    int32_t *__restrict__ expert, int32_t *__restrict__ place, int32_t *__restrict__ hist, int32_t *__restrict__ count,
    int32_t *__restrict__ offset, int32_t *__restrict__ slot)
{
    constexpr int kWaves = kChooseThreads / 64;
    extern __shared__ __attribute__((aligned(16))) int lds[];
    const int64_t first = workgroup() * group;
    if (first >= tokens && first > 0) return;
    const int here = tokens - first < group ? (int)(tokens - first) : group;
    int *const chosen = lds;
    int *const sums = lds + ((here * top_k + 3) & ~3);
    __shared__ int sh[kWaves];
    const int lane = threadIdx.x & 63;
    for (int e = threadIdx.x; e < kWaves * experts; e += kChooseThreads) sums[e] = 0;
    for (int t0 = threadIdx.x >> 6; t0 < here; t0 += kWaves) {
        const int64_t t = first + t0;
        float top, total = 1.0f;
        const Choice c = choose_exactly<T, N>(logits + t * stride, bias, experts, top_k, sigmoid, groups, top_groups,
                                              group_best, !keep || keep[t], top, total);
        const bool has = c.expert >= 0;
        float share;
        if (!renormalize) {
            share = !has ? 0.0f : sigmoid ? sigmoid_of(c.x) : exp_from(c.x, top) / total;
        } else {
            // the scores over that of the largest logit chosen, a factor that they share left out: none underflows to 0 / 0
            const float most = wave_max(c.x);
            if (sigmoid) {
                share = exp_from(fminf(c.x, 0.0f), fminf(most, 0.0f)) / (1.0f + exp_from(-fabsf(c.x), 0.0f));
            } else {
                share = exp_from(c.x, most);
            }
            share = has ? share : 0.0f;
            const float sum = wave_reduce(share, Sum());
            share = has ? share / sum : 0.0f;
        }
        if (lane < top_k) {
            weight[t * top_k + lane] = share * scale;
            expert[t * top_k + lane] = c.expert;
            chosen[t0 * top_k + lane] = c.expert;
        }
    }
    __syncthreads();
    order_rows<kChooseThreads, ALONE>(chosen, sums, sh, here, top_k, first, experts, bits, place, hist, count, offset,
                                      slot);
}

}  // namespace

hipError_t launch_route_balanced(const BalancedRoute &a, hipStream_t s)
{
    const bool alone = a.tokens <= kOneLaunch;
    const int group = alone ? kOneLaunch : group_tokens(a.tokens);
    const int64_t workgroups = alone ? 1 : ceil_div(a.tokens, group);
    int bits = 1;
    while ((1 << bits) <= a.experts) ++bits;   // of the keys 0 .. experts
    const int rows_here = (int)(a.tokens < group ? a.tokens : group) * a.top_k;
    const size_t lds = (((rows_here + 3) & ~3) + (kChooseThreads / 64 + (alone ? 1 : 0)) * a.experts) * sizeof(int);
    int32_t *hist = static_cast<int32_t *>(a.ws);
    const hipError_t e = by_type(a.type, [&](auto t) {
        using T = decltype(t);
        return by_experts(a.experts, [&](auto per) {
            constexpr int N = decltype(per)::value / 4;
            hipLaunchKernelGGL((alone ? k_choose_balanced<T, N, true> : k_choose_balanced<T, N, false>),
                               many(workgroups), dim3(kChooseThreads), lds, s, static_cast<const T *>(a.logits),
                               a.stride, a.tokens, a.experts, a.top_k, a.bias, a.sigmoid ? 1 : 0, a.groups, a.top_groups,
                               a.group_best, a.keep, a.renormalize ? 1 : 0, a.scale, group, bits, a.weight, a.expert,
                               a.place, hist, a.count, a.offset, a.slot);
            return hipGetLastError();
        });
    });
    if (e != hipSuccess || alone) return e;
    return launch_route_order(a.expert, hist, workgroups, a.tokens * a.top_k, a.experts, group * a.top_k, a.count,
                              a.offset, a.place, a.slot, s);
}

}  // namespace hapmoe
