// The router with a balanced choice: scores s = sigmoid(x) or softmax(x), a bias that enters the choice alone, the
// best groups of experts, the best experts of those; weights from the scores without the bias.
//
// The choice is that of the exact scores: with a bias no order of the logits tells it, and two sums s + bias can be
// nearer to each other than fp32 resolves.  So a token is chosen for in fp32 first, by 16 lanes as in route.hip, and each
// pair of neighbours in the order that decides something is looked at: the chosen experts, the first that is not, the last
// group that stays and the first that does not.  Where a pair is nearer than the error of the two, its scores are computed
// again in 64 bits: those of the choices by the same lanes, or, where more than their order may change, all of the token's
// by a wave.  Of equal inputs only a choice and its neighbour are told from near ones: groups of the same logits and
// biases, and three that are equal over the last choice, take the wave too.
//
// Bound by instruction issue (1,340 a wave for four tokens, 79 % of the time) and, in the last workgroup to end, by what is
// computed again.  32,768 tokens, 256 fp32 logits, 8 of 4 of 8 groups by sigmoid and a random bias: choices 28.3 us (153
// with all in 64 bits), the order 11.3 as in route.hip, the gradient 9.4 (it reads logits at the chosen alone).  4 such
// tokens in one launch 8.0 us, five more where one is computed again by a wave.  The choices with a bias of zeros: fp32
// 30.0, bf16, which has equal logits, 35.1 (26.7 with a random bias); where a tenth of the rows are zeros 41.1 and 40.3,
// where all are 104.
#include "router.h"

namespace hapmoe {
namespace {

// One token by a wave in 64 bits, expert i * 64 + lane in a lane's i-th place: its choices to chosen[top_k].  c: [experts]
// and [64] of the wave's LDS.  Of a softmax the largest logit and the sum of exp(x - top) too.
template <typename T, int N>
__device__ inline void choose_exactly(const BalancedRoute &q, const T *__restrict__ row, bool keep, double *c, int *chosen,
                                      float &top, float &total)
{
    const int lane = threadIdx.x & 63, experts = q.experts, each = experts / q.groups;
    float x[N];
    double v[N], sum = 0.0;
    top = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = to_f32(row[min(i * 64 + lane, experts - 1)]);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = keep && i * 64 + lane < experts && x[i] > -INFINITY ? x[i] : -INFINITY;
        top = fmaxf(top, x[i]);
    }
    if (!q.sigmoid) top = wave_value(top, Max());
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = exp(q.sigmoid ? -(double)x[i] : x[i] == top ? 0.0 : (double)x[i] - (double)top);
        if (i * 64 + lane < experts) sum += v[i];
    }
    if (!q.sigmoid) sum = wave_value(sum, Sum());
    total = (float)sum;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = (q.sigmoid ? 1.0 : v[i]) / (q.sigmoid ? 1.0 + v[i] : sum);
        if (q.bias) v[i] += (double)q.bias[min(i * 64 + lane, experts - 1)];
        // closed to the choice: closed by its logit, or by a bias of -inf or NaN
        v[i] = x[i] > -INFINITY && v[i] > -INFINITY ? v[i] : -INFINITY;
    }
    if (q.top_groups < q.groups) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i * 64 + lane < experts) c[i * 64 + lane] = v[i];
        wave_order();
        double first = -INFINITY, next = -INFINITY;   // of group `lane`
        if (lane < q.groups)
#pragma unroll 4
            for (int i = 0; i < each; ++i) {
                const double s = c[lane * each + i];
                next = fmax(next, fmin(first, s));
                first = fmax(first, s);
            }
        if (q.group_best > 1 && next > -INFINITY) first += next;
        wave_order();
        c[lane] = first;   // the groups' scores in the experts' place, which is at least that long
        wave_order();
        int before = 0;   // groups that go before this lane's
#pragma unroll 4
        for (int g = 0; g < q.groups; ++g) before += c[g] > first || (c[g] == first && g < lane);
        const uint64_t taken = __ballot(lane < q.groups && before < q.top_groups);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i * 64 + lane >= experts || !(taken >> ((i * 64 + lane) / each) & 1)) v[i] = -INFINITY;
    }
    if (!q.bias) {   // the scores' order is that of the logits
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] > -INFINITY ? (double)x[i] : -INFINITY;
    }
    for (int j = 0; j < q.top_k; ++j) {
        double own = v[0];
        int at = lane;
#pragma unroll
        for (int i = 1; i < N; ++i) {
            at = v[i] > own ? i * 64 + lane : at;
            own = fmax(own, v[i]);
        }
        const double best = wave_value(own, Max());
        const int won = best > -INFINITY ? wave_value(own == best ? at : INT32_MAX, Min()) : -1;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = won == i * 64 + lane ? -INFINITY : v[i];
        if (lane == 0) chosen[j] = won;
    }
}

// Lanes of a group where its experts are those of 1, 2, 4, 8 or 16 whole lanes; 0: any others.
__host__ __device__ inline int lanes_a_group(int each, int per)
{
    const int m = each / per;
    return each % per == 0 && (m & (m - 1)) == 0 ? m : 0;
}

struct Top2 {
    int a, b;   // keys, the largest and the next
    __device__ void take(int k)
    {
        b = Max()(b, Min()(a, k));
        a = Max()(a, k);
    }
    __device__ void join(int oa, int ob)
    {
        b = Max()(Min()(a, oa), Max()(b, ob));
        a = Max()(a, oa);
    }
    // The other lanes of a group of m = 1, 2, 4 or 8, neighbours in a row of 16 (of 16 there is one group, not looked at).
    __device__ void over_lanes(int m)
    {
        if (m >= 2) join(dpp<0xb1>(a), dpp<0xb1>(b));     // lanes 1 0 3 2
        if (m >= 4) join(dpp<0x4e>(a), dpp<0x4e>(b));     // lanes 2 3 0 1
        if (m >= 8) join(dpp<0x141>(a), dpp<0x141>(b));   // 8 lanes mirrored: the other four's
    }
    // The group's score, and what three roundings add to its error: of each summand, their sum and its bound, 2^-24 of the
    // size each.  It is the group's own, so that one far off does not bring the others near.  A group with an open expert
    // is open: a sum past fp32's ends is the end, not an infinity; its bound beyond is one, as 2^-23 of the end is more
    // than half a step there.
    __device__ int score(int group_best, float &rounding) const
    {
        constexpr float kThree = 3.0f / (1 << 24);
        rounding = 0.0f;
        if (a == kClosed) return kClosed;
        const float x = logit_of(a), y = group_best > 1 && b != kClosed ? logit_of(b) : 0.0f;
        rounding = __builtin_fmaf(kThree, fabsf(x), kThree * fabsf(y));
        return key_of(fminf(fmaxf(x + y, -__FLT_MAX__), __FLT_MAX__));
    }
};

// Of a row of 16 lanes, whose groups are m lanes each and have their scores' keys in the first of them (`first`, kClosed
// in the others): how many groups go before the lane's, those of a larger key and lower ones of the same.  Fifteen looks
// that do not wait for each other, where taking the best of those left does (2,400 cycles for 4 of 8).
template <int R = 1>
__device__ inline int groups_before(int first, int key, int lane, int m)
{
    const int other = dpp<0x120 + R>(first);   // of lane - R, round the row
    const bool lower = ((lane - R) & 15) < (lane & -m);
    const int before = other > key || (other == key && lower) ? 1 : 0;
    if constexpr (R < 15)
        return before + groups_before<R + 1>(first, key, lane, m);
    else
        return before;
}

// Weights from the logit z of a lane's choice or choices (-inf: none), N a lane; reduce: over the token's lanes.
template <bool SIGMOID, int N, typename R>
__device__ inline void shares(const float *z, float *share, bool renormalize, float top, float total, R reduce)
{
    if (!renormalize) {
#pragma unroll
        for (int h = 0; h < N; ++h) share[h] = SIGMOID ? sigmoid_of(z[h]) : exp_from(z[h], top) / total;
    } else {
        // the scores over that of the largest logit chosen, a factor that they share left out: none underflows to 0 / 0
        float largest = z[0], sum = 0.0f;
#pragma unroll
        for (int h = 1; h < N; ++h) largest = fmaxf(largest, z[h]);
        largest = reduce(largest, Max());
#pragma unroll
        for (int h = 0; h < N; ++h) {
            share[h] = SIGMOID ? exp_from(fminf(z[h], 0.0f), fminf(largest, 0.0f)) / (1.0f + exp_from(-fabsf(z[h]), 0.0f))
                               : exp_from(z[h], largest);
            share[h] = z[h] > -INFINITY ? share[h] : 0.0f;
            sum += share[h];
        }
        sum = reduce(sum, Sum());
#pragma unroll
        for (int h = 0; h < N; ++h) share[h] /= sum;
    }
}

constexpr int kAgain = -2;   // in place of a token's first choice: it is chosen for again

// LDS: [here * top_k] choices, then the tokens' keys and, where groups are not whole lanes, their scores; when those are
// done the counts of the order.
template <typename T, int PER, bool VEC, bool SIGMOID>
__global__ __launch_bounds__(choose_threads(PER)) void k_choose_balanced(BalancedRoute q, int group, int bits, bool alone)
{
    constexpr int kChoose = choose_threads(PER), kWaves = kChoose / 64;
    constexpr float kUnit = 1.0f / (1 << 22), kLog2 = 1.44269504f;
    extern __shared__ __attribute__((aligned(16))) int lds[];
    __shared__ int sh[kWaves];
    const int64_t first = workgroup() * group;
    if (first >= q.tokens && first > 0) return;
    const int here = q.tokens - first < group ? (int)(q.tokens - first) : group;
    const int experts = q.experts, top_k = q.top_k, each = experts / q.groups;
    int *const chosen = lds;
    int *const sums = lds + ((here * top_k + 3) & ~3);   // whole vectors
    const int lane = threadIdx.x & 15, wave_lane = threadIdx.x & 63;
    int *const row = sums + (threadIdx.x >> 4) * key_row(PER);
    const int m = lanes_a_group(each, PER);
    const bool grouped = q.top_groups < q.groups, scored = q.bias || grouped || (!SIGMOID && !q.renormalize);
    for (int base = (threadIdx.x >> 6) * 4; base < here; base += kChoose / 16) {   // the same in a wave
        const int t0 = min(base + (wave_lane >> 4), here - 1);
        const int64_t t = first + t0;
        const T *const logits = static_cast<const T *>(q.logits) + t * q.stride;
        const bool keep = !q.keep || q.keep[t];
        float x[PER];
        int v[PER];
        load_logits<T, PER, VEC, true>(x, logits, lane, experts, keep);
        float top = -INFINITY, total = 1.0f, error = 2 * kUnit;
        if (scored) {
            float bias[PER] = {};
            if (q.bias) {
                int at = lane * PER;
                asm volatile("" : "+v"(at));   // loaded for every token: held they are as many registers as the keys
#pragma unroll
                for (int c = 0; c < PER; ++c) bias[c] = q.bias[VEC ? at + c : min(at + c, experts - 1)];
            }
            // A sigmoid by exp2 and rcp, a unit each: its error is below 2^-22, as |x| s (1 - s) < 1/4.  A share of the
            // softmax: below (PER / 2 + 14) 2^-23 of the largest share: PER / 2 + 2 by the sum, 10 by the exponents' rounding,
            // whose mean is of the entropy's at most 10 bits, 2 by rcp and product.  Twice that for the difference of two.
            if constexpr (SIGMOID) {
#pragma unroll
                for (int c = 0; c < PER; ++c)
                    x[c] = x[c] == -INFINITY ? x[c] : __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x[c] * -kLog2));
            } else {
                top = row_reduce(lane_largest<float, PER>(x), Max());
                total = 0.0f;
#pragma unroll
                for (int c = 0; c < PER; ++c) {
                    const float e = x[c] == top ? 1.0f : __builtin_amdgcn_exp2f((x[c] - top) * kLog2);
                    total += e;
                    x[c] = x[c] > -INFINITY ? e : -INFINITY;
                }
                total = row_reduce(total, Sum());   // of a closed token 16 * PER
                const float size = __builtin_amdgcn_rcpf(total);
                error = (PER / 2 + 14) * kUnit * size;
#pragma unroll
                for (int c = 0; c < PER; ++c) x[c] *= size;
            }
#pragma unroll
            for (int c = 0; c < PER; ++c) x[c] += bias[c];
#pragma unroll
            for (int c = 0; c < PER; ++c) v[c] = x[c] > -INFINITY ? key_of(x[c]) : kClosed;   // a NaN bias closes too
        } else {
#pragma unroll
            for (int c = 0; c < PER; ++c) v[c] = key_of(x[c]);
        }
        bool again = false, near = false;   // in the choice of groups, of experts
        if (grouped) {
            float least = INFINITY, most_left = -INFINITY, own_error;   // of a group that stays, of one that does not
            if (m > 0) {
                Top2 best = {v[0], kClosed};
#pragma unroll
                for (int c = 1; c < PER; ++c) best.take(v[c]);
                best.over_lanes(m);
                const int key = best.score(q.group_best, own_error);
                const int better = groups_before(lane % m == 0 ? key : kClosed, key, lane, m);   // by all lanes
                const bool stays = key != kClosed && better < q.top_groups;
                if (stays)
                    least = logit_of(key) - (error + own_error);
                else if (key != kClosed)
                    most_left = logit_of(key) + (error + own_error);
#pragma unroll
                for (int c = 0; c < PER; ++c) v[c] = stays ? v[c] : kClosed;
            } else {
                int *const score = sums + kChoose / 16 * key_row(PER) + (threadIdx.x >> 4) * HAPMOE_MAX_GROUPS;
                wave_order();
#pragma unroll
                for (int c = 0; c < PER; c += 4)
                    *reinterpret_cast<int4 *>(row + lane * PER + c) = make_int4(v[c], v[c + 1], v[c + 2], v[c + 3]);
                wave_order();
#pragma unroll 1
                for (int g0 = 0; g0 < q.groups; g0 += 16) {
                    const int g = g0 + lane;
                    Top2 best = {kClosed, kClosed};
                    if (g < q.groups) {
#pragma unroll 1
                        for (int i = 0; i < each; ++i) best.take(row[g * each + i]);
                        score[g] = best.score(q.group_best, own_error);
                    }
                    wave_order();   // the keys in the first g0 + 16 places are read: the groups' errors go there
                    if (g < q.groups) row[g] = __builtin_bit_cast(int, own_error);
                }
                uint64_t taken = 0;
#pragma unroll 1
                for (int j = 0; j < q.top_groups; ++j) {   // the best of those left, the lowest of equal ones
                    int most = kClosed;
                    for (int g = lane; g < q.groups; g += 16) most = Max()(most, score[g]);
                    most = row_reduce(most, Max());
                    if (most == kClosed) break;
                    int best = lane;
                    while (best < q.groups && score[best] != most) best += 16;
                    best = row_reduce(best < q.groups ? best : INT32_MAX, Min());
                    taken |= 1ull << best;
                    if (best % 16 == lane) {
                        score[best] = kClosed;
                        least = fminf(least, logit_of(most) - (error + __builtin_bit_cast(float, row[best])));
                    }
                }
                for (int g = lane; g < q.groups; g += 16)
                    if (score[g] != kClosed)
                        most_left = fmaxf(most_left, logit_of(score[g]) + (error + __builtin_bit_cast(float, row[g])));
                int g = lane * PER / each;
                asm volatile("" : "+v"(g));   // the groups of PER experts again for every token, not in registers
                int in = lane * PER - g * each;
#pragma unroll
                for (int c = 0; c < PER; ++c) {
                    v[c] = g < q.groups && taken >> g & 1 ? v[c] : kClosed;
                    if (++in == each) in = 0, ++g;
                }
            }
            least = row_reduce(least, Min()), most_left = row_reduce(most_left, Max());
            again = most_left > -INFINITY && !(least > most_left);
        }
        if (!q.bias && scored) {   // the scores' order is that of the logits
            load_logits<T, PER, VEC, true>(x, logits, lane, experts, keep);
#pragma unroll
            for (int c = 0; c < PER; ++c) v[c] = v[c] == kClosed ? kClosed : key_of(x[c]);
        }
        if constexpr (keys_in_lds(PER)) {
            wave_order();   // the keys before are read
#pragma unroll
            for (int c = 0; c < PER; c += 4)
                *reinterpret_cast<int4 *>(row + lane * PER + c) = make_int4(v[c], v[c + 1], v[c + 2], v[c + 3]);
            wave_order();
        }
        int own = lane_largest<int, PER>(v), most = row_reduce(own, Max());
        auto take = [&]() {   // the expert that has `most`, the lowest; `most` of those left
            int best;
            if constexpr (keys_in_lds(PER)) {
                const int from = first_of_row(own == most);
                int k[PER / 16], at = 0;
#pragma unroll
                for (int i = 0; i < PER / 16; ++i) k[i] = row[from * PER + 16 * i + lane];
                const int others = row_reduce(lane == from ? kClosed : own, Max());   // while those are on their way
#pragma unroll
                for (int i = PER / 16 - 1; i >= 0; --i) {
                    const int l = first_of_row(k[i] == most);
                    at = l < 16 ? 16 * i + l : at;
                }
                best = from * PER + at;
#pragma unroll
                for (int i = 0; i < PER / 16; ++i) k[i] = at == 16 * i + lane ? kClosed : k[i];
                if (lane == 0) row[best] = kClosed;
                wave_order();
                const int left = row_reduce(lane_largest<int, PER / 16>(k), Max());
                own = lane == from ? left : own;
                most = Max()(left, others);
            } else {
                int at = PER;
#pragma unroll
                for (int c = PER - 1; c >= 0; --c) at = v[c] == most ? c : at;
                best = row_reduce(at < PER ? lane * PER + at : INT32_MAX, Min());
                const int mine = best - lane * PER;
#pragma unroll
                for (int c = 0; c < PER; ++c) v[c] = c == mine ? kClosed : v[c];
                own = lane_largest<int, PER>(v);
                most = row_reduce(own, Max());
            }
            return best;
        };
        int who[2] = {-1, -1}, won[2] = {kClosed, kClosed};   // choices lane and lane + 16 and their keys
        for (int j = 0; j < top_k; ++j) {
            const int key = most, best = take();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                won[h] = lane + 16 * h == j ? key : won[h];
                who[h] = lane + 16 * h == j && key != kClosed ? best : who[h];
            }
        }
        if (q.bias) {
            // a choice and the one after it, of the next lane; the last one and the first that is not chosen
            auto after = [&](int a, int b, int beyond, int h) {
                const int x0 = dpp<0x12f>(a), x1 = dpp<0x12f>(b);
                return lane + 16 * h == top_k - 1 ? beyond : h == 0 && lane < 15 ? x0 : x1;
            };
            auto within = [&](int key, int next) {
                const float value = logit_of(key);
                return key != kClosed && next != kClosed && !(value - logit_of(next) > error + kUnit / 2 * fabsf(value));
            };
            bool close[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) close[h] = within(won[h], after(won[0], won[1], most, h));
            if (__ballot(close[0] || close[1])) {
                // equal logits and biases have equal sums, however near; others may not be in this order
                const int key = most, best = take(), extra = key != kClosed ? best : -1;
                int found = 0;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int next = after(who[0], who[1], extra, h);
                    if (close[h]) {
                        found |= to_f32(logits[who[h]]) != to_f32(logits[next]) || q.bias[who[h]] != q.bias[next] ? 1 : 0;
                        // the first that is not chosen is near to the last, and another to it
                        found |= lane + 16 * h == top_k - 1 && within(key, most) ? 2 : 0;
                    }
                }
                found = row_reduce(found & 1, Max()) | row_reduce(found & 2, Max());
                near = found & 1;
                again = again || found & 2;
                who[0] = lane == top_k ? extra : who[0];
            }
        }
        // Up to 15 choices and the first that is not are one a lane: where some are near they are put in order here, by their
        // scores in 64 bits.  All else that is near takes a wave.
        again = again || (near && top_k > 15);
        if (__ballot(near && !again)) {
            double all = 0.0;   // of a softmax
            if constexpr (!SIGMOID) {
#pragma unroll 1
                for (int c = lane * PER; c < min(lane * PER + PER, experts); ++c) {
                    const float y = to_f32(logits[c]);
                    all += y > -INFINITY && top > -INFINITY ? exp(y == top ? 0.0 : (double)y - (double)top) : 0.0;
                }
                all = row_reduce(all, Sum());
            }
            const int e = who[0];
            double sum = -INFINITY;
            if (e >= 0) {
                const float y = to_f32(logits[e]);
                const double power = exp(SIGMOID ? -(double)y : y == top ? 0.0 : (double)y - (double)top);
                sum = (SIGMOID ? 1.0 : power) / (SIGMOID ? 1.0 + power : all) + (double)(q.bias ? q.bias[e] : 0.0f);
            }
            int rank = 0, other_e = e;
            double other = sum;
#pragma unroll 1
            for (int i = 1; i < 16; ++i) {
                other = dpp<0x121>(other), other_e = dpp<0x121>(other_e);   // the next lane's of the row
                rank += other > sum || (other == sum && other_e >= 0 && other_e < e);
            }
            wave_order();
            if (near && !again && e >= 0) row[rank] = e;
            wave_order();
            if (near && !again && e >= 0) who[0] = row[lane];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) who[h] = lane + 16 * h < top_k ? who[h] : -1;
        float z[2], share[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) z[h] = who[h] >= 0 ? to_f32(logits[who[h]]) : -INFINITY;
        shares<SIGMOID, 2>(z, share, q.renormalize, top, total, [](float x, auto f) { return row_reduce(x, f); });
        if (base + (wave_lane >> 4) < here) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = lane + 16 * h;
                if (j < top_k) chosen[t0 * top_k + j] = again && j == 0 ? kAgain : who[h];
                if (j < top_k && !again) {
                    q.weight[t * top_k + j] = who[h] >= 0 ? share[h] * q.scale : 0.0f;
                    q.expert[t * top_k + j] = who[h];
                }
            }
        }
    }
    __syncthreads();
    // the tokens that are left, a wave for each in turn
    int number = 0;
    uint64_t left = __ballot(wave_lane < here && chosen[wave_lane * top_k] == kAgain);
    __syncthreads();   // every wave has them before the first is replaced
    for (; left; left &= left - 1) {
        if (number++ % kWaves != (int)(threadIdx.x >> 6)) continue;
        const int t0 = __ffsll((unsigned long long)left) - 1;
        const int64_t t = first + t0;
        const T *const logits = static_cast<const T *>(q.logits) + t * q.stride;
        float top, total, z, share;
        // the wave's four rows of keys are done with, and as long as twice the experts
        choose_exactly<T, PER / 4>(q, logits, !q.keep || q.keep[t],
                                   reinterpret_cast<double *>(sums + (threadIdx.x >> 6) * 4 * key_row(PER)),
                                   chosen + t0 * top_k, top, total);
        wave_order();
        const int who = wave_lane < top_k ? chosen[t0 * top_k + wave_lane] : -1;
        z = who >= 0 ? to_f32(logits[who]) : -INFINITY;
        shares<SIGMOID, 1>(&z, &share, q.renormalize, top, total, [](float x, auto f) { return wave_reduce(x, f); });
        if (wave_lane < top_k) {
            q.weight[t * top_k + wave_lane] = who >= 0 ? share * q.scale : 0.0f;
            q.expert[t * top_k + wave_lane] = who;
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < kWaves * experts; e += kChoose) sums[e] = 0;
    __syncthreads();
    int32_t *const hist = static_cast<int32_t *>(q.ws);
    if (alone)
        order_rows<kChoose, true>(chosen, sums, sh, here, top_k, first, experts, bits, q.place, hist, q.count, q.offset,
                                  q.slot);
    else
        order_rows<kChoose, false>(chosen, sums, sh, here, top_k, first, experts, bits, q.place, hist, q.count, q.offset,
                                   q.slot);
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
    const hipError_t e = by_type(a.type, [&](auto t) {
        using T = decltype(t);
        return by_experts(a.experts, [&](auto per) {
            constexpr int PER = decltype(per)::value;
            constexpr int kChoose = choose_threads(PER);
            const bool vec = a.experts == 16 * PER && aligned(a.logits, 16) && a.stride * (int64_t)sizeof(T) % 16 == 0;
            const int sums = (kChoose / 64 + (alone ? 1 : 0)) * a.experts, keys = kChoose / 16 * key_row(PER);
            const bool any = a.top_groups < a.groups && lanes_a_group(a.experts / a.groups, PER) == 0;
            const int scores = any ? kChoose / 16 * HAPMOE_MAX_GROUPS : 0;
            const size_t lds = (((rows_here + 3) & ~3) + (keys + scores > sums ? keys + scores : sums)) * sizeof(int);
            auto kernel = [&](auto sigmoid) {
                constexpr bool S = decltype(sigmoid)::value;
                return vec ? k_choose_balanced<T, PER, true, S> : k_choose_balanced<T, PER, false, S>;
            };
            hipLaunchKernelGGL((a.sigmoid ? kernel(std::true_type()) : kernel(std::false_type())), many(workgroups),
                               dim3(kChoose), lds, s, a, group, bits, alone);
            return hipGetLastError();
        });
    });
    if (e != hipSuccess || alone) return e;
    return launch_route_order(a.expert, static_cast<int32_t *>(a.ws), workgroups, a.tokens * a.top_k, a.experts,
                              group * a.top_k, a.count, a.offset, a.place, a.slot, s);
}

}  // namespace hapmoe
