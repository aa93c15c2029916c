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
#include "operators.h"

namespace hapmoe {
namespace {

constexpr int kThreads = 256;
constexpr int kPass = kThreads / 16;   // tokens of a workgroup of the gradient
// Up to this many tokens one launch: us by one, by three: 8 experts, top 2: 64 tokens 6.0, 9.3, 128 7.9, 9.3; 256 experts, top
// 8: 64 tokens 9.6, 12.4, 128 15.3, 14.0, 256 26.7, 14.2.
constexpr int kOneLaunch = 64;
constexpr int kPlaceRows = 1024;       // rows of a workgroup of the last kernel

// Tokens of a workgroup.  us by 32, by 64: 256 experts, top 8: 16,384 tokens 18.7, 19.6, 32,768 25.9, 24.5, 65,536 38.6, 34.0;
// 8 experts 13.8, 13.9, 15.7, 15.3, 21.7, 18.4; 1,024 experts, top 4, 32,768 tokens 49, 58.
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
        wave_order();
        if (e >= 0 && below == 0) own[e] += __popcll(same);
        wave_order();
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
        int *const at = sums + kWaves * experts;
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
        if (who[h] >= 0 && who[h] < 16 * PER) row[place_of(who[h])] = w[h] * (renormalize ? g[h] - mean : g[h]);
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
    hipLaunchKernelGGL(k_scan_groups, dim3((unsigned)ceil_div(experts, kScanExperts)), dim3(kScanThreads), 0, s, hist,
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
