// Rows of a table by token, and the table's gradient.
//
// out[t] = scale table[token[t]], a row of zeros where the token is none of the table's.
//
// The gradient's row of a token is the sum over its places in a fixed order, with no atomics.  The places are put in the
// tokens' order by segments of 4,096, few by counting for each place those before it, many by a stable sort of 9 bits a
// pass in LDS; a launch puts up to 16 segments into one order, every place by a search in each of the others.  Then
// workgroups take equal chunks of the sorted places, whatever the tokens' shares: a token that lies within a chunk is
// written, one that goes on into the next leaves its sums in the workspace, and a last launch puts those together.  Rows
// without a token are cleared by further workgroups of the same launch, which look for them in the sorted places.
//
// Bound by HBM where the table's gradient is written whole, by launches that wait for each other where few rows are added
// to.  bf16, 32,768 places, tokens as words fall, of 131,072 x 4,096: forward 74 to 90 us (0.38 GB, 4.2 to 5.1 TB/s), sort
// 12, segments together 11, sums and clears 461 to 495 (2.4 GB, 4.9 to 5.2 TB/s; a fill alone reaches 5.4 to 6.8), what goes
// on 10 to 12.  4,001 places of 1,023 fp16 added to: 4.9 forward, then 5.0, 7.7 and 6.5.
#include "operators.h"

namespace hapmoe {
namespace {

constexpr int kThreads = 256;
constexpr int kSegment = 4096;     // places of a sort
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kSteps = kSegment / kSortThreads;
constexpr int kDigit = 9, kBins = 1 << kDigit;
constexpr int kWays = 16;          // segments that a launch puts together

template <typename I>
__device__ inline int64_t token_at(const void *token, int64_t t)
{
    return (int64_t) static_cast<const I *>(token)[t];
}

// Eight columns of a thread; where less than eight are left, the row's last 8, of which the first `skip` are others'.
struct Columns {
    int first, skip;
    __device__ Columns(int hidden, int k) : first(min(k * 8, hidden - 8)), skip(k * 8 - first) {}
};

template <typename T>
__device__ inline void put(T *__restrict__ row, const Columns &c, const float *v)
{
    if (c.skip == 0) {
        store_words(row + c.first, words_of<T>(v));
    } else {
#pragma unroll
        for (int j = 1; j < 8; ++j)
            if (j >= c.skip) row[c.first + j] = from_f32<T>(v[j]);
    }
}

// Threads of a row (of 8 columns each): a power of two.
__host__ __device__ inline int lanes_of(int64_t hidden)
{
    int lanes = 8;
    while (lanes < kThreads && lanes * 8 < hidden) lanes *= 2;
    return lanes;
}

// A row by `lanes` threads, or by one where it is shorter than a vector.  LANES: that number, 64 at least, so that a
// wave's token and addresses are the same in every lane (32,768 of 4,096: 76 us, 89 with each lane's own), or 0.
template <typename T, typename I, int LANES>
__global__ __launch_bounds__(kThreads) void k_embed(const void *__restrict__ token, int64_t tokens,
                                                    const T *__restrict__ table, int64_t stride, int64_t vocab,
                                                    int hidden, int lanes, float scale, T *__restrict__ out)
{
    if constexpr (LANES > 0) lanes = LANES;
    const int in = threadIdx.x / lanes;
    const int64_t t = workgroup() * (kThreads / lanes) + (LANES > 0 ? __builtin_amdgcn_readfirstlane(in) : in);
    if (t >= tokens) return;
    const int64_t v = token_at<I>(token, t);
    const bool real = (uint64_t)v < (uint64_t)vocab;
    if (LANES == 0 && hidden < 8) {
        for (int h = 0; h < hidden; ++h)
            out[t * hidden + h] = from_f32<T>(real ? to_f32(table[v * stride + h]) * scale : 0.0f);
        return;
    }
    const Columns c(hidden, blockIdx.y * lanes + threadIdx.x % lanes);
    if (c.skip >= 8) return;
    float r[8] = {};
    if (real) {
        const Words<T> w = load_words(table + v * stride + c.first);
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = element<T>(w, j) * scale;
    }
    put(out + t * hidden, c, r);
}

// Segment blockIdx.x: sorted[i] = (token, place) for its places, the tokens ascending, the places of one ascending.
// Tokens that are none of the table's count as `vocab`.  bits: of vocab.
template <typename I>
__global__ __launch_bounds__(kSortThreads) void k_sort(const void *__restrict__ token, int64_t tokens, int64_t vocab,
                                                       int bits, int2 *__restrict__ sorted)
{
    __shared__ int key[kSegment];
    __shared__ uint16_t order[2][kSegment];
    __shared__ __attribute__((aligned(16))) uint16_t count[kSortWaves][kBins];
    __shared__ int sh[kBins / 64];
    static_assert(sizeof(count) == kSortThreads * 16, "a thread clears 16 bytes");
    const int64_t first = (int64_t)blockIdx.x * kSegment;
    const int n = tokens - first < kSegment ? (int)(tokens - first) : kSegment;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < n; i += kSortThreads) {
        const int64_t v = token_at<I>(token, first + i);
        key[i] = (uint64_t)v < (uint64_t)vocab ? (int)v : (int)vocab;
    }
    const int run = (n + kSortThreads - 1) / kSortThreads * 64;   // a wave's
    const int lo = wave * run, hi = min(lo + run, n);
    int from = 0;
    for (int shift = 0; shift < bits; shift += kDigit, from ^= 1) {
        reinterpret_cast<uint4 *>(count)[threadIdx.x] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        int held[kSteps], rank[kSteps];   // place and digit, rank among the wave's of its digit
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int i = lo + s * 64 + lane;
            if (lo + s * 64 >= hi) break;
            const bool in = i < hi;
            const int place = !in ? 0 : shift == 0 ? i : order[from][i];
            const int digit = in ? key[place] >> shift & (kBins - 1) : 0;
            uint64_t same = __ballot(in);
#pragma unroll
            for (int b = 0; b < kDigit; ++b) {
                const bool one = digit >> b & 1;
                const uint64_t on = __ballot(one);
                same &= one ? on : ~on;
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
        if (threadIdx.x < kBins) {
            int own[kSortWaves], total = 0;
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) own[w] = count[w][threadIdx.x];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                const int c = own[w];
                own[w] = total;
                total += c;
            }
            int inc = total;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int o = __shfl_up(inc, d, 64);
                if (lane >= d) inc += o;
            }
            if (lane == 63) sh[wave] = inc;
            const int before = inc - total;
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) count[w][threadIdx.x] = (uint16_t)(own[w] + before);
        }
        __syncthreads();
        // the digits' totals by 64: each thread adds what is before its own digits
        int base[kBins / 64], sum = 0;
#pragma unroll
        for (int g = 0; g < kBins / 64; ++g) {
            base[g] = sum;
            sum += sh[g];
        }
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int i = lo + s * 64 + lane;
            if (i >= hi) continue;
            const int digit = held[s] >> 16;
            int before = 0;
#pragma unroll
            for (int g = 1; g < kBins / 64; ++g) before = digit >> 6 == g ? base[g] : before;
            order[from ^ 1][before + count[wave][digit] + rank[s]] = (uint16_t)(held[s] & 0xffff);
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < n; i += kSortThreads) {
        const int place = order[from][i];
        sorted[first + i] = make_int2(key[place], (int)first + place);
    }
}

// The same order by counting: a place's is the number of places of lower tokens and of earlier ones of its own.  A
// workgroup counts for 16 places of a segment, each of its threads for one of them over a 64th of the segment's, four at a
// time out of LDS: so that a few thousand places are all CUs' work and not one's.
constexpr int kRanked = 16;
template <typename I>
__global__ __launch_bounds__(kSortThreads) void k_rank(const void *__restrict__ token, int64_t tokens, int64_t vocab,
                                                       int2 *__restrict__ sorted)
{
    __shared__ __attribute__((aligned(16))) int key[kSegment];
    __shared__ int part[kSortWaves][kRanked];
    constexpr int kGroups = kSegment / kRanked;
    const int64_t first = (int64_t)(blockIdx.x / kGroups) * kSegment;
    const int n = tokens - first < kSegment ? (int)(tokens - first) : kSegment, i0 = blockIdx.x % kGroups * kRanked;
    if (i0 >= n) return;
    const int fours = (n + 3) / 4;
    for (int i = threadIdx.x; i < fours * 4; i += kSortThreads) {
        const int64_t v = i < n ? token_at<I>(token, first + i) : 0;
        key[i] = i >= n ? INT32_MAX : (uint64_t)v < (uint64_t)vocab ? (int)v : (int)vocab;   // behind all: counted by none
    }
    __syncthreads();
    const int wave = threadIdx.x >> 6, i = i0 + (threadIdx.x & 15);
    const int mine = i < n ? key[i] : 0;
    int count = 0;
    for (int f = threadIdx.x >> 4; f < fours; f += kSortThreads / 16) {
        const int4 k = reinterpret_cast<const int4 *>(key)[f];
        const int below = mine + (f * 4 + 3 < i ? 1 : 0);   // equal ones count where they are earlier
        count += (k.x < below) + (k.y < below) + (k.z < below) + (k.w < below);
    }
    if ((threadIdx.x >> 4) == 0 && i < n)   // and those in the place's own four
        for (int j = i & ~3; j < i; ++j) count += key[j] == mine;
    count += __shfl_xor(count, 16, 64);
    count += __shfl_xor(count, 32, 64);
    if ((threadIdx.x & 63) < kRanked) part[wave][threadIdx.x & 63] = count;
    __syncthreads();
    if (threadIdx.x < kRanked && i < n) {
        int at = 0;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) at += part[w][threadIdx.x];
        sorted[first + at] = make_int2(mine, (int)first + i);
    }
}

// Runs of `run` sorted places each -> runs of kWays * run: a place goes behind its own run's earlier ones and, of every
// other run, those of lower tokens, and of the runs before its own those of the same token too.  A search begins in
// kSamples places of each run, out of LDS: 17 us for 32,768 places with all of its steps out of the cache.
constexpr int kSamples = 128;
__global__ __launch_bounds__(kThreads) void k_merge(const int2 *__restrict__ from, int2 *__restrict__ to, int n, int run)
{
    __shared__ int sample[kWays][kSamples];
    const int64_t first = workgroup() * kThreads, whole = (int64_t)run * kWays;
    if (first >= n) return;
    const int64_t base = first / whole * whole;   // of all of this workgroup's places: kThreads divides a run
    const int i = (int)min(first + threadIdx.x, (int64_t)n - 1), step = run / kSamples;
    auto begin = [&](int w) { return (int)min(base + (int64_t)w * run, (int64_t)n); };
    const int2 v = from[i];
#pragma unroll
    for (int q = 0; q < kWays * kSamples / kThreads; ++q) {
        const int s = q * kThreads + threadIdx.x;
        const int64_t at = base + (int64_t)s * step;
        (&sample[0][0])[s] = at < n ? from[at].x : INT32_MAX;
    }
    __syncthreads();
    const int mine = i / run * run;
    int lo[kWays], size[kWays];   // the first that goes behind v is in lo .. lo + size
#pragma unroll
    for (int w = 0; w < kWays; ++w) {
        const int key = begin(w) < mine ? v.x : v.x - 1;   // those up to it go before: tokens are whole numbers
        int c = 0;   // samples that do
#pragma unroll
        for (int half = kSamples / 2; half > 0; half >>= 1) c += sample[w][c + half - 1] <= key ? half : 0;
        c += sample[w][c] <= key ? 1 : 0;
        lo[w] = begin(w) + (c > 0 ? (c - 1) * step + 1 : 0);
        const int end = (int)min(begin(w) + (int64_t)c * step, (int64_t)begin(w + 1));
        size[w] = begin(w) == mine || c == 0 ? 0 : max(end - lo[w], 0);
    }
    for (int most = step; most > 0; most >>= 1) {   // all runs' searches side by side
        int other[kWays];
#pragma unroll
        for (int w = 0; w < kWays; ++w) other[w] = from[min(lo[w] + (size[w] >> 1), n - 1)].x;
#pragma unroll
        for (int w = 0; w < kWays; ++w) {
            const int half = size[w] >> 1;
            const bool before = size[w] > 0 && other[w] <= (begin(w) < mine ? v.x : v.x - 1);
            size[w] = before ? size[w] - half - 1 : half;
            lo[w] += before ? half + 1 : 0;
        }
    }
    int64_t at = base + (i - mine);
#pragma unroll
    for (int w = 0; w < kWays; ++w)
        if (begin(w) != mine) at += lo[w] - begin(w);
    if (first + threadIdx.x < n) to[at] = v;
}

// The first sorted place of a token, or of those above it.
__device__ inline int64_t first_place(const int2 *__restrict__ sorted, int64_t n, int token)
{
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t half = (lo + hi) >> 1;
        if (sorted[half].x < token)
            lo = half + 1;
        else
            hi = half;
    }
    return lo;
}

constexpr int kChunkMost = 128, kRowsAhead = 8;

// The first `sums` workgroups of x have chunks of the n sorted places, the others rows to clear where they have no token.
// ADD: no rows to clear; what a token's row holds is loaded with the rows that are added to it.
template <typename T, bool ADD>
__global__ __launch_bounds__(kThreads) void k_embed_sum(const T *__restrict__ d_out, int64_t stride, int hidden,
                                                        const int2 *__restrict__ sorted, int64_t n, int chunk, int lanes,
                                                        int vocab, float scale, float *__restrict__ d_table,
                                                        float *__restrict__ part, int64_t sums, int rows_each)
{
    extern __shared__ int2 lds[];   // a chunk's places, those before and behind it at its ends
    const int64_t group = workgroup();
    if (group >= sums) {
        const int64_t row0 = ((group - sums) * gridDim.y + blockIdx.y) * rows_each;
        if (ADD || row0 >= vocab) return;
        const int rows = vocab - row0 < rows_each ? (int)(vocab - row0) : rows_each;
        int *const named = reinterpret_cast<int *>(lds);
        if ((int)threadIdx.x < rows) {
            const int row = (int)row0 + threadIdx.x;
            const int64_t lo = first_place(sorted, n, row);
            named[threadIdx.x] = lo < n && sorted[lo].x == row;
        }
        __syncthreads();
        // 16 bytes a thread side by side, whole rows one behind the other
        const int across = lanes < kThreads / 2 ? 2 * lanes : kThreads, per = kThreads / across;
        for (int r = threadIdx.x / across; r < rows; r += per) {
            if (named[r]) continue;
            float *const to = d_table + (row0 + r) * hidden;
            for (int k = threadIdx.x % across * 4; k < hidden; k += 4 * across) {
                if (k + 4 <= hidden) {
                    typedef uint32_t Four __attribute__((ext_vector_type(4)));
                    const Four none = {};
                    __builtin_memcpy(to + k, &none, sizeof(none));
                } else {
                    for (int j = k; j < hidden; ++j) to[j] = 0.0f;
                }
            }
        }
        return;
    }
    const int mine = threadIdx.x / lanes;
    const int64_t which = group * (kThreads / lanes) + mine, lo = which * chunk;
    int2 *const at = lds + mine * (chunk + 2) + 1;   // at[-1] .. at[chunk]
    for (int i = (int)(threadIdx.x % lanes) - 1; i <= chunk; i += lanes) {
        const int64_t p = lo + i;
        at[i] = p >= 0 && p < n ? sorted[p] : make_int2(p < 0 ? -1 : vocab, 0);
    }
    __syncthreads();
    const Columns c(hidden, blockIdx.y * lanes + threadIdx.x % lanes);
    if (lo >= n || c.skip >= 8) return;
    float sum[8] = {};
    for (int i0 = 0; i0 < chunk && at[i0].x != vocab; i0 += kRowsAhead) {
        Words<T> w[kRowsAhead];
        Words<float> old[ADD ? kRowsAhead : 1];
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) w[u] = load_words(d_out + at[i0 + u].y * stride + c.first);
        if constexpr (ADD)
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u) {   // where no row ends: one that is in the cache
                const int token = at[i0 + u].x;
                const int row = token != vocab && at[i0 + u + 1].x != token ? token : at[i0].x;
                old[u] = load_words(d_table + (int64_t)row * hidden + c.first);
            }
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            const int i = i0 + u, token = at[i].x;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += element<T>(w[u], j);
            const bool goes_on = at[i + 1].x == token;
            if (token == vocab || (goes_on && i + 1 < chunk)) continue;
            const bool began = at[-1].x == token;
            if (began || goes_on) {
                put(part + (which * 2 + (began ? 0 : 1)) * hidden, c, sum);
            } else {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[j] = sum[j] * scale;
                    if constexpr (ADD) v[j] += element<float>(old[u], j);
                }
                put(d_table + (int64_t)token * hidden, c, v);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
        }
    }
}

// The token that begins in a chunk and goes on: its sums there and in the chunks that follow, a run of them for each
// quarter of the workgroup, then the quarters in their order.  All of a token's chunks are one workgroup's for its columns,
// so where most places have one token and the columns are few, it is what bounds the call: 32,768 places of one token, 64
// columns 186 us (as words fall 15), 512 83 (9), 4,096 44 (10), 7,168 28 (14).
constexpr int kJoinThreads = 1024, kQuarters = kJoinThreads / kThreads;
__global__ __launch_bounds__(kJoinThreads) void k_embed_join(int hidden, const int2 *__restrict__ sorted, int64_t n,
                                                             int chunk, int lanes, int vocab, float scale, bool add,
                                                             const float *__restrict__ part, float *__restrict__ d_table)
{
    constexpr int kAhead = 8;
    __shared__ float sh[kQuarters - 1][8][kThreads];
    const int thread = threadIdx.x % kThreads, quarter = threadIdx.x / kThreads;
    const int64_t which = workgroup() * (kThreads / lanes) + thread / lanes, lo = which * chunk, hi = lo + chunk;
    const Columns c(hidden, blockIdx.y * lanes + thread % lanes);
    int token = vocab;
    if (hi < n) {
        token = sorted[hi - 1].x;
        if (sorted[hi].x != token || (lo > 0 && sorted[lo - 1].x == token)) token = vocab;
    }
    const bool goes_on = token != vocab, has = goes_on && c.skip < 8;
    if (!__syncthreads_or(goes_on)) return;
    // chunks behind this one that begin with the token, of `size` that may: by 64 of them at once where a wave has one token
    // (in all its lanes, those without columns too)
    int64_t chunks = 0, size = goes_on ? (n - hi + chunk - 1) / chunk : 0;
    if (lanes >= 64) {
        while (size > 0) {
            const int64_t step = (size + 63) / 64, at = ((threadIdx.x & 63) + 1) * step - 1;
            const bool more = at < size && sorted[hi + (chunks + at) * chunk].x == token;
            const int64_t passed = (int64_t)__popcll(__ballot(more)) * step;
            chunks += passed;
            size = min(step - 1, size - passed);
        }
    } else {
        while (size > 0) {
            const int64_t half = size >> 1;
            const bool more = sorted[hi + (chunks + half) * chunk].x == token;
            chunks += more ? half + 1 : 0;
            size = more ? size - half - 1 : half;
        }
    }
    // sum 0 is this chunk's, sum i of the chunk i behind it
    const int64_t each = (chunks + kQuarters) / kQuarters, first = min(quarter * each, chunks + 1);
    const int64_t last = min(first + each, chunks + 1);
    const float *const from = part + which * 2 * hidden + c.first;
    float sum[8] = {};
    for (int64_t i = first; has && i < last; i += kAhead) {
        Words<float> x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t at = min(i + u, last - 1);
            x[u] = load_words(from + (at * 2 + (at == 0 ? 1 : 0)) * hidden);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u < last) {
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += element<float>(x[u], j);
            }
    }
    if (quarter > 0)
#pragma unroll
        for (int j = 0; j < 8; ++j) sh[quarter - 1][j][thread] = sum[j];
    __syncthreads();
    if (quarter > 0 || !has) return;
#pragma unroll
    for (int q = 1; q < kQuarters; ++q)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += sh[q - 1][j][thread];
    float *const row = d_table + (int64_t)token * hidden;
    Words<float> old = {};
    if (add) old = load_words(row + c.first);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = element<float>(old, j) + sum[j] * scale;
    put(row, c, sum);
}

// Rows of less than 8 columns: a wave a row of the table, each lane every 64th of its places, then the lanes' sums.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_embed_narrow(const T *__restrict__ d_out, int64_t stride, int hidden,
                                                           const int2 *__restrict__ sorted, int64_t n, int vocab,
                                                           float scale, bool add, float *__restrict__ d_table)
{
    const int64_t row = workgroup() * (kThreads / 64) + (threadIdx.x >> 6);
    if (row >= vocab) return;
    const int lane = threadIdx.x & 63;
    const int64_t lo = first_place(sorted, n, (int)row), hi = first_place(sorted, n, (int)row + 1);
    if (add && lo == hi) return;
    float sum[7] = {};
    for (int64_t i = lo + lane; i < hi; i += 64) {
        const T *const from = d_out + sorted[i].y * stride;
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < hidden) sum[j] += to_f32(from[j]);
    }
#pragma unroll
    for (int j = 0; j < 7; ++j) sum[j] = wave_reduce(sum[j], Sum());
    if (lane > 0) return;
#pragma unroll
    for (int j = 0; j < 7; ++j)
        if (j < hidden) d_table[row * hidden + j] = (add ? d_table[row * hidden + j] : 0.0f) + sum[j] * scale;
}

// Up to this many places are sorted by counting.  us of a call of 64 columns by counting, by digits: 1,000 places 13.3, 13.6
// (the host's), 4,096 16.1, 22.7, 8,192 49, 55, 16,384 54, 56, 32,768 66, 58.  Beyond one segment the segments are put
// together by a launch more, 9 to 10 us: 4,096 places 5.3 to count, 4,097 5.3 and 9.1, 8,192 7.3 and 9.7, 16,384 11.9 and 9.6.
constexpr int64_t kRankMost = 16384;

// Places of a chunk: the most that leave two workgroups a CU, if any do, else 8.  us by 64, 128: 32,768 places: 131,072 x
// 4,096, tokens as words fall 513, 527, all of one token 559, 524; 32,768 x 4,096 230, 222 and 273, 228; 1,000 x 7,168 170,
// 154 and 194, 159.
int chunk_of(int64_t tokens, int64_t hidden)
{
    int chunk = kRowsAhead;
    while (chunk < kChunkMost && ceil_div(tokens, 2 * chunk) * ceil_div(hidden, 8) >= 512 * kThreads) chunk *= 2;
    return chunk;
}

template <typename F>
hipError_t by_type(int type, F f)
{
    if (type == HAPMOE_F32) return f(float());
    if (type == HAPMOE_BF16) return f(bf16());
    return f(f16());
}

}  // namespace

// sorted places twice, the sums of tokens that go on beyond a chunk
int64_t embed_ws_bytes(int64_t tokens, int64_t hidden)
{
    const int64_t places = ceil_div(tokens, 2) * 16;
    return (tokens > kSegment ? 2 : 1) * places + ceil_div(tokens, chunk_of(tokens, hidden)) * 2 * hidden * 4;
}

hipError_t launch_embed(const void *token, bool wide, int64_t tokens, const void *table, int type, int64_t stride,
                        int64_t vocab, int64_t hidden, float scale, void *out, hipStream_t s)
{
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        const int lanes = hidden < 8 ? 1 : lanes_of(hidden);
        auto kernel = [&](auto i) {
            using I = decltype(i);
            return lanes == 256   ? k_embed<T, I, 256>
                   : lanes == 128 ? k_embed<T, I, 128>
                   : lanes == 64  ? k_embed<T, I, 64>
                                  : k_embed<T, I, 0>;
        };
        hipLaunchKernelGGL((wide ? kernel(int64_t()) : kernel(int32_t())),
                           many(ceil_div(tokens, kThreads / lanes), (unsigned)ceil_div(hidden, lanes * 8)), dim3(kThreads), 0,
                           s, token, tokens, static_cast<const T *>(table), stride, vocab, (int)hidden, lanes, scale,
                           static_cast<T *>(out));
        return hipGetLastError();
    });
}

hipError_t launch_embed_backward(const void *d_out, int type, int64_t stride, int64_t tokens, int64_t hidden,
                                 const void *token, bool wide, int64_t vocab, float scale, bool add, float *d_table,
                                 void *ws, hipStream_t s)
{
    if (tokens == 0 && add) return hipSuccess;
    const int64_t places = ceil_div(tokens, 2) * 2;
    int2 *sorted = static_cast<int2 *>(ws), *other = sorted + places;
    float *part = reinterpret_cast<float *>(tokens > kSegment ? other + places : other);
    int bits = 1;
    while (vocab >> bits) ++bits;
    if (tokens > kRankMost)
        hipLaunchKernelGGL((wide ? k_sort<int64_t> : k_sort<int32_t>), dim3((unsigned)ceil_div(tokens, kSegment)),
                           dim3(kSortThreads), 0, s, token, tokens, vocab, bits, sorted);
    else if (tokens > 0)
        hipLaunchKernelGGL((wide ? k_rank<int64_t> : k_rank<int32_t>),
                           dim3((unsigned)(tokens > kSegment ? ceil_div(tokens, kSegment) * (kSegment / kRanked)
                                                             : ceil_div(tokens, kRanked))),
                           dim3(kSortThreads), 0, s, token, tokens, vocab, sorted);
    for (int64_t run = kSegment; run < tokens; run *= kWays) {
        hipLaunchKernelGGL(k_merge, many(ceil_div(tokens, kThreads)), dim3(kThreads), 0, s, sorted, other, (int)tokens,
                           (int)run);
        int2 *const t = sorted;
        sorted = other, other = t;
    }
    const int chunk = chunk_of(tokens, hidden), lanes = lanes_of(hidden);
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        const T *d = static_cast<const T *>(d_out);
        if (hidden < 8) {
            hipLaunchKernelGGL(k_embed_narrow<T>, many(ceil_div(vocab, kThreads / 64)), dim3(kThreads), 0, s, d, stride,
                               (int)hidden, sorted, tokens, (int)vocab, scale, add, d_table);
            return hipGetLastError();
        }
        const int64_t chunks = ceil_div(tokens, chunk), sums = ceil_div(chunks, kThreads / lanes);
        const unsigned columns = (unsigned)ceil_div(hidden, lanes * 8);
        // about 256 KB to clear a workgroup
        const int64_t fit = ceil_div(256 << 10, hidden * 4), rows_each = fit < kThreads ? fit : kThreads;
        const int64_t clears = add ? 0 : ceil_div(vocab, rows_each * columns);
        const size_t lds = sizeof(int2) * (kThreads / lanes) * (chunk + 2);
        hipLaunchKernelGGL((add ? k_embed_sum<T, true> : k_embed_sum<T, false>), many(sums + clears, columns),
                           dim3(kThreads), lds > kThreads * 4 ? lds : kThreads * 4, s, d, stride, (int)hidden, sorted,
                           tokens, chunk, lanes, (int)vocab, scale, d_table, part, sums, (int)rows_each);
        if (chunks > 1)
            hipLaunchKernelGGL(k_embed_join, many(ceil_div(chunks - 1, kThreads / lanes), columns), dim3(kJoinThreads), 0, s,
                               (int)hidden, sorted, tokens, chunk, lanes, (int)vocab, scale, add, part, d_table);
        return hipGetLastError();
    });
}

}  // namespace hapmoe
