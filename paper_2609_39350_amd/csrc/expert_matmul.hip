// Matrix products grouped by expert: y = x w^T, d_x = d_y w, d_w = d_y^T x, with
// a ragged number of rows for each expert.
//
// All three are one product out[q][p] = sum_k Q[q][k] P[p][k]: the rows of the
// output are Q's, its contiguous columns P's.
//   y    Q = x (rows, gathered)   P = w[e]             k: inputs
//   d_x  Q = d_y (rows)           P = w[e] transposed  k: outputs
//   d_w  Q = d_y transposed       P = x transposed     k: the expert's rows
// P goes in as the first operand of v_mfma_f32_16x16x32, so a lane's four results
// are neighbours in an output row and are stored at once.  An operand whose
// memory runs along k is read from LDS 16 bytes a lane, one whose memory runs
// across k by the transposing LDS read, 4 x 16 elements a row of lanes.
//
// Few rows an expert: bound by the reading of w.  16 tokens, 8 of 64 experts of 4,096
// x 2,048: 156 us, 6.9 TB/s.  Many: bound by the products (MFMA busy 52 to 66 % of the
// cycles) and by whole rounds of tiles over 256 CUs.  32,768 rows: 64 uneven experts
// of 4,096 x 2,048 530 to 540 us by the card, 1,020 to 1,040 TFLOP/s; 16 of 8,192 x 4,096
// y 1,858 to 1,869, d_x 1,889 to 1,920, d_w 2,172 to 2,250 us, down to 1,176, 1,145 and 977
// TFLOP/s, where one library product of 8,192^3 reaches 1,233 to 1,418.
#include <type_traits>

#include "operators.h"

namespace hapmoe {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ inline f32x4 mfma(s16x8 p, s16x8 q, f32x4 c, bf16)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, p), __builtin_bit_cast(bf16x8, q), c, 0,
                                                   0, 0);
}
__device__ inline f32x4 mfma(s16x8 p, s16x8 q, f32x4 c, f16)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, p), __builtin_bit_cast(f16x8, q), c, 0, 0,
                                                  0);
}

// The rows of expert e, clamped to the rows that exist.
__device__ inline int2 expert_rows(const int32_t *offset, int e, int64_t rows)
{
    const int r = (int)rows;
    const int lo = min(max(offset[e], 0), r), hi = min(max(offset[e + 1], lo), r);
    return make_int2(lo, hi);
}

struct Tile {
    int expert;   // `experts`: the rows that no expert has
    int lo, hi;   // its rows
    int q, p;     // tile of its rows and of the columns
};

// Workgroup -> tile.  Workgroups go to the eight XCDs in turn; each XCD gets a run of neighbouring tiles, which share
// rows or columns in its L2.  -1 past the last tile.
__device__ inline int64_t xcd_order(int64_t block, int64_t tiles)
{
    const int64_t run = (tiles + 7) >> 3;
    const int64_t id = (block & 7) * run + (block >> 3);
    return (block >> 3) < run && id < tiles ? id : -1;
}

// The tile of a workgroup where rows are ragged: expert by expert, the column tiles one after another and for each the
// expert's row tiles, so that neighbouring tiles share a column tile of the weights.  Every wave finds it by itself: 64
// experts at a time, a sum over their tiles, then a scan.  False past the last tile.
template <int BQ>
__device__ inline bool find_tile(const int32_t *offset, int experts, int64_t rows, int p_tiles, int64_t block, Tile &t)
{
    const int lane = threadIdx.x & 63;
    auto range = [&](int e) {
        if (e < experts) return expert_rows(offset, e, rows);
        if (e == experts) return make_int2(min(max(offset[experts], 0), (int)rows), (int)rows);
        return make_int2(0, 0);
    };
    int tiles = 0;   // at most rows + experts + 1
    for (int e0 = 0; e0 <= experts; e0 += 64) {
        const int2 r = range(e0 + lane);
        tiles += (r.y - r.x + BQ - 1) / BQ;
    }
    tiles = __builtin_amdgcn_readfirstlane(wave_reduce(tiles, Sum()));
    const int64_t id = xcd_order(block, (int64_t)tiles * p_tiles);
    if (id < 0) return false;
    int64_t before = 0;
    for (int e0 = 0; e0 <= experts; e0 += 64) {
        const int2 r = range(e0 + lane);
        const int mine = (r.y - r.x + BQ - 1) / BQ;
        int sum = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(sum, d, 64);
            if (lane >= d) sum += o;
        }
        const uint64_t has = __ballot((before + sum) * p_tiles > id);
        if (has) {
            const int l = __ffsll((unsigned long long)has) - 1;
            const int lo = __builtin_amdgcn_readlane(r.x, l), hi = __builtin_amdgcn_readlane(r.y, l);
            const int64_t start = (before + __builtin_amdgcn_readlane(sum - mine, l)) * p_tiles;
            const int q_tiles = (hi - lo + BQ - 1) / BQ;
            const int local = (int)(id - start);
            t.expert = e0 + l;
            t.lo = lo;
            t.hi = hi;
            t.q = local % q_tiles;
            t.p = local / q_tiles;
            return true;
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}

// LDS places (in 16-byte units) of a tile along k, [128][64], and across k, [64][128].  Along: row pairs take turns at
// the eight places of a row, so 16 rows at one k lie in 16 different places of two rows' 256 bytes.  Across: rows k take
// turns at the pairs of places, for the transposing read of rows 0-3, 8-11, ... of a 16-element column.
__device__ inline int along_place(int i, int c) { return i * 8 + (c ^ ((i >> 1) & 7)); }
__device__ inline int across_place(int k, int c, int places)
{
    return k * places + (c ^ (((k & 3) | ((k >> 1) & 4)) << 1 & (places - 1)));
}

// The operand of a 16 x 16 x 32 product: row i0 + lane % 16, summands k0 + 8 (lane / 16) .. + 7.
template <bool ALONG>
__device__ inline s16x8 fragment(const u32x4 *lds, int i0, int k0, int lane, int places)
{
    if constexpr (ALONG) {
        return __builtin_bit_cast(s16x8, lds[along_place(i0 + (lane & 15), (k0 >> 3) + (lane >> 4))]);
    } else {
        // lane a of 16 gives the address of row a / 4 of four, elements 4 (a % 4) on, and takes column a of them
        const int k = k0 + (lane >> 4) * 8 + ((lane & 15) >> 2), c = (i0 >> 3) + ((lane & 3) >> 1);
        using Lds = __attribute__((address_space(3))) s16x4;
        const s16x4 *a = reinterpret_cast<const s16x4 *>(lds + across_place(k, c, places)) + (lane & 1);
        const s16x4 *b = reinterpret_cast<const s16x4 *>(lds + across_place(k + 4, c, places)) + (lane & 1);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds *)a);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds *)b);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
}

enum { kForward, kGradX, kGradW };

// the most tiles of b rows that `rows` rows of any split over the experts (and the rest) can have
int64_t most_row_tiles(int64_t rows, int experts, int b)
{
    const int64_t parts = rows < experts + 1 ? rows : experts + 1;
    return (rows - parts) / b + parts;
}

// All but this wave's last LOADS loads into LDS have landed, its LDS reads are done, and so for every wave.
template <int LOADS>
__device__ inline void sync_tiles()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS) : "memory");
}

// The results of a workgroup's waves to rows q0 .. q_end of out, columns p0 .. p_end.  LDS is read by now: it takes them,
// as many rows at a time as fit, and they leave it as whole rows of the tile.  A row's places are turned by its number,
// so that neither the 16 rows of a write nor a row's read meet in a bank.
// WHOLE: rows and columns begin and end on 16 bytes.
template <typename O, int BQ, int BP, int WQ, int WP, int SPACE, bool WHOLE = true>
__device__ inline void store_tile(u32x4 *lds, const f32x4 (&acc)[BQ / WQ / 16][BP / WP / 16], O *out, int64_t q0,
                                  int64_t q_end, int64_t p0, int64_t p_end)
{
    constexpr int kThreads = 64 * WQ * WP, kFq = BQ / WQ / 16, kFp = BP / WP / 16;
    constexpr int kOut = 16 / (int)sizeof(O);                 // results in 16 bytes
    constexpr int kRow = BP / kOut;                           // places of a row
    constexpr int kRounds = BQ * kRow <= SPACE ? 1 : 2;
    constexpr int kPart = kFq / kRounds * 16;                 // a wave's rows of a round
    static_assert(BQ / kRounds * kRow <= SPACE && kFq % kRounds == 0, "the results' LDS");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wp = (wave % WP) * (BP / WP);
    char *const bytes = reinterpret_cast<char *>(lds);
#pragma unroll
    for (int h = 0; h < kRounds; ++h) {
        sync_tiles<0>();
#pragma unroll
        for (int i = 0; i < kPart / 16; ++i) {
            const int r = wave / WP * kPart + 16 * i + (lane & 15);
#pragma unroll
            for (int j = 0; j < kFp; ++j) {
                const int c = wp + 16 * j + (lane >> 4) * 4;
                struct alignas(4 * sizeof(O)) Four {
                    O v[4];
                } f;
#pragma unroll
                for (int k = 0; k < 4; ++k) f.v[k] = from_f32<O>(acc[h * (kPart / 16) + i][j][k]);
                *reinterpret_cast<Four *>(bytes + (r * kRow + (c / kOut ^ (r & (kRow - 1)))) * 16 +
                                          c % kOut * (int)sizeof(O)) = f;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll 4
        for (int u = threadIdx.x; u < BQ / kRounds * kRow; u += kThreads) {
            const int r = u / kRow, c = u % kRow;
            const int64_t q = q0 + r / kPart * (BQ / WQ) + h * kPart + r % kPart, p = p0 + c * kOut;
            if (q >= q_end || p >= p_end) continue;
            const u32x4 x = lds[r * kRow + (c ^ (r & (kRow - 1)))];
            O *const to = out + q * p_end + p;
            if constexpr (WHOLE) {
                *reinterpret_cast<u32x4 *>(to) = x;
            } else if (p + kOut <= p_end) {
                __builtin_memcpy(to, &x, 16);
            } else {
                O v[kOut];
                __builtin_memcpy(v, &x, 16);
#pragma unroll
                for (int i = 0; i < kOut; ++i)
                    if (p + i < p_end) to[i] = v[i];
            }
        }
    }
}

// The rank-th expert by falling number of rows, in classes of a power of two: the long sums begin first and the short
// ones fill the gaps.  Every wave by itself, 64 experts a lane group.
__device__ inline int expert_of_rank(const int32_t *offset, int experts, int64_t rows, int rank)
{
    constexpr int kGroups = HAPMOE_MAX_EXPERTS / 64;
    const int lane = threadIdx.x & 63;
    int size[kGroups], top = -1;   // class of the expert, -1 without rows, -2 past the last
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        size[g] = -2;
        if (g * 64 >= experts) break;
        const int e = g * 64 + lane;
        if (e < experts) {
            const int2 r = expert_rows(offset, e, rows);
            size[g] = r.y > r.x ? 31 - __clz(r.y - r.x) : -1;
        }
        top = max(top, size[g]);
    }
    top = __builtin_amdgcn_readfirstlane(wave_reduce(top, Max()));
    for (int c = top; c >= -1; --c) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            if (g * 64 >= experts) break;
            uint64_t in = __ballot(size[g] == c);
            const int n = __popcll(in);
            if (rank < n) {
                for (; rank > 0; --rank) in &= in - 1;
                return g * 64 + __ffsll((unsigned long long)in) - 1;
            }
            rank -= n;
        }
    }
    return 0;   // not reached: rank < experts
}

// The tile of a workgroup of d_w: the experts by falling number of rows, each one's tiles spread over the XCDs.  False for
// one past an expert's tiles or past the last expert.
__device__ inline bool find_grad_w_tile(const int32_t *offset, int experts, int64_t rows, int p_tiles, int q_tiles,
                                        uint32_t block, Tile &t)
{
    const uint32_t tiles = (uint32_t)p_tiles * q_tiles, rounds = (tiles + 7) & ~7u;
    const int id = (int)xcd_order(block % rounds, tiles);
    if (id < 0) return false;
    if (block / rounds >= (uint32_t)experts) return false;
    t.expert = expert_of_rank(offset, experts, rows, (int)(block / rounds));
    t.q = id % q_tiles;
    t.p = id / q_tiles;
    const int2 r = expert_rows(offset, t.expert, rows);
    t.lo = __builtin_amdgcn_readfirstlane(r.x);
    t.hi = __builtin_amdgcn_readfirstlane(r.y);
    return true;
}
int64_t grad_w_grid(int64_t experts, int64_t p_tiles, int64_t q_tiles)
{
    const int64_t grid = experts * (ceil_div(p_tiles * q_tiles, 8) * 8);
    return p_tiles * q_tiles < 0x7ffffff0 ? grid : int64_t(1) << 40;
}

// ------------------------------------------------------------------ the kernel for any alignment
// Rows that begin anywhere, any number of columns and summands: 16-byte loads of any alignment into registers, from there
// into LDS.  B x B outputs a workgroup of four waves, 64 summands at a time, AHEAD tiles on their way: a tile's loads are
// some 2 us under way, which is what bounds a product with few tiles.
namespace any {

constexpr int kThreads = 256;

// n of the 8 elements at p, zeros for the others
__device__ inline u32x4 load_some(const char *p, int n)
{
    short s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = i < n ? reinterpret_cast<const short *>(p)[i] : 0;
    u32x4 x;
    __builtin_memcpy(&x, s, 16);
    return x;
}
// x without its first s elements, zeros behind them
__device__ inline u32x4 drop(u32x4 x, int s)
{
    uint64_t lo = (uint64_t)x[1] << 32 | x[0], hi = (uint64_t)x[3] << 32 | x[2];
    if (s >= 4) {
        lo = hi;
        hi = 0;
    }
    const int bits = (s & 3) * 16;
    if (bits) {
        lo = lo >> bits | hi << (64 - bits);
        hi >>= bits;
    }
    if (s >= 8) lo = hi = 0;
    return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// One operand's tiles, kLoads pieces of 8 elements a thread.  fetch() is the load alone, of eight elements that exist;
// fixed(), once it has landed, drops those before the piece and clears what does not exist.  SMALL: fewer than 8
// columns or summands, element by element.
template <bool ALONG, int SIDE, bool GATHER, bool SMALL>
struct Loader {
    static constexpr int kPlaces = ALONG ? 8 : SIDE / 8, kRows = kThreads / kPlaces, kLoads = SIDE / 32;
    const char *row[ALONG ? kLoads : 1];   // along: of each piece; across: the thread's column of row 0
    bool there[ALONG ? kLoads : 1];        // along: the row exists
    int slots[ALONG ? 1 : kLoads];         // gathered across: of the next tile
    const int32_t *slot;
    int64_t ld2;
    int first, shift, n, k_end, top_k, rows;

    __device__ void begin(const void *memory, int64_t ld, const int32_t *all_slots, int k, int64_t row0,
                          int64_t memory_rows, int64_t i0, int64_t i_end, int summands)
    {
        const auto *const bytes = static_cast<const char *>(memory);
        const int r = threadIdx.x / kPlaces, c = threadIdx.x % kPlaces;
        ld2 = ld * 2;
        k_end = summands;
        top_k = k;
        rows = (int)memory_rows;
        if constexpr (ALONG) {
            first = c * 8;
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int64_t i = min(i0 + j * kRows + r, i_end - 1) + row0;   // results past the last go nowhere
                int64_t from = i;
                there[j] = true;
                if constexpr (GATHER) {
                    const int s = all_slots[i];
                    there[j] = s >= 0 && s / top_k < rows;
                    from = there[j] ? s / top_k : 0;
                }
                row[j] = bytes + from * ld2;
            }
        } else {
            first = r;
            const int64_t i = i0 + c * 8, from = SMALL ? min(i, i_end - 1) : min(i, i_end - 8);
            n = (int)min((int64_t)8, max((int64_t)0, i_end - i));
            shift = (int)(i - from);
            row[0] = bytes + (GATHER ? 0 : row0 * ld2) + from * 2;
            slot = GATHER ? all_slots + row0 : nullptr;
            next_slots(0);
        }
    }
    __device__ void next_slots(int tile)
    {
        if constexpr (!ALONG && GATHER) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) slots[j] = slot[min(tile * 64 + first + j * kRows, k_end - 1)];
        }
    }
    // the loads of a tile, and what `fixed` has to know of gathered rows
    __device__ void fetch(int tile, u32x4 *x, uint32_t &have)
    {
        have = 0;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const char *p;
            int m = 8;
            if constexpr (ALONG) {
                const int k = tile * 64 + first;
                p = row[j] + (int64_t)(SMALL ? min(k, k_end - 1) : min(k, k_end - 8)) * 2;
                if constexpr (SMALL) m = k < k_end ? min(8, k_end - k) : 0;
                have |= (uint32_t)there[j] << j;
            } else {
                int k = min(tile * 64 + first + j * kRows, k_end - 1);
                bool ok = true;
                if constexpr (GATHER) {
                    ok = slots[j] >= 0 && slots[j] / top_k < rows;
                    k = ok ? slots[j] / top_k : 0;
                }
                p = row[0] + k * ld2;
                if constexpr (SMALL) m = n;
                have |= (uint32_t)ok << j;
            }
            if constexpr (SMALL)
                x[j] = load_some(p, m);
            else
                __builtin_memcpy(&x[j], p, 16);
        }
        next_slots(tile + 1);
    }
    __device__ void store(int tile, const u32x4 *x, uint32_t have, u32x4 *lds) const
    {
        const bool last = tile * 64 + 64 > k_end;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            u32x4 v = x[j];
            const int r = threadIdx.x / kPlaces + j * kRows, c = threadIdx.x % kPlaces;
            if constexpr (ALONG) {
                const int k = tile * 64 + first;
                if (!SMALL && last) v = drop(v, k - min(k, k_end - 8));
            } else {
                if (!SMALL && shift) v = drop(v, shift);
                if (last && tile * 64 + r >= k_end) v = u32x4{0, 0, 0, 0};
            }
            if (GATHER && !(have >> j & 1)) v = u32x4{0, 0, 0, 0};
            lds[ALONG ? along_place(r, c) : across_place(r, c, kPlaces)] = v;
        }
    }
};

template <int KIND, typename T, typename O, bool GATHER, bool SMALL, int B, int AHEAD>
__global__ __launch_bounds__(kThreads, 2) void k_product(const ExpertProduct a, int p_tiles, int q_tiles)
{
    constexpr bool kQAlong = KIND != kGradW, kPAlong = KIND == kForward;
    constexpr int kF = B / 32;   // a wave's fragments of each operand
    __shared__ u32x4 lds[2 * B * 8];
    u32x4 *const lds_q = lds, *const lds_p = lds + B * 8;
    Tile t;
    Loader<kQAlong, B, GATHER && KIND == kForward, SMALL> lq;
    Loader<kPAlong, B, GATHER && KIND == kGradW, SMALL> lp;
    int64_t q_end, p_end, out_row;
    int k_end;
    if constexpr (KIND == kGradW) {
        if (!find_grad_w_tile(a.offset, a.experts, a.rows, p_tiles, q_tiles, (uint32_t)workgroup(), t)) return;
        q_end = a.outputs;
        p_end = a.inputs;
        k_end = t.hi - t.lo;
        out_row = (int64_t)t.expert * a.outputs;
        if (k_end > 0) {
            lq.begin(a.d_y, a.d_y_stride, nullptr, 1, t.lo, a.rows, (int64_t)t.q * B, q_end, k_end);
            lp.begin(a.x, a.x_stride, a.slot, a.top_k, t.lo, a.x_rows, (int64_t)t.p * B, p_end, k_end);
        }
        if (GATHER && a.x_rows == 0) k_end = 0;
    } else {
        if (!find_tile<B>(a.offset, a.experts, a.rows, p_tiles, workgroup(), t)) return;
        q_end = t.hi - t.lo;
        p_end = KIND == kForward ? a.outputs : a.inputs;
        k_end = t.expert == a.experts ? 0 : KIND == kForward ? (int)a.inputs : (int)a.outputs;
        if (GATHER && a.x_rows == 0) k_end = 0;
        out_row = t.lo;
        if (k_end > 0) {
            const char *w = static_cast<const char *>(a.w) + t.expert * a.outputs * a.inputs * 2;
            lq.begin(KIND == kForward ? a.x : a.d_y, KIND == kForward ? a.x_stride : a.d_y_stride, a.slot, a.top_k, t.lo,
                     KIND == kForward ? a.x_rows : a.rows, (int64_t)t.q * B, q_end, k_end);
            lp.begin(w, a.inputs, nullptr, 1, 0, a.outputs, (int64_t)t.p * B, p_end, k_end);
        }
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wq = (wave >> 1) * (B / 2), wp = (wave & 1) * (B / 2);
    const int tiles = (k_end + 63) >> 6;
    f32x4 acc[kF][kF] = {};
    u32x4 xq[AHEAD][decltype(lq)::kLoads], xp[AHEAD][decltype(lp)::kLoads];
    uint32_t hq[AHEAD], hp[AHEAD];
#pragma unroll
    for (int d = 0; d < AHEAD; ++d)
        if (d < tiles) {
            lq.fetch(d, xq[d], hq[d]);
            lp.fetch(d, xp[d], hp[d]);
        }
    for (int t0 = 0; t0 < tiles; t0 += AHEAD) {
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
            const int tile = t0 + d;
            if (tile >= tiles) break;
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // the tile before is read
            lq.store(tile, xq[d], hq[d], lds_q);
            lp.store(tile, xp[d], hp[d], lds_p);
            if (tile + AHEAD < tiles) {
                lq.fetch(tile + AHEAD, xq[d], hq[d]);
                lp.fetch(tile + AHEAD, xp[d], hp[d]);
            }
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // this one is written
#pragma unroll
            for (int k = 0; k < 64; k += 32) {
                s16x8 fq[kF], fp[kF];
#pragma unroll
                for (int i = 0; i < kF; ++i) {
                    fq[i] = fragment<kQAlong>(lds_q, wq + 16 * i, k, lane, B / 8);
                    fp[i] = fragment<kPAlong>(lds_p, wp + 16 * i, k, lane, B / 8);
                }
#pragma unroll
                for (int i = 0; i < kF; ++i)
#pragma unroll
                    for (int j = 0; j < kF; ++j) acc[i][j] = mfma(fp[j], fq[i], acc[i][j], T());
            }
        }
    }
    store_tile<O, B, B, 2, 2, 2 * B * 8, false>(lds, acc, static_cast<O *>(a.out) + out_row * p_end, (int64_t)t.q * B, q_end,
                                                (int64_t)t.p * B, p_end);
}

template <int KIND, typename T, typename O, bool GATHER, bool SMALL, int B, int AHEAD>
hipError_t launch(const ExpertProduct &a, hipStream_t s)
{
    const int64_t p_tiles = ceil_div(KIND == kForward ? a.outputs : a.inputs, B), q_tiles = ceil_div(a.outputs, B);
    const int64_t tiles = KIND == kGradW ? grad_w_grid(a.experts, p_tiles, q_tiles)
                                         : most_row_tiles(a.rows, a.experts, B) * p_tiles;
    const int64_t grid = ceil_div(tiles, 8) * 8;   // whole rounds of the XCDs
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    hipLaunchKernelGGL((k_product<KIND, T, O, GATHER, SMALL, B, AHEAD>), many(grid), dim3(kThreads), 0, s, a,
                       (int)p_tiles, (int)q_tiles);
    return hipGetLastError();
}

template <int KIND, typename T, typename O, bool GATHER>
hipError_t by_size(const ExpertProduct &a, hipStream_t s)
{
    if (a.inputs < 8 || a.outputs < 8) return launch<KIND, T, O, GATHER, true, 64, 1>(a, s);
    const int64_t p_size = KIND == kForward ? a.outputs : a.inputs;
    // us by 64 x 64, by 128 x 128.  Few tiles, or few rows an expert, favour the smaller: 8 experts of 1,093 x 1,093, y: 1,024
    // rows (72 tiles) 18, 24; 64 experts, 4,096 rows (288 tiles) 39, 54.  At 512 tiles of 512 rows an expert the larger are
    // ahead (8 of 2,047 x 2,049: y 86, 55; d_x 100, 90; d_w of 552 tiles 25, 25), with 1,024 rows an expert by more: 175, 103;
    // 188, 136; 209, 147.
    const int64_t tiles = ceil_div(KIND == kGradW ? a.experts * a.outputs : a.rows, 128) * ceil_div(p_size, 128);
    if (tiles < 1024) return launch<KIND, T, O, GATHER, false, 64, 4>(a, s);
    return launch<KIND, T, O, GATHER, false, 128, 2>(a, s);
}

template <int KIND, typename T, typename O>
hipError_t product(const ExpertProduct &a, hipStream_t s)
{
    return a.slot && KIND != kGradX ? by_size<KIND, T, O, true>(a, s) : by_size<KIND, T, O, false>(a, s);
}

}  // namespace any

// ------------------------------------------------------------------ the kernel for whole vectors
// Rows and columns that begin on 16 bytes, columns and summands in eights.  The loads go from memory straight into LDS
// (16 bytes a lane, no registers), 64 summands at a time, while earlier tiles are multiplied.  What does not exist
// (rows past the expert's, summands past the end) is read from a page of zeros.
namespace fast {

__device__ u32x4 zeros[16];   // 256 bytes, never written

using Shared = __attribute__((address_space(3))) void;

// n / d for n < 2^31 by a multiplication
struct Divisor {
    uint32_t factor;
    int shift;
    __device__ int operator()(int n) const { return (int)(((uint64_t)(uint32_t)n * factor) >> shift); }
};
Divisor divisor(int d)
{
    int bits = 0;
    while ((int64_t(1) << bits) < d) ++bits;
    return Divisor{(uint32_t)(((uint64_t(1) << (31 + bits)) + d - 1) / d), 31 + bits};
}

struct Args {
    ExpertProduct a;
    Divisor by_top_k;
    int p_tiles, q_tiles;
};

// An address that is the same in all lanes, in scalar registers
__device__ inline const char *scalar(const char *p)
{
    const uint64_t x = reinterpret_cast<uint64_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    return reinterpret_cast<const char *>((uint64_t)hi << 32 | lo);
}

// 16 bytes a lane from memory to LDS at `to` (the wave's first lane; the others follow), counted by vmcnt alone: the
// caller waits for it, and the compiler, which would wait for it at the next LDS read, does not see it.  m0 is a
// register that the compiler keeps nothing in between instructions, and nothing else here uses it.
__device__ inline void load_to_lds(uint64_t from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "memory");
}
__device__ inline void load_to_lds(const char *base, uint32_t offset, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(scalar(base)), "s"(to)
                 : "memory");
}
// One operand's tiles: kLoads pieces of 16 bytes for each of THREADS threads.
// ALONG: SIDE rows of DEPTH summands.  Across: DEPTH summands of SIDE columns.
// Rows and columns past the last are read as the last, their results go nowhere; summands past the last are read as
// others of the row (the last tile's caller clears them).  Gathered rows have addresses of their own, and one that does
// not exist is read from the zeros; the others are 32-bit offsets from the tile's base, which moves on.
template <bool ALONG, int SIDE, int THREADS, bool GATHER, int DEPTH = 64>
struct Loader {
    static constexpr int kLoads = SIDE * DEPTH / 8 / THREADS;
    static constexpr int kPlaces = ALONG ? 8 : SIDE / 8;      // of a row in LDS
    static constexpr int kRows = THREADS / kPlaces;           // rows of LDS of one load of all threads
    static_assert(kLoads >= 1 && (ALONG ? DEPTH == 64 && kRows % 16 == 0 : kRows * kLoads == DEPTH), "whole tiles");
    const char *base;       // of the next tile
    uint32_t off[kLoads];   // of the pieces
    int64_t move;           // bytes from a tile to the next
    uint64_t at[kLoads];    // gathered along: the pieces of the next tile
    uint32_t step[kLoads];  // gathered along: bytes to the next tile's, 0 where there is no row
    int64_t ld2;            // bytes between rows
    // gathered across: a wave's piece is two rows, whose slots are scalars
    using Slots = __attribute__((address_space(4))) const int32_t;
    Slots *slot;            // of the expert's first row
    int next[kLoads][2];    // the slots of the next tile
    uint32_t column[kLoads];
    int first;              // summand of the first piece in the tile
    int k, k_end, rows;

    // i0: first row (along) or column (across), i_end: those that exist, at least one beyond i0; row0: added to the row
    // (along) or summand
    __device__ void begin(const void *memory, int64_t ld, const int32_t *slots, Divisor by, int64_t row0,
                          int64_t memory_rows, int64_t i0, int64_t i_end, int summands)
    {
        const int tid = threadIdx.x, r = tid / kPlaces;
        const auto *const bytes = static_cast<const char *>(memory);
        k = 0;
        k_end = summands;
        ld2 = ld * 2;
        rows = (int)memory_rows;
        const int left = (int)min((int64_t)SIDE, i_end - i0);   // rows or columns of the tile that exist
        if constexpr (ALONG) {
            first = ((tid & 7) ^ ((tid >> 4) & 7)) * 8;
            move = 128;
            base = scalar(bytes + (row0 + i0) * ld2);
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int i = min(j * kRows + r, left - 1);
                if constexpr (GATHER) {
                    const int s = slots[row0 + i0 + i], from = by(s);
                    const bool ok = s >= 0 && from < rows;
                    at[j] = ok ? reinterpret_cast<uint64_t>(bytes + from * ld2 + first * 2)
                               : reinterpret_cast<uint64_t>(zeros);
                    step[j] = ok ? 128 : 0;
                } else {
                    off[j] = (uint32_t)(i * ld2) + first * 2;
                }
            }
        } else {
            first = r;
            move = DEPTH * ld2;
            base = scalar(bytes + row0 * ld2 + i0 * 2);
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int k = j * kRows + r, place = across_place(k, tid % kPlaces, kPlaces) - k * kPlaces;
                const int column = min(place * 8, left - 8);
                if constexpr (GATHER)
                    this->column[j] = column * 2;
                else
                    off[j] = (uint32_t)(k * ld2) + column * 2;
            }
            if constexpr (GATHER) {
                static_assert(kPlaces == 32, "two rows a wave");
                base = scalar(bytes + i0 * 2);
                slot = (Slots *)(uintptr_t)scalar(reinterpret_cast<const char *>(slots + row0));
                fetch();
            }
        }
    }
    __device__ void fetch()
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                next[j][h] = slot[min(k + j * kRows + wave * 2 + h, k_end - 1)];
    }
    // Piece j of the next tile into LDS at `to`.  TAIL: the tile may end early.
    template <bool TAIL>
    __device__ void issue(int j, uint32_t to, Divisor by)
    {
        to += (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 1024 + j * THREADS * 16;
        if constexpr (GATHER && ALONG) {
            load_to_lds(TAIL && k + first >= k_end ? reinterpret_cast<uint64_t>(zeros) : at[j], to);
            at[j] += step[j];
        } else if constexpr (GATHER) {
            const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
            uint64_t row[2];
            uint32_t there[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = by(next[j][h]);
                const bool some = (next[j][h] >= 0) & (r < rows) & (!TAIL | (k + j * kRows + wave * 2 + h < k_end));
                const uint64_t ok = some ? ~uint64_t(0) : 0;
                row[h] = (reinterpret_cast<uint64_t>(base) + (uint64_t)(r * ld2)) & ok;
                row[h] |= reinterpret_cast<uint64_t>(zeros) & ~ok;
                there[h] = (uint32_t)ok;
            }
            const bool low = (threadIdx.x & 32) == 0;
            load_to_lds((low ? row[0] : row[1]) + (column[j] & (low ? there[0] : there[1])), to);
        } else if constexpr (TAIL) {
            const int mine = ALONG ? first : first + j * kRows;
            const int other = ALONG ? 0 : k_end - 1 - k;   // a summand of the tile that exists
            const uint32_t unit = ALONG ? 2 : (uint32_t)ld2;
            load_to_lds(base, k + mine < k_end ? off[j] : off[j] - (mine - other) * unit, to);
        } else {
            load_to_lds(base, off[j], to);
        }
    }
    __device__ void advance()
    {
        k += DEPTH;
        if constexpr (!ALONG && GATHER)
            fetch();
        else
            base += move;
    }
    // Zeros for the summands past `left` of the tile in LDS.
    __device__ static void clear(u32x4 *tile, int left)
    {
        for (int u = threadIdx.x; u < SIDE * DEPTH / 8; u += THREADS) {
            const int k = ALONG ? ((u & 7) ^ (u >> 4 & 7)) * 8 : u / kPlaces;
            if (k >= left) tile[u] = u32x4{0, 0, 0, 0};
        }
    }
};

// A wave's fragments of one half (32 summands) of a tile.
template <bool ALONG, int N>
struct Fragments {
    s16x8 f[N];
    __device__ void read(const u32x4 *tile, int i0, int k, int lane, int places)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = fragment<ALONG>(tile, i0 + 16 * i, k, lane, places);
    }
};

// BQ x BP outputs from row q0 of the tile's rows by a workgroup of WQ x WP waves.  STAGES tiles of 64 summands in LDS.
template <int KIND, typename T, typename O, bool GATHER, int BQ, int BP, int WQ, int WP, int STAGES>
__device__ inline void product_tile(const Args &args, const Tile &t, int64_t q0, u32x4 *lds)
{
    constexpr bool kQAlong = KIND != kGradW, kPAlong = KIND == kForward;
    constexpr int kThreads = 64 * WQ * WP;
    constexpr int kTileQ = BQ * 8, kTile = (BQ + BP) * 8;   // of LDS, in 16 bytes
    constexpr int kFq = BQ / WQ / 16, kFp = BP / WP / 16;    // a wave's fragments
    constexpr int kQPlaces = BQ / 8, kPPlaces = BP / 8;
    const ExpertProduct &a = args.a;
    Loader<kQAlong, BQ, kThreads, GATHER && KIND == kForward> lq;
    Loader<kPAlong, BP, kThreads, GATHER && KIND == kGradW> lp;
    int64_t q_end, p_end, out_row;
    int k_end;
    if constexpr (KIND == kGradW) {
        q_end = a.outputs;
        p_end = a.inputs;
        k_end = t.hi - t.lo;
        out_row = (int64_t)t.expert * a.outputs;
        if (k_end > 0) {
            lq.begin(a.d_y, a.d_y_stride, nullptr, args.by_top_k, t.lo, a.rows, q0, q_end, k_end);
            lp.begin(a.x, a.x_stride, a.slot, args.by_top_k, t.lo, a.x_rows, (int64_t)t.p * BP, p_end, k_end);
        }
    } else {
        q_end = t.hi - t.lo;
        p_end = KIND == kForward ? a.outputs : a.inputs;
        k_end = t.expert == a.experts ? 0 : KIND == kForward ? (int)a.inputs : (int)a.outputs;
        out_row = t.lo;
        if (k_end > 0) {
            const char *w = static_cast<const char *>(a.w) + t.expert * a.outputs * a.inputs * 2;
            lq.begin(KIND == kForward ? a.x : a.d_y, KIND == kForward ? a.x_stride : a.d_y_stride, a.slot,
                     args.by_top_k, t.lo, KIND == kForward ? a.x_rows : a.rows, q0, q_end, k_end);
            lp.begin(w, a.inputs, nullptr, args.by_top_k, 0, a.outputs, (int64_t)t.p * BP, p_end, k_end);
        }
    }
    constexpr int kLoadsQ = decltype(lq)::kLoads, kLoads = kLoadsQ + decltype(lp)::kLoads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wq = (wave / WP) * (BQ / WQ), wp = (wave % WP) * (BP / WP);
    const int tiles = (k_end + 63) >> 6, tail = k_end & 63;
    // The wave's fragments of rows that exist: the last tile of an expert multiplies no others.  2 % off 4,096 to 32,768
    // rows over 64 or 256 uneven experts; not in the largest tile, whose whole tiles the tests cost 1 to 5 %.
    constexpr bool kSkip = KIND != kGradW && BQ < 256;
    const int some = !kSkip ? kFq : __builtin_amdgcn_readfirstlane(
        (int)max((int64_t)0, min((int64_t)kFq, (q_end - q0 - wq + 15) / 16)));
    f32x4 acc[kFq][kFp] = {};
    const uint32_t lds0 = (uint32_t)(uintptr_t)(Shared *)lds;
    auto issue_one = [&](auto may_end, int j, int stage) {
        const uint32_t to = lds0 + stage * kTile * 16;
        if (j < kLoadsQ)
            lq.template issue<decltype(may_end)::value>(j, to, args.by_top_k);
        else
            lp.template issue<decltype(may_end)::value>(j - kLoadsQ, to + kTileQ * 16, args.by_top_k);
    };
    auto issue = [&](int stage) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) issue_one(std::true_type(), j, stage);
        lq.advance();
        lp.advance();
    };
    auto clear_tail = [&](int stage) {
        lq.clear(lds + stage * kTile, tail);
        lp.clear(lds + stage * kTile + kTileQ, tail);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    auto multiply = [&](const Fragments<kQAlong, kFq> &fq, const Fragments<kPAlong, kFp> &fp, int i) {
#pragma unroll
        for (int j = 0; j < kFp; ++j) acc[i][j] = mfma(fp.f[j], fq.f[i], acc[i][j], T());
    };
    if constexpr (STAGES == 2) {
        // Bound by the products.  Those of one half of a tile hide the LDS reads of the next half, and the loads of a
        // tile have the time of a whole one: once every wave has read a tile's second half, its LDS takes the tile
        // after the next.
        Fragments<kQAlong, kFq> q0f, q1f;
        Fragments<kPAlong, kFp> p0f, p1f;
        // the products of one half with the reads of the next among them, and with the loads of a tile (ISSUE 1; 2: it
        // may end early) among both
        auto half = [&](auto issue_mode, int into, const u32x4 *tile, int k, const Fragments<kQAlong, kFq> &fq,
                        const Fragments<kPAlong, kFp> &fp, Fragments<kQAlong, kFq> &nq, Fragments<kPAlong, kFp> &np) {
            constexpr int kMode = decltype(issue_mode)::value;
            constexpr int kReads = kFq + kFp;
#pragma unroll
            for (int i = 0; i < kFq; ++i) {
                if constexpr (kMode > 0) {
#pragma unroll
                    for (int j = i * kLoads / kFq; j < (i + 1) * kLoads / kFq; ++j)
                        issue_one(std::integral_constant<bool, kMode == 2>(), j, into);
                }
#pragma unroll
                for (int r = i * kReads / kFq; r < (i + 1) * kReads / kFq; ++r) {
                    if (r < kFp)
                        np.f[r] = fragment<kPAlong>(tile + kTileQ, wp + 16 * r, k, lane, kPPlaces);
                    else
                        nq.f[r - kFp] = fragment<kQAlong>(tile, wq + 16 * (r - kFp), k, lane, kQPlaces);
                }
                if (!kSkip || i < some) multiply(fq, fp, i);
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (kMode > 0) {
                lq.advance();
                lp.advance();
            }
        };
        int turn = 0;
        auto step = [&](auto issue_mode, bool last_is_next) {
            half(std::integral_constant<int, 0>(), 0, lds + turn * kTile, 32, q0f, p0f, q1f, p1f);
            sync_tiles<0>();
            if (last_is_next) clear_tail(turn ^ 1);
            half(issue_mode, turn, lds + (turn ^ 1) * kTile, 0, q1f, p1f, q0f, p0f);
            turn ^= 1;
        };
        if (tiles > 0) {
            issue(0);
            if (tiles > 1) {
                issue(1);
                sync_tiles<kLoads>();
            } else {
                sync_tiles<0>();
                if (tail) clear_tail(0);
            }
            p0f.read(lds + kTileQ, wp, 0, lane, kPPlaces);
            q0f.read(lds, wq, 0, lane, kQPlaces);
        }
        int i = 0;
        for (; i + 3 < tiles; ++i) step(std::integral_constant<int, 1>(), false);
        if (i + 2 < tiles) {
            step(std::integral_constant<int, 2>(), false);
            ++i;
        }
        for (; i < tiles; ++i) step(std::integral_constant<int, 0>(), tail != 0 && i + 2 == tiles);
    } else {
        // Bound by the loads of w: all tiles but one are under way.
        for (int i = 0; i < STAGES - 1 && i < tiles; ++i) issue(i);
        int stage = 0;
        for (int i = 0; i < tiles; ++i) {
            if (i + STAGES - 1 < tiles + 1)
                sync_tiles<(STAGES - 2) * kLoads>();
            else
                sync_tiles<0>();
            if (i + STAGES - 1 < tiles) issue(stage == 0 ? STAGES - 1 : stage - 1);
            if (tail && i + 1 == tiles) clear_tail(stage);
            const u32x4 *const tile = lds + stage * kTile;
            stage = stage == STAGES - 1 ? 0 : stage + 1;
#pragma unroll
            for (int k = 0; k < 64; k += 32) {
                Fragments<kQAlong, kFq> fq;
                Fragments<kPAlong, kFp> fp;
                fp.read(tile + kTileQ, wp, k, lane, kPPlaces);
                fq.read(tile, wq, k, lane, kQPlaces);
#pragma unroll
                for (int f = 0; f < kFq; ++f)
                    if (!kSkip || f < some) multiply(fq, fp, f);
            }
        }
    }
    store_tile<O, BQ, BP, WQ, WP, STAGES * kTile>(lds, acc, static_cast<O *>(a.out) + out_row * p_end, q0, q_end,
                                                  (int64_t)t.p * BP, p_end);
}

template <int KIND, typename T, typename O, bool GATHER, int BQ, int BP, int WQ, int WP, int STAGES>
__global__ __launch_bounds__(64 * WQ * WP) void k_product(const Args args)
{
    __shared__ u32x4 lds[STAGES * (BQ + BP) * 8];
    const ExpertProduct &a = args.a;
    Tile t;
    if constexpr (KIND == kGradW) {
        if (!find_grad_w_tile(a.offset, a.experts, a.rows, args.p_tiles, args.q_tiles, (uint32_t)workgroup(), t)) return;
    } else {
        if (!find_tile<BQ>(a.offset, a.experts, a.rows, args.p_tiles, workgroup(), t)) return;
    }
    const int64_t q0 = (int64_t)t.q * BQ;
    // an expert's last tile of up to half the rows is a tile of half the rows
    if constexpr (KIND != kGradW && BQ == 256) {
        if (t.hi - t.lo - q0 <= BQ / 2)
            return product_tile<KIND, T, O, GATHER, BQ / 2, BP, WQ, WP, STAGES>(args, t, q0, lds);
    }
    product_tile<KIND, T, O, GATHER, BQ, BP, WQ, WP, STAGES>(args, t, q0, lds);
}

// d_w: BQ x BP outputs of one expert a workgroup of four waves, 32 rows at a time, three tiles in LDS, two workgroups a
// CU: the one's LDS reads and results leave while the other multiplies.  A tile's loads have the time of two.
template <typename T, typename O, bool GATHER, int BQ, int BP>
__global__ __launch_bounds__(256, 2) void k_grad_w(const Args args)
{
    constexpr int kThreads = 256, kDepth = 32, kStages = 3, kWQ = 2, kWP = 2;
    constexpr int kTileQ = BQ * kDepth / 8, kTileP = BP * kDepth / 8;   // of LDS, in 16 bytes
    constexpr int kFq = BQ / kWQ / 16, kFp = BP / kWP / 16;
    __shared__ u32x4 lds[kStages * (kTileQ + kTileP)];
    const ExpertProduct &a = args.a;
    Tile t;
    if (!find_grad_w_tile(a.offset, a.experts, a.rows, args.p_tiles, args.q_tiles, (uint32_t)workgroup(), t)) return;
    const int64_t q0 = (int64_t)t.q * BQ, p0 = (int64_t)t.p * BP;
    const int k_end = t.hi - t.lo;
    Loader<false, BQ, kThreads, false, kDepth> lq;
    Loader<false, BP, kThreads, GATHER, kDepth> lp;
    constexpr int kLoadsQ = decltype(lq)::kLoads, kLoads = kLoadsQ + decltype(lp)::kLoads;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wq = wave / kWP * (BQ / kWQ), wp = wave % kWP * (BP / kWP);
    const int tiles = (k_end + kDepth - 1) / kDepth, tail = k_end % kDepth;
    f32x4 acc[kFq][kFp] = {};
    u32x4 *const lds_q = lds, *const lds_p = lds + kStages * kTileQ;
    const uint32_t to_q = (uint32_t)(uintptr_t)(Shared *)lds_q, to_p = (uint32_t)(uintptr_t)(Shared *)lds_p;
    auto issue_one = [&](auto may_end, int j, int stage) {
        if (j < kLoadsQ)
            lq.template issue<decltype(may_end)::value>(j, to_q + stage * kTileQ * 16, args.by_top_k);
        else
            lp.template issue<decltype(may_end)::value>(j - kLoadsQ, to_p + stage * kTileP * 16, args.by_top_k);
    };
    auto issue = [&](int stage) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) issue_one(std::true_type(), j, stage);
        lq.advance();
        lp.advance();
    };
    auto clear_tail = [&](int stage) {
        lq.clear(lds_q + stage * kTileQ, tail);
        lp.clear(lds_p + stage * kTileP, tail);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    if (tiles > 0) {
        lq.begin(a.d_y, a.d_y_stride, nullptr, args.by_top_k, t.lo, a.rows, q0, a.outputs, k_end);
        lp.begin(a.x, a.x_stride, a.slot, args.by_top_k, t.lo, a.x_rows, p0, a.inputs, k_end);
        issue(0);
        if (tiles > 1) issue(1);
    }
    // mode 0: none left to load, 1: a whole tile, 2: one that may end early
    auto step = [&](auto mode, int i, int stage) {
        constexpr int kMode = decltype(mode)::value;
        if (kMode > 0 || i + 1 < tiles)
            sync_tiles<kLoads>();
        else
            sync_tiles<0>();
        if (kMode == 0 && tail && i + 1 == tiles) clear_tail(stage);
        const int into = stage == 0 ? kStages - 1 : stage - 1;
        const u32x4 *const tq = lds_q + stage * kTileQ, *const tp = lds_p + stage * kTileP;
        Fragments<false, kFq> fq;
        Fragments<false, kFp> fp;
        fp.read(tp, wp, 0, lane, BP / 8);
        fq.f[0] = fragment<false>(tq, wq, 0, lane, BQ / 8);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int f = 0; f < kFq; ++f) {
            if constexpr (kMode > 0) {
#pragma unroll
                for (int j = f * kLoads / kFq; j < (f + 1) * kLoads / kFq; ++j)
                    issue_one(std::integral_constant<bool, kMode == 2>(), j, into);
            }
            if (f + 1 < kFq) fq.f[f + 1] = fragment<false>(tq, wq + 16 * (f + 1), 0, lane, BQ / 8);
#pragma unroll
            for (int j = 0; j < kFp; ++j) acc[f][j] = mfma(fp.f[j], fq.f[f], acc[f][j], T());
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (kMode > 0) {
            lq.advance();
            lp.advance();
        }
    };
    int i = 0, stage = 0;
    auto turn = [&] { stage = stage == kStages - 1 ? 0 : stage + 1; };
    for (; i + 3 < tiles; ++i, turn()) step(std::integral_constant<int, 1>(), i, stage);
    if (i + 2 < tiles) {
        step(std::integral_constant<int, 2>(), i, stage);
        ++i;
        turn();
    }
    for (; i < tiles; ++i, turn()) step(std::integral_constant<int, 0>(), i, stage);
    store_tile<O, BQ, BP, kWQ, kWP, kStages * (kTileQ + kTileP)>(
        lds, acc, static_cast<O *>(a.out) + t.expert * a.outputs * a.inputs, q0, a.outputs, p0, a.inputs);
}

template <int KIND, typename T, typename O, int BQ, int BP, int WQ, int WP, int STAGES>
hipError_t launch(const ExpertProduct &a, hipStream_t s)
{
    Args args;
    args.a = a;
    args.by_top_k = divisor(a.slot ? a.top_k : 1);
    args.p_tiles = (int)ceil_div(KIND == kForward ? a.outputs : a.inputs, BP);
    args.q_tiles = (int)ceil_div(a.outputs, BQ);
    const int64_t tiles = KIND == kGradW ? grad_w_grid(a.experts, args.p_tiles, args.q_tiles)
                                         : most_row_tiles(a.rows, a.experts, BQ) * args.p_tiles;
    const int64_t grid = ceil_div(tiles, 8) * 8;
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    constexpr int kThreads = 64 * WQ * WP;
    if (a.slot && KIND != kGradX)
        hipLaunchKernelGGL((k_product<KIND, T, O, true, BQ, BP, WQ, WP, STAGES>), many(grid), dim3(kThreads),
                           0, s, args);
    else
        hipLaunchKernelGGL((k_product<KIND, T, O, false, BQ, BP, WQ, WP, STAGES>), many(grid),
                           dim3(kThreads), 0, s, args);
    return hipGetLastError();
}

template <typename T, typename O, int BQ, int BP>
hipError_t launch_grad_w(const ExpertProduct &a, hipStream_t s)
{
    Args args;
    args.a = a;
    args.by_top_k = divisor(a.slot ? a.top_k : 1);
    args.p_tiles = (int)ceil_div(a.inputs, BP);
    args.q_tiles = (int)ceil_div(a.outputs, BQ);
    const int64_t grid = grad_w_grid(a.experts, args.p_tiles, args.q_tiles);
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    hipLaunchKernelGGL((a.slot ? k_grad_w<T, O, true, BQ, BP> : k_grad_w<T, O, false, BQ, BP>), many(grid),
                       dim3(256), 0, s, args);
    return hipGetLastError();
}

template <int KIND, typename T, typename O>
hipError_t product(const ExpertProduct &a, hipStream_t s)
{
    const int64_t some = a.rows / a.experts;   // rows an expert
    if constexpr (KIND == kGradW) {
        // Up to 128 tiles of 256 x 256 leave CUs idle: tiles of a quarter, two workgroups a CU.  8 experts of 512 x 2,048 with
        // 2,048 rows each: 45 us by 64 x 256, 47 by 128 x 256, 56 by 256 x 256, with uneven rows 78, 104, 126.  Many rows are
        // for the largest: 16 of 4,096 x 7,168 with 512 rows: 1,051, 831, 759 us.
        if (a.experts * a.outputs * a.inputs >> 16 <= 128) return launch_grad_w<T, O, 64, 256>(a, s);
        if (some < 512) return launch_grad_w<T, O, 128, 256>(a, s);
        return launch<KIND, T, O, 256, 256, 2, 4, 2>(a, s);
    } else {
        // Tiles by the rows of an expert, which fill them or not, and smaller ones where there are too few for 256 CUs.
        // us by 256 x 256, 128 x 128, 64 x 128: 8 experts of 512 x 2,048, rows 2,048: 39, 23, 18; 8,192: 40, 31, 38; 16,384:
        // 42, 52, 58; 16 of 4,096 x 7,168, rows 32,768: 1,648, 2,092, 2,950.  d_x of 64 experts of 2,048 x 4,096 with 160
        // rows each: 256 us by 256 x 256, 323 by 128 x 128, of 1,024 x 1,024 with uneven ones 53 and 43.  64 x 128 against
        // 128 x 128, 64 experts of 2,048 x 4,096, uneven rows, on average 32: y 195, 221, d_x 214, 216; 48: 210, 232, 229, 221;
        // 96: 255, 237, 270, 260.
        const int64_t large = a.rows * (KIND == kForward ? a.outputs : a.inputs) >> 16;   // tiles of 256 x 256
        if (some < 48 || large <= 32) return launch<KIND, T, O, 64, 128, 2, 2, 3>(a, s);
        if (some < (KIND == kGradX && large >= 256 ? 128 : 192) || large <= 80)
            return launch<KIND, T, O, 128, 128, 2, 2, 2>(a, s);
        return launch<KIND, T, O, 256, 256, 2, 4, 2>(a, s);
    }
}

}  // namespace fast

// whether whole vectors can be loaded and stored
bool whole_vectors(const ExpertProduct &a)
{
    constexpr int64_t kFar = int64_t(1) << 22;   // 256 rows this many elements long are within 32-bit offsets
    return a.inputs <= kFar && a.outputs <= kFar && a.x_stride <= kFar && a.d_y_stride <= kFar && a.outputs % 8 == 0 &&
           a.inputs % 8 == 0 && a.x_stride % 8 == 0 && a.d_y_stride % 8 == 0 && aligned(a.x, 16) && aligned(a.w, 16) &&
           aligned(a.d_y, 16) && aligned(a.out, 16);
}

template <int KIND, typename T, typename O>
hipError_t product(const ExpertProduct &a, hipStream_t s)
{
    return whole_vectors(a) ? fast::product<KIND, T, O>(a, s) : any::product<KIND, T, O>(a, s);
}

}  // namespace

hipError_t launch_expert_matmul(const ExpertProduct &a, hipStream_t s)
{
    return a.type == HAPMOE_BF16 ? product<kForward, bf16, bf16>(a, s) : product<kForward, f16, f16>(a, s);
}

hipError_t launch_expert_matmul_grad_x(const ExpertProduct &a, hipStream_t s)
{
    return a.type == HAPMOE_BF16 ? product<kGradX, bf16, bf16>(a, s) : product<kGradX, f16, f16>(a, s);
}

hipError_t launch_expert_matmul_grad_w(const ExpertProduct &a, hipStream_t s)
{
    if (a.type == HAPMOE_BF16)
        return a.out_type == HAPMOE_F32 ? product<kGradW, bf16, float>(a, s) : product<kGradW, bf16, bf16>(a, s);
    return a.out_type == HAPMOE_F32 ? product<kGradW, f16, float>(a, s) : product<kGradW, f16, f16>(a, s);
}

}  // namespace hapmoe
