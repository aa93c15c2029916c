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

// An operand as the kernels see it: element (i, k) of row i and summand k.  16-bit elements.
// ALONG: memory runs along k, row i at base + row(i) * ld.  Otherwise across it, summand k at base + row(k) * ld.
// row(): through slot (slot / top_k, none where that is past `rows`), or the number itself plus row0.
struct Operand {
    const short *base;
    const int32_t *slot;
    int64_t ld, row0;
    int64_t rows;      // rows of the memory that exist
    int top_k;
    __device__ const short *row(int64_t i, int64_t most_slots) const
    {
        i += row0;
        if (slot) {
            if (i >= most_slots) return nullptr;
            const int s = slot[i];
            i = s < 0 ? rows : s / top_k;
        }
        return i < rows ? base + i * ld : nullptr;
    }
};

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

// Tile `id` of the products whose rows are ragged: expert by expert, the column tiles one after another and for each the
// expert's row tiles, so that workgroups of neighbouring numbers share a column tile of the weights.  Every wave finds
// it by itself: 64 experts at a time, a scan over their tiles.  False past the last tile.
template <int BQ>
__device__ inline bool find_tile(const int32_t *offset, int experts, int64_t rows, int p_tiles, int64_t id, Tile &t)
{
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    for (int e0 = 0; e0 <= experts; e0 += 64) {
        const int e = e0 + lane;
        int2 r = make_int2(0, 0);
        if (e < experts)
            r = expert_rows(offset, e, rows);
        else if (e == experts)
            r = make_int2(min(max(offset[experts], 0), (int)rows), (int)rows);
        const int64_t mine = (int64_t)((r.y - r.x + BQ - 1) / BQ) * p_tiles;
        int64_t sum = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t o = __shfl_up(sum, d, 64);
            if (lane >= d) sum += o;
        }
        const uint64_t has = __ballot(before + sum > id);
        if (has) {
            const int l = __ffsll((unsigned long long)has) - 1;
            const int lo = __builtin_amdgcn_readlane(r.x, l), hi = __builtin_amdgcn_readlane(r.y, l);
            const int64_t start = before + __shfl(sum - mine, l, 64);
            const int q_tiles = (hi - lo + BQ - 1) / BQ;
            const int local = __builtin_amdgcn_readfirstlane((int)(id - start));
            t.expert = e0 + l;
            t.lo = lo;
            t.hi = hi;
            t.q = local % q_tiles;
            t.p = local / q_tiles;
            return true;
        }
        before += __shfl(sum, 63, 64);
    }
    return false;
}

// ------------------------------------------------------------------ the kernel for any alignment
// 128 x 128 outputs a workgroup of four waves (64 x 64 each), 64 summands at a time through registers into LDS.
constexpr int kThreads = 256;
constexpr int kB = 128;    // rows and columns
constexpr int kK = 64;     // summands

// 16 bytes from an address of any alignment, n of the 8 elements exist
__device__ inline u32x4 load8(const short *p, int n)
{
    u32x4 x = {0, 0, 0, 0};
    if (n >= 8) {
        __builtin_memcpy(&x, p, 16);
    } else if (n > 0) {
        short s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = i < n ? p[i] : 0;
        __builtin_memcpy(&x, s, 16);
    }
    return x;
}

// LDS places (in 16-byte units) of a tile along k, [128][64], and across k, [64][128].  Along: row pairs take turns at
// the eight places of a row, so 16 rows at one k lie in 16 different places of two rows' 256 bytes.  Across: rows k take
// turns at the pairs of places, for the transposing read of rows 0-3, 8-11, ... of a 16-element column.
__device__ inline int along_place(int i, int c) { return i * 8 + (c ^ ((i >> 1) & 7)); }
__device__ inline int across_place(int k, int c, int places) { return k * places + (c ^ (((k & 3) | ((k >> 1) & 4)) << 1)); }

template <bool ALONG>
struct Stage {
    u32x4 x[4];
    // the thread's four 16-byte pieces of the tile at row i0, summand k0 (i_end rows, k_end summands exist)
    __device__ void load(const Operand &o, int64_t i0, int64_t i_end, int64_t k0, int64_t k_end, int64_t most_slots)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int u = j * kThreads + threadIdx.x;
            if constexpr (ALONG) {
                const int64_t i = i0 + (u >> 3), k = k0 + (u & 7) * 8;
                const short *r = i < i_end ? o.row(i, most_slots) : nullptr;
                x[j] = r ? load8(r + k, (int)min((int64_t)8, k_end - k)) : u32x4{0, 0, 0, 0};
            } else {
                const int64_t k = k0 + (u >> 4), i = i0 + (u & 15) * 8;
                const short *r = k < k_end ? o.row(k, most_slots) : nullptr;
                x[j] = r ? load8(r + i, (int)min((int64_t)8, i_end - i)) : u32x4{0, 0, 0, 0};
            }
        }
    }
    __device__ void store(u32x4 *lds) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int u = j * kThreads + threadIdx.x;
            lds[ALONG ? along_place(u >> 3, u & 7) : across_place(u >> 4, u & 15, 16)] = x[j];
        }
    }
};

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

template <typename O>
__device__ inline void store_results(O *out, int n, f32x4 c)   // four neighbours, n of them exist
{
    struct Four {
        O v[4];
    };
    Four f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f.v[i] = from_f32<O>(c[i]);
    if (n >= 4) {
        __builtin_memcpy(out, &f, sizeof(f));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) out[i] = f.v[i];
    }
}

enum { kForward, kGradX, kGradW };

template <int KIND, typename T, typename O>
__global__ __launch_bounds__(kThreads) void k_product_any(const ExpertProduct a, int p_tiles, int q_tiles)
{
    constexpr bool kQAlong = KIND != kGradW, kPAlong = KIND == kForward;
    __shared__ u32x4 lds_q[kB * kK / 8], lds_p[kB * kK / 8];
    Tile t;
    Operand q, p;
    int64_t q_end, p_end, k_end;
    int64_t out_row;
    if constexpr (KIND == kGradW) {
        const int64_t id = blockIdx.x;
        t.expert = (int)(id / ((int64_t)p_tiles * q_tiles));
        const int local = (int)(id % ((int64_t)p_tiles * q_tiles));
        t.q = local % q_tiles;
        t.p = local / q_tiles;
        const int2 r = expert_rows(a.offset, t.expert, a.rows);
        q = Operand{static_cast<const short *>(a.d_y), nullptr, a.d_y_stride, r.x, a.rows, 1};
        p = Operand{static_cast<const short *>(a.x), a.slot, a.x_stride, r.x, a.x_rows, a.top_k};
        q_end = a.outputs;
        p_end = a.inputs;
        k_end = r.y - r.x;
        out_row = (int64_t)t.expert * a.outputs;
    } else {
        if (!find_tile<kB>(a.offset, a.experts, a.rows, p_tiles, blockIdx.x, t)) return;
        const int64_t ld = KIND == kForward ? a.x_stride : a.d_y_stride;
        q = Operand{static_cast<const short *>(KIND == kForward ? a.x : a.d_y), KIND == kForward ? a.slot : nullptr, ld,
                    t.lo, KIND == kForward ? a.x_rows : a.rows, a.top_k};
        const int64_t e = t.expert < a.experts ? t.expert : 0;
        p = Operand{static_cast<const short *>(a.w) + e * a.outputs * a.inputs, nullptr, a.inputs, 0, a.outputs, 1};
        q_end = t.hi - t.lo;
        p_end = KIND == kForward ? a.outputs : a.inputs;
        k_end = t.expert < a.experts ? (KIND == kForward ? a.inputs : a.outputs) : 0;
        out_row = t.lo;
    }
    const int64_t q0 = (int64_t)t.q * kB, p0 = (int64_t)t.p * kB;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wq = (wave >> 1) * 64, wp = (wave & 1) * 64;
    f32x4 acc[4][4] = {};
    Stage<kQAlong> sq;
    Stage<kPAlong> sp;
    if (k_end > 0) {
        sq.load(q, q0, q_end, 0, k_end, a.rows);
        sp.load(p, p0, p_end, 0, k_end, a.rows);
    }
    for (int64_t k0 = 0; k0 < k_end; k0 += kK) {
        __syncthreads();
        sq.store(lds_q);
        sp.store(lds_p);
        __syncthreads();
        if (k0 + kK < k_end) {
            sq.load(q, q0, q_end, k0 + kK, k_end, a.rows);
            sp.load(p, p0, p_end, k0 + kK, k_end, a.rows);
        }
#pragma unroll
        for (int k = 0; k < kK; k += 32) {
            s16x8 fq[4], fp[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                fq[i] = fragment<kQAlong>(lds_q, wq + 16 * i, k, lane, 16);
                fp[i] = fragment<kPAlong>(lds_p, wp + 16 * i, k, lane, 16);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = mfma(fp[j], fq[i], acc[i][j], T());
        }
    }
    O *out = static_cast<O *>(a.out);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t r = q0 + wq + 16 * i + (lane & 15);
        if (r >= q_end) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t c = p0 + wp + 16 * j + (lane >> 4) * 4;
            if (c < p_end) store_results(out + (out_row + r) * p_end + c, (int)min((int64_t)4, p_end - c), acc[i][j]);
        }
    }
}

// the most tiles of b rows that `rows` rows of any split over the experts (and the rest) can have
int64_t most_row_tiles(int64_t rows, int experts, int b)
{
    const int64_t parts = rows < experts + 1 ? rows : experts + 1;
    return (rows - parts) / b + parts;
}

template <int KIND, typename T, typename O>
hipError_t product_any(const ExpertProduct &a, hipStream_t s)
{
    const int64_t p_size = KIND == kForward ? a.outputs : a.inputs;
    const int64_t p_tiles = ceil_div(p_size, kB), q_tiles = ceil_div(a.outputs, kB);
    const int64_t grid = KIND == kGradW ? a.experts * p_tiles * q_tiles : most_row_tiles(a.rows, a.experts, kB) * p_tiles;
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    hipLaunchKernelGGL((k_product_any<KIND, T, O>), dim3((unsigned)grid), dim3(kThreads), 0, s, a, (int)p_tiles,
                       (int)q_tiles);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_expert_matmul(const ExpertProduct &a, hipStream_t s)
{
    return a.type == HAPMOE_BF16 ? product_any<kForward, bf16, bf16>(a, s) : product_any<kForward, f16, f16>(a, s);
}

hipError_t launch_expert_matmul_grad_x(const ExpertProduct &a, hipStream_t s)
{
    return a.type == HAPMOE_BF16 ? product_any<kGradX, bf16, bf16>(a, s) : product_any<kGradX, f16, f16>(a, s);
}

hipError_t launch_expert_matmul_grad_w(const ExpertProduct &a, hipStream_t s)
{
    if (a.type == HAPMOE_BF16)
        return a.out_type == HAPMOE_F32 ? product_any<kGradW, bf16, float>(a, s) : product_any<kGradW, bf16, bf16>(a, s);
    return a.out_type == HAPMOE_F32 ? product_any<kGradW, f16, float>(a, s) : product_any<kGradW, f16, f16>(a, s);
}

}  // namespace hapmoe
