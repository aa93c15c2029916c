// AdamW over many tensors, moments in fp32 or in 8 bits.  Bound by HBM: every
// operand is read once and written once.  The tensors' addresses travel in the
// kernel's arguments (up to kTensors a launch), so a step copies nothing to the
// device and may be captured; a workgroup takes kChunk elements of one tensor.
//
// Every operation is a single fp32 one, rounded to nearest (no contraction), in
// the order of the formula in the header.
#include "operators.h"

namespace hapmoe {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;
constexpr int kBlock = 256;    // elements that share an exponent: four a lane of a wave
constexpr int kTensors = 40;

struct Entry {
    float *param;
    const void *grad;
    void *copy, *m, *v;
    int8_t *m_exp, *v_exp;
    int64_t n;
    int64_t first;      // index of the element 0 for the random bits, a multiple of kBlock
    float decay;        // lr * weight_decay
    uint32_t chunk0;    // first workgroup; bit 31: whole vectors are aligned
};

struct Batch {
    float beta1, rest1, beta2, rest2, eps, grad_scale, size, root;
    uint64_t seed;
    const int32_t *skip;
    int32_t count;
    uint32_t chunks;
    Entry t[kTensors];
};
static_assert(sizeof(Batch) <= 4096, "kernel arguments");

__device__ inline int entry_of(const Batch &b, uint32_t chunk)
{
    int lo = 0, hi = b.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((b.t[mid].chunk0 & 0x7fffffffu) <= chunk)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

// Four consecutive elements; n of them exist where the tensor ends or its vectors are not aligned (VEC false).
template <typename T, bool VEC>
__device__ inline void load4(float *x, const void *p, int64_t i, int n)
{
    const T *q = static_cast<const T *>(p) + i;
    if constexpr (VEC) {
        struct alignas(4 * sizeof(T)) Four {
            T v[4];
        };
        const Four f = *reinterpret_cast<const Four *>(q);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = to_f32(f.v[k]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = k < n ? to_f32(q[k]) : 0.0f;
    }
}
template <typename T, bool VEC>
__device__ inline void store4(void *p, int64_t i, int n, const float *x)
{
    T *q = static_cast<T *>(p) + i;
    if constexpr (VEC) {
        struct alignas(4 * sizeof(T)) Four {
            T v[4];
        };
        Four f;
#pragma unroll
        for (int k = 0; k < 4; ++k) f.v[k] = from_f32<T>(x[k]);
        *reinterpret_cast<Four *>(q) = f;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < n) q[k] = from_f32<T>(x[k]);
    }
}
template <bool VEC>
__device__ inline uint32_t load_codes(const void *p, int64_t i, int n)
{
    const uint8_t *q = static_cast<const uint8_t *>(p) + i;
    if constexpr (VEC) return *reinterpret_cast<const uint32_t *>(q);
    uint32_t c = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) c |= k < n ? (uint32_t)q[k] << 8 * k : 0u;
    return c;
}
template <bool VEC>
__device__ inline void store_codes(void *p, int64_t i, int n, uint32_t c)
{
    uint8_t *q = static_cast<uint8_t *>(p) + i;
    if constexpr (VEC) {
        *reinterpret_cast<uint32_t *>(q) = c;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < n) q[k] = (uint8_t)(c >> 8 * k);
    }
}

__device__ inline float power_of_two(int e) { return __builtin_bit_cast(float, (uint32_t)(127 + e) << 23); }

// The value of a code at scale 1: BIAS 7, sign and 4 exponent bits; BIAS 15, 5 exponent bits.
template <int BIAS>
__device__ inline float decode(uint32_t code)
{
    constexpr uint32_t kMark = BIAS == 7 ? 127 : 255;
    const uint32_t size = code & kMark;
    const float small = (float)size * power_of_two(-BIAS - 2);
    const float normal = __builtin_bit_cast(float, (size << 20) + ((uint32_t)(127 - BIAS) << 23));
    float v = size < 8 ? small : normal;
    v = size == kMark ? NAN : v;
    return BIAS == 7 && code > 127 ? -v : v;
}

// a >= 0 to the code below or above it: above with the probability of what is cut off, by 16 random bits.
template <int BIAS>
__device__ inline uint32_t encode(float a, uint32_t random)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, a);
    const uint32_t normal = ((b + (random << 4)) >> 20) - ((127 - BIAS) << 3);
    const uint32_t small = ((uint32_t)fminf(a * power_of_two(BIAS + 18), 1048576.0f) + random) >> 16;
    const uint32_t code = a < power_of_two(1 - BIAS) ? small : normal;
    return b >= 0x7f800000u ? (BIAS == 7 ? 127u : 255u) : code;
}

// 32 random bits for an element of a step: its index and the seed, mixed by odd multipliers and shifts.
__device__ inline uint32_t random32(uint64_t seed, uint64_t i)
{
    uint32_t h = (uint32_t)i * 0x9E3779B1u + (uint32_t)seed;
    h ^= (uint32_t)(i >> 32) * 0xC8B3A5D7u + (uint32_t)(seed >> 32);
    h = (h ^ h >> 16) * 0x6C5B7F4Du;
    h = (h ^ h >> 15) * 0xB1E5A92Bu;
    return h ^ h >> 16;
}

__device__ inline int exponent_field(float x) { return (int)(__builtin_bit_cast(uint32_t, x) >> 23 & 255); }

template <typename G, typename C, int BITS, bool VEC>
__device__ inline void update(const Batch &b, const Entry &t, int64_t i, int n)
{
    // with BITS 8 every lane of the wave takes part in the maxima, those past the end with zeros
    float p[4], g[4], m[4], v[4];
    if (n > 0) {
        load4<float, VEC>(p, t.param, i, n);
        load4<G, VEC>(g, t.grad, i, n);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) p[k] = g[k] = 0.0f;
    }
    if constexpr (BITS == 32) {
        load4<float, VEC>(m, t.m, i, n);
        load4<float, VEC>(v, t.v, i, n);
    } else {
        const uint32_t cm = n > 0 ? load_codes<VEC>(t.m, i, n) : 0, cv = n > 0 ? load_codes<VEC>(t.v, i, n) : 0;
        const int64_t block = n > 0 ? i / kBlock : 0;
        const float sm = power_of_two(t.m_exp[block]), sv = power_of_two(t.v_exp[block]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            m[k] = decode<7>(cm >> 8 * k & 255) * sm;
            v[k] = decode<15>(cv >> 8 * k & 255) * sv;
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float gk = g[k] * b.grad_scale;
        m[k] = m[k] * b.beta1 + gk * b.rest1;
        v[k] = v[k] * b.beta2 + gk * b.rest2 * gk;
        p[k] = p[k] - (m[k] * b.size / (sqrtf(v[k]) * b.root + b.eps) + t.decay * p[k]);
    }
    if (n > 0) {
        store4<float, VEC>(t.param, i, n, p);
        if constexpr (sizeof(C) == 2) store4<C, VEC>(t.copy, i, n, p);
    }
    if constexpr (BITS == 32) {
        store4<float, VEC>(t.m, i, n, m);
        store4<float, VEC>(t.v, i, n, v);
    } else {
        int em = 0, ev = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            em = k < n ? Max()(em, exponent_field(m[k])) : em;
            ev = k < n ? Max()(ev, exponent_field(v[k])) : ev;
        }
        // the largest exponents of the block, both in one reduction
        const int both = wave_reduce(em << 16, Max()), other = wave_reduce(ev, Max());
        em = Max()(Min()(both >> 16, 254) - 127, -119) - 7;
        ev = Max()(Min()(other, 254) - 127, -111) - 15;
        if (n <= 0) return;
        const float sm = power_of_two(-em), sv = power_of_two(-ev);
        uint32_t cm = 0, cv = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t r = random32(b.seed, (uint64_t)(t.first + i + k));
            uint32_t x = encode<7>(fabsf(m[k]) * sm, r & 0xffff);
            x |= m[k] < 0.0f ? 128u : 0u;
            cm |= x << 8 * k;
            x = encode<15>(v[k] * sv, r >> 16);
            x = v[k] > 0.0f && x == 0 ? 1u : x;
            cv |= x << 8 * k;
        }
        store_codes<VEC>(t.m, i, n, cm);
        store_codes<VEC>(t.v, i, n, cv);
        if ((threadIdx.x & 63) == 0) {
            t.m_exp[i / kBlock] = (int8_t)em;
            t.v_exp[i / kBlock] = (int8_t)ev;
        }
    }
}

template <typename G, typename C, int BITS>
__global__ __launch_bounds__(kThreads) void k_adamw(const Batch b)
{
    if (b.skip && *b.skip) return;
    const uint32_t chunk = blockIdx.x;
    const Entry &t = b.t[entry_of(b, chunk)];
    const int64_t lo = (int64_t)(chunk - (t.chunk0 & 0x7fffffffu)) * kChunk;
    const bool vec = t.chunk0 >> 31 && lo + kChunk <= t.n;
#pragma unroll 2
    for (int r = 0; r < kChunk / (4 * kThreads); ++r) {
        const int64_t i = lo + (int64_t)(r * kThreads + threadIdx.x) * 4;
        const int64_t left = t.n - i;
        if (vec)
            update<G, C, BITS, true>(b, t, i, 4);
        else if (BITS == 8 || left > 0)
            update<G, C, BITS, false>(b, t, i, left > 4 ? 4 : left < 0 ? 0 : (int)left);
    }
}

template <typename G, typename C>
void launch(const Batch &b, int bits, hipStream_t s)
{
    if (bits == 32)
        hipLaunchKernelGGL((k_adamw<G, C, 32>), dim3(b.chunks), dim3(kThreads), 0, s, b);
    else
        hipLaunchKernelGGL((k_adamw<G, C, 8>), dim3(b.chunks), dim3(kThreads), 0, s, b);
}
template <typename G>
void launch(const Batch &b, int copy_type, int bits, hipStream_t s)   // copy_type F32: none
{
    if (copy_type == HAPMOE_F32)
        launch<G, float>(b, bits, s);
    else if (copy_type == HAPMOE_BF16)
        launch<G, bf16>(b, bits, s);
    else
        launch<G, f16>(b, bits, s);
}

template <int BIAS, typename T>
__global__ __launch_bounds__(kThreads) void k_moment(const uint8_t *__restrict__ code, const int8_t *__restrict__ exp,
                                                     int64_t n, int vec, T *__restrict__ out)
{
    const int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 4;
    if (i >= n) return;
    const int left = n - i > 4 ? 4 : (int)(n - i);
    const float scale = power_of_two(exp[i / kBlock]);
    const bool whole = vec && left == 4;
    const uint32_t c = whole ? load_codes<true>(code, i, 4) : load_codes<false>(code, i, left);
    float x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = decode<BIAS>(c >> 8 * k & 255) * scale;
    if (whole)
        store4<T, true>(out, i, 4, x);
    else
        store4<T, false>(out, i, left, x);
}

}  // namespace

hipError_t launch_adamw(const hapmoe_adamw_tensor *tensors, int n, const hapmoe_adamw_args &a, hipStream_t s)
{
    Batch b;
    b.beta1 = (float)a.beta1;
    b.rest1 = (float)(1.0 - a.beta1);
    b.beta2 = (float)a.beta2;
    b.rest2 = (float)(1.0 - a.beta2);
    b.eps = (float)a.eps;
    b.grad_scale = (float)a.grad_scale;
    // the bias corrections in 64 bits, rounded once
    b.size = (float)(a.lr / (1.0 - __builtin_pow(a.beta1, (double)a.step)));
    b.root = (float)(1.0 / __builtin_sqrt(1.0 - __builtin_pow(a.beta2, (double)a.step)));
    b.seed = a.seed;
    b.skip = a.d_skip;
    const int64_t grad_bytes = type_bytes(a.grad_type);
    int64_t first = 0;
    for (int i = 0; i < n;) {
        b.count = 0;
        b.chunks = 0;
        int copy_type = HAPMOE_F32;
        for (; i < n && b.count < kTensors; ++i) {
            const hapmoe_adamw_tensor &x = tensors[i];
            const int64_t chunks = ceil_div(x.n, kChunk);
            if (x.n == 0) continue;
            if (b.count && b.chunks + chunks > 0x7fffffff) break;
            Entry &t = b.t[b.count++];
            t.param = x.param;
            t.grad = x.grad;
            t.copy = x.copy;
            t.m = x.m;
            t.v = x.v;
            t.m_exp = x.m_exp;
            t.v_exp = x.v_exp;
            t.n = x.n;
            t.first = first;
            t.decay = x.weight_decay * (float)a.lr;
            const bool vec = aligned(x.param, 16) && aligned(x.grad, 4 * grad_bytes) && aligned(x.copy, 8) &&
                             aligned(x.m, a.state_bits == 32 ? 16 : 4) && aligned(x.v, a.state_bits == 32 ? 16 : 4);
            t.chunk0 = b.chunks | (vec ? 0x80000000u : 0);
            b.chunks += (uint32_t)chunks;
            first += ceil_div(x.n, kBlock) * kBlock;
            if (x.copy) copy_type = a.copy_type;
        }
        if (b.count == 0) break;
        if (a.grad_type == HAPMOE_F32)
            launch<float>(b, copy_type, a.state_bits, s);
        else if (a.grad_type == HAPMOE_BF16)
            launch<bf16>(b, copy_type, a.state_bits, s);
        else
            launch<f16>(b, copy_type, a.state_bits, s);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

hipError_t launch_adamw_moment(const uint8_t *code, const int8_t *exp, int64_t n, bool second, int out_type, void *out,
                               hipStream_t s)
{
    const unsigned grid = (unsigned)ceil_div(n, 4 * kThreads);
    const int vec = aligned(code, 4) && aligned(out, 4 * type_bytes(out_type));
    if (out_type == HAPMOE_F32)
        hipLaunchKernelGGL((second ? k_moment<15, float> : k_moment<7, float>), dim3(grid), dim3(kThreads), 0, s, code,
                           exp, n, vec, static_cast<float *>(out));
    else
        hipLaunchKernelGGL((second ? k_moment<15, bf16> : k_moment<7, bf16>), dim3(grid), dim3(kThreads), 0, s, code,
                           exp, n, vec, static_cast<bf16 *>(out));
    return hipGetLastError();
}

}  // namespace hapmoe
