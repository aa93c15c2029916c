// AdamW over many tensors, moments in fp32 or in 8 bits.  Bound by HBM: every
// operand is read once and written once.  The tensors' addresses travel in the
// kernel's arguments (up to kTensors a launch), so a step copies nothing to the
// device and may be captured.  So do the numbers of the step: a captured one
// replays with the lr, step and seed of its capture.
//
// Every operation is a single fp32 one, rounded to nearest (no contraction), in
// the order of the formula in the header.
//
// 537 M elements in 16 tensors, fp32 with a bf16 copy: 2,631 to 2,896 us by the
// card, 5.6 to 6.1 TB/s.  235 M, 8-bit moments, bf16 gradient and copy: 730 to 850 us
// (16 bytes an element, 4.4 to 5.1 TB/s), their values 300 us.  24 tensors of 3,413:
// 4.7 us, a launch.
#include "operators.h"

namespace hapmoe {
namespace {

constexpr int kThreads = 256;
constexpr int kRound = 4 * kThreads;   // elements of a workgroup at a time
// A call over more elements than this streams: 4 rounds a workgroup and non-temporal loads and stores, for nothing is
// read twice in a step and little of it stays in the last cache (256 MB) until the next.  268 M elements in fp32 with a bf16
// copy: 1,510 us without, 1,426 with (5.33 -> 5.65 TB/s); but 9.6 M (288 MB), step after step: 47 without, 58 with.
constexpr int64_t kStream = int64_t(1) << 24;
constexpr int rounds_of(bool stream) { return stream ? 4 : 1; }
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

template <typename B>
__device__ inline int entry_of(const B &b, uint32_t chunk)
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

// Four elements of a type, as words.
template <typename T>
using Words = uint32_t __attribute__((ext_vector_type(sizeof(T))));
template <bool STREAM, typename W>
__device__ inline W load(const W *p)
{
    return STREAM ? __builtin_nontemporal_load(p) : *p;
}
template <bool STREAM, typename W>
__device__ inline void store(W x, W *p)
{
    if constexpr (STREAM)
        __builtin_nontemporal_store(x, p);
    else
        *p = x;
}

// Four consecutive elements; n of them exist where the tensor ends or its vectors are not aligned (VEC false).
template <typename T, bool VEC, bool STREAM>
__device__ inline void load4(float *x, const void *p, int64_t i, int n)
{
    const T *q = static_cast<const T *>(p) + i;
    if constexpr (VEC) {
        struct Four {
            T v[4];
        };
        const Four f = __builtin_bit_cast(Four, load<STREAM>(reinterpret_cast<const Words<T> *>(q)));
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = to_f32(f.v[k]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = k < n ? to_f32(q[k]) : 0.0f;
    }
}
template <typename T, bool VEC, bool STREAM>
__device__ inline void store4(void *p, int64_t i, int n, const float *x)
{
    T *q = static_cast<T *>(p) + i;
    if constexpr (VEC) {
        struct Four {
            T v[4];
        };
        Four f;
#pragma unroll
        for (int k = 0; k < 4; ++k) f.v[k] = from_f32<T>(x[k]);
        store<STREAM>(__builtin_bit_cast(Words<T>, f), reinterpret_cast<Words<T> *>(q));
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < n) q[k] = from_f32<T>(x[k]);
    }
}
template <bool VEC, bool STREAM>
__device__ inline uint32_t load_codes(const void *p, int64_t i, int n)
{
    const uint8_t *q = static_cast<const uint8_t *>(p) + i;
    if constexpr (VEC) return load<STREAM>(reinterpret_cast<const uint32_t *>(q));
    uint32_t c = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) c |= k < n ? (uint32_t)q[k] << 8 * k : 0u;
    return c;
}
template <bool VEC, bool STREAM>
__device__ inline void store_codes(void *p, int64_t i, int n, uint32_t c)
{
    uint8_t *q = static_cast<uint8_t *>(p) + i;
    if constexpr (VEC) {
        store<STREAM>(c, reinterpret_cast<uint32_t *>(q));
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

template <typename G, typename C, int BITS, bool VEC, bool STREAM>
__device__ inline void update(const Batch &b, const Entry &t, int64_t i, int n)
{
    // with BITS 8 every lane of the wave takes part in the maxima, those past the end with zeros
    float p[4], g[4], m[4], v[4];
    if (n > 0) {
        load4<float, VEC, STREAM>(p, t.param, i, n);
        load4<G, VEC, STREAM>(g, t.grad, i, n);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) p[k] = g[k] = 0.0f;
    }
    if constexpr (BITS == 32) {
        load4<float, VEC, STREAM>(m, t.m, i, n);
        load4<float, VEC, STREAM>(v, t.v, i, n);
    } else {
        const uint32_t cm = n > 0 ? load_codes<VEC, STREAM>(t.m, i, n) : 0, cv = n > 0 ? load_codes<VEC, STREAM>(t.v, i, n) : 0;
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
        store4<float, VEC, STREAM>(t.param, i, n, p);
        if constexpr (sizeof(C) == 2) store4<C, VEC, STREAM>(t.copy, i, n, p);
    }
    if constexpr (BITS == 32) {
        store4<float, VEC, STREAM>(t.m, i, n, m);
        store4<float, VEC, STREAM>(t.v, i, n, v);
    } else {
        int em = 0, ev = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            em = k < n ? Max()(em, exponent_field(m[k])) : em;
            ev = k < n ? Max()(ev, exponent_field(v[k])) : ev;
        }
        // the largest exponents of the block
        em = Max()(Min()(wave_reduce(em, Max()), 254) - 127, -119) - 7;
        ev = Max()(Min()(wave_reduce(ev, Max()), 254) - 127, -111) - 15;
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
        store_codes<VEC, STREAM>(t.m, i, n, cm);
        store_codes<VEC, STREAM>(t.v, i, n, cv);
        if ((threadIdx.x & 63) == 0) {
            t.m_exp[i / kBlock] = (int8_t)em;
            t.v_exp[i / kBlock] = (int8_t)ev;
        }
    }
}

template <typename G, typename C, int BITS, bool STREAM>
__global__ __launch_bounds__(kThreads) void k_adamw(const Batch b)
{
    if (b.skip && *b.skip) return;
    constexpr int kRounds = rounds_of(STREAM);
    const uint32_t chunk = blockIdx.x;
    const Entry &t = b.t[entry_of(b, chunk)];
    const int64_t lo = (int64_t)(chunk - (t.chunk0 & 0x7fffffffu)) * kRounds * kRound;
    const bool vec = t.chunk0 >> 31 && lo + kRounds * kRound <= t.n;
#pragma unroll 2
    for (int r = 0; r < kRounds; ++r) {
        const int64_t i = lo + r * kRound + threadIdx.x * 4, left = t.n - i;
        if (vec)
            update<G, C, BITS, true, STREAM>(b, t, i, 4);
        else if (BITS == 8 || left > 0)
            update<G, C, BITS, false, STREAM>(b, t, i, left > 4 ? 4 : left < 0 ? 0 : (int)left);
    }
}

template <typename G, typename C>
void launch(const Batch &b, int bits, bool stream, hipStream_t s)
{
    auto *kernel = bits == 32 ? (stream ? k_adamw<G, C, 32, true> : k_adamw<G, C, 32, false>)
                              : (stream ? k_adamw<G, C, 8, true> : k_adamw<G, C, 8, false>);
    hipLaunchKernelGGL(kernel, dim3(b.chunks), dim3(kThreads), 0, s, b);
}
template <typename G>
void launch(const Batch &b, int copy_type, int bits, bool stream, hipStream_t s)   // copy_type F32: none
{
    if (copy_type == HAPMOE_F32)
        launch<G, float>(b, bits, stream, s);
    else if (copy_type == HAPMOE_BF16)
        launch<G, bf16>(b, bits, stream, s);
    else
        launch<G, f16>(b, bits, stream, s);
}

// Both moments of up to kTensors tensors as values, a wave a block of 256 elements at a time.
struct Moment {
    const uint8_t *m, *v;
    const int8_t *m_exp, *v_exp;
    void *out_m, *out_v;
    int64_t n;
    uint32_t chunk0;   // as in Entry
};
struct Moments {
    int32_t count;
    uint32_t chunks;
    Moment t[kTensors];
};
static_assert(sizeof(Moments) <= 4096, "kernel arguments");

template <int BIAS, typename T, bool VEC, bool STREAM>
__device__ inline void expand(const uint8_t *code, const int8_t *exp, void *out, int64_t i, int n)
{
    const uint32_t c = load_codes<VEC, STREAM>(code, i, n);
    const float scale = power_of_two(exp[i / kBlock]);
    float x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = decode<BIAS>(c >> 8 * k & 255) * scale;
    store4<T, VEC, STREAM>(out, i, n, x);
}

template <typename T, bool STREAM>
__global__ __launch_bounds__(kThreads) void k_moments(const Moments b)
{
    constexpr int kRounds = rounds_of(STREAM);
    const Moment &t = b.t[entry_of(b, blockIdx.x)];
    const int64_t lo = (int64_t)(blockIdx.x - (t.chunk0 & 0x7fffffffu)) * kRounds * kRound;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int64_t i = lo + r * kRound + threadIdx.x * 4, left = t.n - i;
        if (left <= 0) return;
        if (t.chunk0 >> 31 && left >= 4) {
            expand<7, T, true, STREAM>(t.m, t.m_exp, t.out_m, i, 4);
            expand<15, T, true, STREAM>(t.v, t.v_exp, t.out_v, i, 4);
        } else {
            expand<7, T, false, STREAM>(t.m, t.m_exp, t.out_m, i, left > 4 ? 4 : (int)left);
            expand<15, T, false, STREAM>(t.v, t.v_exp, t.out_v, i, left > 4 ? 4 : (int)left);
        }
    }
}

bool streams(const hapmoe_adamw_tensor *tensors, int n)
{
    int64_t total = 0;
    for (int i = 0; i < n; ++i) total += tensors[i].n;
    return total > kStream;
}

}  // namespace

hipError_t launch_adamw(const hapmoe_adamw_tensor *tensors, const void *const *grads, int n, const hapmoe_adamw_args &a,
                        hipStream_t s)
{
    Batch b;
    const bool stream = streams(tensors, n);
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
            const int64_t chunks = ceil_div(x.n, rounds_of(stream) * kRound);
            if (x.n == 0) continue;
            if (b.count && b.chunks + chunks > 0x7fffffff) break;
            Entry &t = b.t[b.count++];
            t.param = x.param;
            t.grad = grads[i];
            t.copy = x.copy;
            t.m = x.m;
            t.v = x.v;
            t.m_exp = x.m_exp;
            t.v_exp = x.v_exp;
            t.n = x.n;
            t.first = first;
            t.decay = x.weight_decay * (float)a.lr;
            const bool vec = aligned(x.param, 16) && aligned(grads[i], 4 * grad_bytes) && aligned(x.copy, 8) &&
                             aligned(x.m, a.state_bits == 32 ? 16 : 4) && aligned(x.v, a.state_bits == 32 ? 16 : 4);
            t.chunk0 = b.chunks | (vec ? 0x80000000u : 0);
            b.chunks += (uint32_t)chunks;
            first += ceil_div(x.n, kBlock) * kBlock;
            if (x.copy) copy_type = a.copy_type;
        }
        if (b.count == 0) break;
        if (a.grad_type == HAPMOE_F32)
            launch<float>(b, copy_type, a.state_bits, stream, s);
        else if (a.grad_type == HAPMOE_BF16)
            launch<bf16>(b, copy_type, a.state_bits, stream, s);
        else
            launch<f16>(b, copy_type, a.state_bits, stream, s);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

hipError_t launch_adamw_moments(const hapmoe_adamw_tensor *tensors, void *const *out_m, void *const *out_v, int n,
                                int out_type, hipStream_t s)
{
    Moments b;
    const bool stream = streams(tensors, n);
    for (int i = 0; i < n;) {
        b.count = 0;
        b.chunks = 0;
        for (; i < n && b.count < kTensors; ++i) {
            const hapmoe_adamw_tensor &x = tensors[i];
            if (x.n == 0) continue;
            const int64_t chunks = ceil_div(x.n, rounds_of(stream) * kRound), bytes = 4 * type_bytes(out_type);
            if (b.count && b.chunks + chunks > 0x7fffffff) break;
            const bool vec = aligned(x.m, 4) && aligned(x.v, 4) && aligned(out_m[i], bytes) && aligned(out_v[i], bytes);
            b.t[b.count++] = Moment{static_cast<const uint8_t *>(x.m), static_cast<const uint8_t *>(x.v), x.m_exp, x.v_exp,
                                    out_m[i], out_v[i], x.n, b.chunks | (vec ? 0x80000000u : 0)};
            b.chunks += (uint32_t)chunks;
        }
        if (b.count == 0) break;
        auto *kernel = out_type == HAPMOE_F32 ? (stream ? k_moments<float, true> : k_moments<float, false>)
                                              : (stream ? k_moments<bf16, true> : k_moments<bf16, false>);
        hipLaunchKernelGGL(kernel, dim3(b.chunks), dim3(kThreads), 0, s, b);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace hapmoe
