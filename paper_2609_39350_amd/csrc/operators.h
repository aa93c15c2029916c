// The operators' launchers and what their kernels share: element types, 16-byte
// vectors of them, reductions over 16 and 64 lanes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hapmoe.h"

namespace hapmoe {

using bf16 = __bf16;
using f16 = _Float16;

inline int64_t type_bytes(int type) { return type == HAPMOE_F32 ? 4 : 2; }
inline bool aligned(const void *p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

#ifdef __HIPCC__
// A launch's threads along one axis have to stay below 2^32, so many workgroups take two axes, here x and z; those of
// the last z that exceed n are the kernel's to leave out.
inline dim3 many(int64_t n, unsigned y = 1)
{
    constexpr int64_t kMost = int64_t(1) << 22;   // of up to 512 threads
    return n <= kMost ? dim3((unsigned)n, y) : dim3((unsigned)kMost, y, (unsigned)ceil_div(n, kMost));
}
__device__ inline int64_t workgroup() { return (int64_t)blockIdx.z * gridDim.x + blockIdx.x; }
#endif

hipError_t launch_route(const void *logits, int type, int64_t stride, int64_t tokens, int experts, int top_k,
                        const uint8_t *keep, bool renormalize, float *weight, int32_t *expert, int32_t *count,
                        int32_t *offset, int32_t *slot, int32_t *place, void *ws, hipStream_t s);
int64_t route_ws_bytes(int64_t tokens, int experts, int top_k);
hipError_t launch_route_backward(const void *logits, int type, int64_t stride, int64_t tokens, int experts, int top_k,
                                 const uint8_t *keep, bool renormalize, const int32_t *expert, const float *weight,
                                 const float *d_weight, void *d_logits, hipStream_t s);
hipError_t launch_combine(const void *y, int type, int64_t rows, int64_t tokens, int top_k, int64_t hidden,
                          const int32_t *place, const float *weight, void *out, hipStream_t s);
hipError_t launch_combine_backward(const void *d_out, const void *y, int type, int64_t tokens, int top_k,
                                   int64_t hidden, const int32_t *slot, const int32_t *place, const float *weight,
                                   void *d_y, float *d_weight, hipStream_t s);

// Products grouped by expert.  q: the operand whose rows are the output's, p the one whose rows are its columns.
struct ExpertProduct {
    const void *x;            // [x_rows][inputs], x_stride apart
    const void *w;            // [experts][outputs][inputs]
    const void *d_y;          // [rows][outputs], d_y_stride apart
    void *out;
    const int32_t *offset;    // [experts + 1]
    const int32_t *slot;      // [rows] or null
    int64_t x_rows, x_stride, d_y_stride, rows, outputs, inputs;
    int experts, top_k, type, out_type;
};
hipError_t launch_expert_matmul(const ExpertProduct &a, hipStream_t s);
hipError_t launch_expert_matmul_grad_x(const ExpertProduct &a, hipStream_t s);
hipError_t launch_expert_matmul_grad_w(const ExpertProduct &a, hipStream_t s);

hipError_t launch_adamw(const hapmoe_adamw_tensor *t, const void *const *grads, int n, const hapmoe_adamw_args &a,
                        hipStream_t s);
hipError_t launch_adamw_moments(const hapmoe_adamw_tensor *t, void *const *out_m, void *const *out_v, int n,
                                int out_type, hipStream_t s);

#ifdef __HIPCC__
// Eight elements, 16 bytes of a 16-bit type or 32 of fp32.
template <typename T>
struct alignas(sizeof(T) * 8) Vec8 {
    T v[8];
};

// Such a vector that nothing reads again soon: kept out of the caches' way.
template <typename T>
__device__ inline Vec8<T> load_once(const T *p)
{
    typedef uint32_t W __attribute__((ext_vector_type(2 * sizeof(T))));
    return __builtin_bit_cast(Vec8<T>, __builtin_nontemporal_load(reinterpret_cast<const W *>(p)));
}
template <typename T>
__device__ inline void store_once(T *p, const Vec8<T> &v)
{
    typedef uint32_t W __attribute__((ext_vector_type(2 * sizeof(T))));
    __builtin_nontemporal_store(__builtin_bit_cast(W, v), reinterpret_cast<W *>(p));
}

__device__ inline float to_f32(float x) { return x; }
__device__ inline float to_f32(bf16 x) { return (float)x; }
__device__ inline float to_f32(f16 x) { return (float)x; }
// to nearest even
template <typename T>
__device__ inline T from_f32(float x)
{
    return (T)x;
}

template <int CTRL>
__device__ inline int dpp(int x)
{
    return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true);   // every lane has a source: no old value
}
template <int CTRL>
__device__ inline float dpp(float x)
{
    return __builtin_bit_cast(float, dpp<CTRL>(__builtin_bit_cast(int, x)));
}

// Over the 16 lanes of a row, the result in each of them: rotations of the row by 8, 4, 2 and 1.
template <typename V, typename F>
__device__ inline V row_reduce(V v, F f)
{
    v = f(v, dpp<0x128>(v));
    v = f(v, dpp<0x124>(v));
    v = f(v, dpp<0x122>(v));
    return f(v, dpp<0x121>(v));
}
// Over the wave, the result in every lane.
template <typename V, typename F>
__device__ inline V wave_reduce(V v, F f)
{
    v = row_reduce(v, f);
    v = f(v, __shfl_xor(v, 16, 64));
    return f(v, __shfl_xor(v, 32, 64));
}
struct Max {
    __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
    __device__ int operator()(int a, int b) const { return a > b ? a : b; }
};
struct Min {
    __device__ int operator()(int a, int b) const { return a < b ? a : b; }
};
struct Sum {
    __device__ float operator()(float a, float b) const { return a + b; }
    __device__ int operator()(int a, int b) const { return a + b; }
};
#endif

}  // namespace hapmoe
