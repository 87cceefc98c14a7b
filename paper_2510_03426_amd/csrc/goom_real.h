// Real tensors of the layer operators: element types, loads and stores of 1 or 8 elements, operands of the matrix instructions.
#pragma once

#include <hip/hip_runtime.h>

#include "goom_internal.h"

namespace goom_layer {

typedef __bf16 bf16;
typedef _Float16 f16;
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x4 __attribute__((ext_vector_type(4)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

inline bool real_type(int type) { return type == GOOM_REAL_F32 || type == GOOM_REAL_BF16 || type == GOOM_REAL_F16; }
inline size_t real_bytes(int type) { return type == GOOM_REAL_F32 ? 4 : 2; }

// vectors of N elements in memory
template <typename T, int N> struct Vec { typedef T type __attribute__((ext_vector_type(N))); };

template <typename T, int N> __device__ inline void load_floats(const T *p, float (&x)[N])
{
    const typename Vec<T, N>::type v = *reinterpret_cast<const typename Vec<T, N>::type *>(p);
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = (float)v[i];
}

template <typename T, int N> __device__ inline void store_floats(T *p, const float (&x)[N])
{
    typename Vec<T, N>::type v;
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = (T)x[i];
    *reinterpret_cast<typename Vec<T, N>::type *>(p) = v;
}

// the same from addresses aligned to one element only (the hardware takes them, as one access)
template <typename T, int N> __device__ inline typename Vec<T, N>::type load_unaligned(const T *p)
{
    typedef typename Vec<T, N>::type V __attribute__((aligned(sizeof(T))));
    return *reinterpret_cast<const V *>(p);
}
template <typename T, int N> __device__ inline void load_floats_unaligned(const T *p, float (&x)[N])
{
    const typename Vec<T, N>::type v = load_unaligned<T, N>(p);
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = (float)v[i];
}
template <typename T, int N> __device__ inline void store_floats_unaligned(T *p, const float (&x)[N])
{
    typedef typename Vec<T, N>::type V __attribute__((aligned(sizeof(T))));
    typename Vec<T, N>::type v;
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = (T)x[i];
    *reinterpret_cast<V *>(p) = v;
}

// f(type tag) with the element type that `type` (GOOM_REAL_*) names
template <typename T> struct Tag { typedef T type; };
template <typename F> int with_type(int type, F f)
{
    switch (type) {
    case GOOM_REAL_F32: return f(Tag<float>());
    case GOOM_REAL_BF16: return f(Tag<bf16>());
    default: return f(Tag<f16>());
    }
}

// A grid of any number of workgroups in one order.  The hardware counts the threads along an axis in 32 bits: more go on along y, and
// the last workgroups may be beyond `blocks`.
inline dim3 grid_of(long long blocks, int threads)
{
    const long long most = 0xffffffffll / threads, rows = (blocks + most - 1) / most;
    return rows <= 1 ? dim3((unsigned)blocks) : dim3((unsigned)((blocks + rows - 1) / rows), (unsigned)rows);
}
__device__ inline long long block_of() { return blockIdx.y * (long long)gridDim.x + blockIdx.x; }

// entry checks that the layer operators share (goom_linear_attention.hip)
int enter(goom_ctx *ctx);
int check_workspace(goom_ctx *ctx, const void *ws, size_t given, size_t need);

} // namespace goom_layer
