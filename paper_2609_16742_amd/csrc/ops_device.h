// Device helpers of the operators in ops.hip.
#pragma once
#include "ops.h"

#include <hip/hip_runtime.h>

#include <type_traits>

namespace ctc {
namespace ops {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef int i8v __attribute__((ext_vector_type(8)));

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float INF = __builtin_inff();

// One value of a 16-bit type as fp32, and back (to nearest, ties to even).
// The value is in a register of its own before it is narrowed, so a
// multiply-add in front is rounded to fp32 first (v_fma_mixlo_f16 would
// round once, and differently).
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(_Float16 v) { return (float)v; }
__device__ __forceinline__ float widen(__bf16 v) { return (float)v; }
template <typename T> __device__ __forceinline__ T narrow(float v) {
    if constexpr (sizeof(T) == 2) asm("" : "+v"(v));
    return (T)v;
}

// V consecutive elements at p, which need only be aligned like one element
// (global loads and stores of any width take any address of 4 or 2 bytes).
template <typename T, int V> struct Pack { T e[V]; };
template <typename T, int V>
__device__ __forceinline__ void load(const T *p, float (&v)[V]) {
    Pack<T, V> r;
    __builtin_memcpy(&r, p, sizeof r);
#pragma unroll
    for (int i = 0; i < V; i++) v[i] = widen(r.e[i]);
}
template <typename T, int V>
__device__ __forceinline__ void store(T *p, const float (&v)[V]) {
    Pack<T, V> r;
#pragma unroll
    for (int i = 0; i < V; i++) r.e[i] = narrow<T>(v[i]);
    __builtin_memcpy(p, &r, sizeof r);
}

// V elements kept as they stand in memory.  hold() hides where they came
// from: the compiler would keep the widened values instead, twice the
// registers for 16-bit types.
template <typename T, int V> struct Raw {
    typedef typename std::conditional<
        V * sizeof(T) == 16, u4,
        typename std::conditional<
            V * sizeof(T) == 8, u2,
            typename std::conditional<V * sizeof(T) == 4, uint32_t, uint16_t>::type>::type>::type
        Bits;
    Bits bits;
    __device__ __forceinline__ void load(const T *p) { __builtin_memcpy(&bits, p, sizeof bits); }
    __device__ __forceinline__ void values(float (&v)[V]) const {
        const Pack<T, V> q = __builtin_bit_cast(Pack<T, V>, bits);
#pragma unroll
        for (int i = 0; i < V; i++) v[i] = widen(q.e[i]);
    }
    __device__ __forceinline__ void hold() {
        if constexpr (V * sizeof(T) == 16) {
            uint32_t a = bits[0], b = bits[1], c = bits[2], d = bits[3];
            asm volatile("" : "+v"(a), "+v"(b), "+v"(c), "+v"(d));
            bits = u4{a, b, c, d};
        }
    }
};

// The larger of values, a NaN lost against a number (as single
// instructions: fmaxf first quiets its arguments).
__device__ __forceinline__ float vmax(float a, float b) {
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ float vmax3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float exp2_hw(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float exp_hw(float v) { return exp2_hw(v * LOG2E); }

template <typename F> __device__ __forceinline__ F wave_sum(F v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// ReLU lets NaN through.  (The hardware's reciprocal is good to one ulp.)
__device__ __forceinline__ float relu(float z) { return z < 0.f ? 0.f : z; }
__device__ __forceinline__ float sigmoid(float z) {
    return __builtin_amdgcn_rcpf(1.f + exp_hw(-z));
}
// act(z) of V values; `act` is the same for the whole launch, so the choice
// is one branch.
template <int V> __device__ __forceinline__ void act_of(int act, float (&z)[V]) {
    if (act == ACT_RELU) {
#pragma unroll
        for (int e = 0; e < V; e++) z[e] = relu(z[e]);
    } else if (act == ACT_SILU) {
#pragma unroll
        for (int e = 0; e < V; e++) z[e] *= sigmoid(z[e]);
    }
}
// d act(z) / dz in place of z
template <int V> __device__ __forceinline__ void act_grad(int act, float (&z)[V]) {
    if (act == ACT_RELU) {
#pragma unroll
        for (int e = 0; e < V; e++) z[e] = z[e] > 0.f ? 1.f : 0.f;
    } else if (act == ACT_SILU) {
#pragma unroll
        for (int e = 0; e < V; e++) {
            const float s = sigmoid(z[e]);
            z[e] = s * (1.f + z[e] * (1.f - s));
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; e++) z[e] = 1.f;
    }
}

// Workgroups numbered over two dimensions of a grid: along one a launch takes
// fewer than 2^32 threads.  (Those past the last have to leave.)
constexpr int64_t GRID_ROW = 1 << 20;
static dim3 grid_of(int64_t workgroups) {
    if (workgroups <= GRID_ROW) return dim3((unsigned)workgroups);
    return dim3((unsigned)GRID_ROW, (unsigned)((workgroups + GRID_ROW - 1) / GRID_ROW));
}
__device__ __forceinline__ uint32_t workgroup() {
    return blockIdx.y * (uint32_t)GRID_ROW + blockIdx.x;
}

template <typename K, typename... A>
static hipError_t start(K kernel, dim3 grid, int block, hipStream_t st, A... args) {
    hipLaunchKernelGGL(kernel, grid, dim3(block), 0, st, args...);
    return hipGetLastError();
}

template <typename T> struct Tag { typedef T type; };
// f(Tag<T>()) for the element type of `type`.
template <typename F> static hipError_t by_type(int type, F f) {
    if (type == F32) return f(Tag<float>());
    if (type == F16) return f(Tag<_Float16>());
    return f(Tag<__bf16>());
}

}  // namespace ops
}  // namespace ctc
