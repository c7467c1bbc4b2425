// The global norm of many tensors, and their values scaled to a largest norm
// (part of ops.hip).
//
// Two passes: sums of squares in fp64 (fp32's squares overflow past 1.8e19; the
// products of two fp32 values are exact), one partial sum a workgroup, then
// every workgroup of the second pass adds up all partial sums, always in the
// same order, and scales.  Tensors are taken in chunks, dealt out to the
// workgroups; a launch's table of tensors is one of its arguments.
// What bounds it: bytes, the values read twice and written once.  138 million in
// fp32: 311 us (5.3 TB/s); 270 thousand in 49 tensors: two launches, 13 us.
#pragma once
#include "ops_device.h"

namespace ctc {
namespace ops {

constexpr int CLIP_CHUNK = 4096;                 // elements
constexpr int CLIP_GROUPS = 1024;                // of a launch: four a CU

// The tensor of chunk `c`, the last whose first chunk is not behind it: how
// many begin there or before, two for each lane.
static_assert(CLIP_TENSORS <= 128, "two a lane");
__device__ __forceinline__ int clip_find(const ClipTable &t, uint32_t c) {
    const int lane = threadIdx.x & 63;
    const uint64_t lo = __ballot(lane < t.n && t.first[lane] <= c);
    const uint64_t hi =
        t.n > 64 ? __ballot(64 + lane < t.n && t.first[64 + lane] <= c) : (uint64_t)0;
    return __builtin_amdgcn_readfirstlane(__popcll(lo) + __popcll(hi) - 1);
}
// f(elements of a chunk) for 16 bytes of each lane at a time; a whole chunk is
// under way at once.
template <typename T, typename F>
__device__ __forceinline__ void clip_chunk(const T *x, int n, F f) {
    constexpr int V = 16 / sizeof(T), U = CLIP_CHUNK / (256 * V);
    int i = threadIdx.x * V;
    if (n == CLIP_CHUNK) {
        Raw<T, V> r[U];
#pragma unroll
        for (int j = 0; j < U; j++) r[j].load(x + i + j * 256 * V);
#pragma unroll
        for (int j = 0; j < U; j++) {
            float v[V];
            r[j].values(v);
            f(std::integral_constant<int, V>(), i + j * 256 * V, v);
        }
        return;
    }
    for (; i + V <= n; i += 256 * V) {
        float v[V];
        load<T, V>(x + i, v);
        f(std::integral_constant<int, V>(), i, v);
    }
    // (the lane whose vector the end cuts)
    for (; i < n; i++) {
        float v[1] = {widen(x[i])};
        f(std::integral_constant<int, 1>(), i, v);
    }
}
__device__ __forceinline__ double clip_join(double v, double *lds) {
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

__global__ __launch_bounds__(256) void clip_squares(ClipTable t, double *part) {
    __shared__ double lds[4];
    double sum = 0;
    for (uint32_t c = blockIdx.x; c < t.first[t.n]; c += gridDim.x) {
        const int i = clip_find(t, c);
        const int64_t at = (int64_t)(c - t.first[i]) * CLIP_CHUNK;
        const int n = t.size[i] - at < CLIP_CHUNK ? (int)(t.size[i] - at) : CLIP_CHUNK;
        auto add = [&](auto w, int, const float *v) {
#pragma unroll
            for (int e = 0; e < decltype(w)::value; e++) {
                const double x = v[e];
                sum = __builtin_fma(x, x, sum);
            }
        };
        if (t.type[i] == F32) clip_chunk((const float *)t.x[i] + at, n, add);
        else if (t.type[i] == F16) clip_chunk((const _Float16 *)t.x[i] + at, n, add);
        else clip_chunk((const __bf16 *)t.x[i] + at, n, add);
    }
    sum = clip_join(sum, lds);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

__global__ __launch_bounds__(256) void clip_scale(ClipTable t, const double *part, int parts,
                                                  double max_norm, float *norm) {
    __shared__ double lds[4];
    double sum = 0;
    for (int i = threadIdx.x; i < parts; i += 256) sum += part[i];
    sum = __builtin_sqrt(clip_join(sum, lds));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)sum;
    // (a norm that is no number leaves everything as it is)
    const bool over = sum > max_norm && sum < __builtin_inf();
    // (in fp64: in fp32 the factor would cost a rounding of its own, and all its
    // bits below 2^-126, which norms past 2^126 max_norm reach)
    const double f = over ? max_norm / sum : 1.0;
    for (uint32_t c = blockIdx.x; c < t.first[t.n]; c += gridDim.x) {
        const int i = clip_find(t, c);
        if (!over && t.y[i] == t.x[i]) continue;
        const int64_t at = (int64_t)(c - t.first[i]) * CLIP_CHUNK;
        const int n = t.size[i] - at < CLIP_CHUNK ? (int)(t.size[i] - at) : CLIP_CHUNK;
        auto go = [&](auto tag) {
            typedef typename decltype(tag)::type T;
            T *y = (T *)t.y[i] + at;
            clip_chunk((const T *)t.x[i] + at, n, [&](auto w, int e, const float *v) {
                constexpr int V = decltype(w)::value;
                float o[V];
#pragma unroll
                for (int k = 0; k < V; k++) o[k] = (float)((double)v[k] * f);
                store<T, V>(y + e, o);
            });
        };
        if (t.type[i] == F32) go(Tag<float>());
        else if (t.type[i] == F16) go(Tag<_Float16>());
        else go(Tag<__bf16>());
    }
}

// ------------------------------------------------------------------- host

static uint32_t clip_chunks(const ClipTable &t) { return t.first[t.n]; }
int clip_parts(const ClipTable &t) {
    return clip_chunks(t) < CLIP_GROUPS ? (int)clip_chunks(t) : CLIP_GROUPS;
}
int64_t clip_chunks_of(int64_t size) { return (size + CLIP_CHUNK - 1) / CLIP_CHUNK; }
hipError_t launch_clip_squares(const ClipTable &t, double *part, hipStream_t st) {
    return clip_parts(t) ? start(clip_squares, dim3(clip_parts(t)), 256, st, t, part) : hipSuccess;
}
hipError_t launch_clip_scale(const ClipTable &t, const double *part, int parts, double max_norm,
                             float *norm, hipStream_t st) {
    const int groups = clip_parts(t);
    return start(clip_scale, dim3(groups ? groups : 1), 256, st, t, part, parts, max_norm, norm);
}

}  // namespace ops
}  // namespace ctc
