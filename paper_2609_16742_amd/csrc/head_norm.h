// RMS norm of each head of queries and keys with the rotation by their
// positions in the same pass, and its gradients (part of ops.hip).
//
//   z = x / sqrt(mean x^2 + eps) w,   (y_a, y_b) = R(angle) (z_a, z_b)
//
// for the pairs (a, b) of a head, angle = position on the pair's axis times
// the pair's frequency.  What bounds both passes is bytes.  A workgroup takes
// some tokens with all their heads, so an angle's sine and cosine, in turns
// reduced in fp64, are computed once a token and kept in LDS.  (A position times
// a frequency has up to 55 bits, fp64 53: of a product below 2^29 that and the
// roundings of the turns leave an angle good to 2^-21.)  L lanes hold a head, V
// pairs each, and the norm's sum is an exchange between them.
// 2 x 6272 tokens, 40 heads of 128, bf16: 46 us (5.6 TB/s), gradients 82 (4.7).
#pragma once
#include "ops_device.h"

namespace ctc {
namespace ops {

// Pairs p, p + 1, .. of V: where their first and second values stand in a head
// of `half` pairs, the first `turned` of which are rotated.
//   halves: turned values a, then turned values b; then the rest likewise
template <int V, bool INTER> struct HeadPairs {
    int a, b;
    __device__ __forceinline__ HeadPairs(int p, int turned, int half) {
        if (INTER) {
            a = b = 2 * p;
        } else {
            a = p < turned ? p : p + turned;
            b = a + (p < turned ? turned : half - turned);
        }
    }
    template <typename T>
    __device__ __forceinline__ void load(const T *x, float (&u)[V], float (&v)[V]) const {
        if constexpr (INTER) {
            float t[2 * V];
            ops::load<T, 2 * V>(x + a, t);
#pragma unroll
            for (int i = 0; i < V; i++) u[i] = t[2 * i], v[i] = t[2 * i + 1];
        } else {
            ops::load<T, V>(x + a, u);
            ops::load<T, V>(x + b, v);
        }
    }
    template <typename T>
    __device__ __forceinline__ void store(T *x, const float (&u)[V], const float (&v)[V]) const {
        if constexpr (INTER) {
            float t[2 * V];
#pragma unroll
            for (int i = 0; i < V; i++) t[2 * i] = u[i], t[2 * i + 1] = v[i];
            ops::store<T, 2 * V>(x + a, t);
        } else {
            ops::store<T, V>(x + a, u);
            ops::store<T, V>(x + b, v);
        }
    }
};

constexpr int HEAD_TOKENS = 16;

__device__ __forceinline__ void head_angles(const HeadArgs &a, int64_t token0, int n,
                                            float2 *table) {
    const int half = a.d / 2;
    for (int i = threadIdx.x; i < n * half; i += 256) {
        const int p = i % half;
        const int64_t token = token0 + i / half;
        float s = 0.f, c = 1.f;
        if (p < a.turned) {
            int axis = 0, end = a.axes[0];
            while (p >= end) end += a.axes[++axis];
            const int64_t row = a.per_image ? token : token % a.t;
            const int pos = a.positions[row * a.n_axes + axis];
            double turns = (double)pos * (double)a.frequencies[p] * 0.15915494309189533577;
            turns -= __builtin_rint(turns);
            sincospif(2.f * (float)turns, &s, &c);
        }
        table[i] = float2{c, s};
    }
}

// The sum over the L lanes of a head.
__device__ __forceinline__ float head_sum(float v, int L) {
    for (int o = L >> 1; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// 1 / sqrt(mean x^2 + eps) of a head.  Where the mean is infinite or has lost
// bits in fp32 (values past 2^59 or so, or far below 1 with an eps as small), the
// values are multiplied by a power of two `t` first, and the result is 1 / t of
// theirs: their product is the normed value all the same.  `scaled` if a head of
// the wave is; elsewhere one comparison is all that this costs.
struct HeadRoot {
    float r, t = 1.f;
    bool scaled;
    template <int V>
    __device__ __forceinline__ HeadRoot(float (&u)[V], float (&v)[V], int L, int d, float eps) {
        const float m = mean(u, v, L, d) + eps;
        r = 1.f / sqrtf(m);
        scaled = __any(!(m < INF && m > 0x1p-100f));
        if (!scaled) return;
        if (!(m < INF)) t = 0x1p-80f;
        else if (!(m > 0x1p-100f)) t = 0x1p110f;
#pragma unroll
        for (int i = 0; i < V; i++) u[i] *= t, v[i] *= t;
        r = 1.f / sqrtf(mean(u, v, L, d) + eps * t * t);
    }
    template <int V>
    static __device__ __forceinline__ float mean(const float (&u)[V], const float (&v)[V], int L,
                                                 int d) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < V; i++) sum += u[i] * u[i] + v[i] * v[i];
        return head_sum(sum, L) / d;
    }
};

template <typename T, typename U, int V, bool INTER>
__global__ __launch_bounds__(256) void head_norm_forward(HeadArgs a) {
    extern __shared__ float2 table[];            // [tokens][half]: cosine, sine
    const int half = a.d / 2, L = a.lanes, sub = threadIdx.x / L, p = threadIdx.x % L * V;
    const int64_t token0 = (int64_t)workgroup() * a.tokens, all = (int64_t)a.b * a.t;
    if (token0 >= all) return;
    const int n = all - token0 < a.tokens ? (int)(all - token0) : a.tokens;
    if (a.turned) head_angles(a, token0, n, table);
    __syncthreads();
    const HeadPairs<V, INTER> at(p, a.turned, half);
    const bool mine = p < half, turn = mine && p < a.turned;
    for (int which = 0; which < 2; which++) {
        const HeadSide &s = a.side[which];
        if (!s.heads) continue;
        float wu[V], wv[V];
#pragma unroll
        for (int i = 0; i < V; i++) wu[i] = wv[i] = 1.f;
        if (s.weight && mine) at.load(s.weight, wu, wv);
        for (int unit = sub; unit < n * s.heads; unit += 256 / L) {
            const int k = unit / s.heads, head = unit - k * s.heads;
            const int64_t token = token0 + k, b = token / a.t, t = token - b * a.t;
            float u[V], v[V];
#pragma unroll
            for (int i = 0; i < V; i++) u[i] = v[i] = 0.f;
            if (mine)
                at.load((const T *)s.x + b * s.xs[0] + t * s.xs[1] + head * s.xs[2], u, v);
            if (a.norm) {
                const HeadRoot root(u, v, L, a.d, a.eps);
#pragma unroll
                for (int i = 0; i < V; i++) u[i] *= root.r, v[i] *= root.r;
            }
#pragma unroll
            for (int i = 0; i < V; i++) u[i] *= wu[i], v[i] *= wv[i];
            if (turn) {
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const float2 cs = table[k * half + p + i];
                    const float x = u[i] * cs.x - v[i] * cs.y;
                    v[i] = u[i] * cs.y + v[i] * cs.x;
                    u[i] = x;
                }
            }
            if (mine) at.store((U *)s.y + b * s.ys[0] + t * s.ys[1] + head * s.ys[2], u, v);
        }
    }
}

// Gradients: dz = R^T dy, dw = sum dz xhat, dx = r (dz w - xhat mean(dz w xhat)).
// A workgroup goes through groups of tokens; its sums over them (fp32 a lane)
// are joined in LDS and written as partial sums, which head_norm_join adds up
// in fp64, always in the same order.
template <typename T, typename U, int V, bool INTER>
__global__ __launch_bounds__(256) void head_norm_backward(HeadArgs a) {
    extern __shared__ float2 table[];
    const int half = a.d / 2, L = a.lanes, sub = threadIdx.x / L, p = threadIdx.x % L * V;
    const int64_t all = (int64_t)a.b * a.t;
    const HeadPairs<V, INTER> at(p, a.turned, half);
    const bool mine = p < half, turn = mine && p < a.turned;
    // (one side after the other: the sums of both would halve the waves)
#pragma unroll 1
    for (int which = 0; which < 2; which++) {
        const HeadSide &s = a.side[which];
        if (!s.heads) continue;
        float gu[V], gv[V], wu[V], wv[V];
#pragma unroll
        for (int i = 0; i < V; i++) {
            gu[i] = gv[i] = 0.f;
            wu[i] = wv[i] = 1.f;
        }
        if (s.weight && mine) at.load(s.weight, wu, wv);
        for (int64_t token0 = (int64_t)blockIdx.x * a.tokens; token0 < all;
             token0 += (int64_t)gridDim.x * a.tokens) {
            const int n = all - token0 < a.tokens ? (int)(all - token0) : a.tokens;
            __syncthreads();
            if (a.turned) head_angles(a, token0, n, table);
            __syncthreads();
            for (int unit = sub; unit < n * s.heads; unit += 256 / L) {
                const int k = unit / s.heads, head = unit - k * s.heads;
                const int64_t token = token0 + k, b = token / a.t, t = token - b * a.t;
                float u[V], v[V], xu[V], xv[V];
#pragma unroll
                for (int i = 0; i < V; i++) u[i] = v[i] = xu[i] = xv[i] = 0.f;
                if (mine) {
                    at.load((const U *)s.dy + b * s.dys[0] + t * s.dys[1] + head * s.dys[2], u, v);
                    at.load((const T *)s.x + b * s.xs[0] + t * s.xs[1] + head * s.xs[2], xu, xv);
                }
                if (turn) {
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        const float2 cs = table[k * half + p + i];
                        const float x = u[i] * cs.x + v[i] * cs.y;
                        v[i] = v[i] * cs.x - u[i] * cs.y;
                        u[i] = x;
                    }
                }
                float r = 1.f, lift = 1.f;
                bool scaled = false;
                if (a.norm) {
                    const HeadRoot root(xu, xv, L, a.d, a.eps);
                    r = root.r;
                    lift = root.t;
                    scaled = root.scaled;
#pragma unroll
                    for (int i = 0; i < V; i++) xu[i] *= r, xv[i] *= r;
                }
                float dot = 0.f;
#pragma unroll
                for (int i = 0; i < V; i++) {
                    gu[i] += u[i] * xu[i];
                    gv[i] += v[i] * xv[i];
                    u[i] *= wu[i];
                    v[i] *= wv[i];
                    dot += u[i] * xu[i] + v[i] * xv[i];
                }
                if (a.norm) {
                    dot = head_sum(dot, L) / a.d;
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        u[i] = r * (u[i] - xu[i] * dot);
                        v[i] = r * (v[i] - xv[i] * dot);
                    }
                    if (scaled) {
#pragma unroll
                        for (int i = 0; i < V; i++) u[i] *= lift, v[i] *= lift;
                    }
                }
                if (mine) at.store((T *)s.dx + b * s.dxs[0] + t * s.dxs[1] + head * s.dxs[2], u, v);
            }
        }
        if (!s.dweight) continue;
        float *sums = (float *)table;            // [sub][d]
        __syncthreads();
        if (mine) at.store(sums + sub * a.d, gu, gv);
        __syncthreads();
        for (int e = threadIdx.x; e < a.d; e += 256) {
            float v = 0.f;
            for (int i = 0; i < 256 / L; i++) v += sums[i * a.d + e];
            a.ws[((int64_t)blockIdx.x * 2 + which) * a.d + e] = v;
        }
    }
}
// 32 elements a workgroup, 32 of the partial sums at a time.
__global__ __launch_bounds__(1024) void head_norm_join(HeadArgs a, int parts) {
    __shared__ double sums[32][33];
    const int e = threadIdx.x & 31, g0 = threadIdx.x >> 5, i = blockIdx.x * 32 + e;
    const float *p = a.ws + i;
    double v = 0;
    if (i < 2 * a.d) {
        int g = g0;
        for (; g + 224 < parts; g += 256) {
            float t[8];
#pragma unroll
            for (int k = 0; k < 8; k++) t[k] = p[(int64_t)(g + 32 * k) * 2 * a.d];
#pragma unroll
            for (int k = 0; k < 8; k++) v += t[k];
        }
        for (; g < parts; g += 32) v += p[(int64_t)g * 2 * a.d];
    }
    sums[g0][e] = v;
    __syncthreads();
    if (g0 || i >= 2 * a.d) return;
    for (int g = 1; g < 32; g++) v += sums[g][e];
    const int which = i >= a.d;
    float *out = a.side[which].dweight;
    if (out && a.side[which].heads) out[i - which * a.d] = (float)v;
}

// ------------------------------------------------------------------- host

// Pairs of a lane: as many as divide the turned ones and the rest.
static int head_vector(const HeadArgs &a) {
    const int rest = a.d / 2 - a.turned;
    for (int v = 8; v > 1; v /= 2)
        if (a.turned % v == 0 && rest % v == 0) return v;
    return 1;
}
static int head_lanes(const HeadArgs &a) {
    const int n = (a.d / 2 + head_vector(a) - 1) / head_vector(a);
    int l = 1;
    while (l < n) l *= 2;
    return l;
}
bool head_norm_ok(const HeadArgs &a) { return head_lanes(a) <= 64; }
static int head_tokens(const HeadArgs &a) {
    // four heads a lane group, but first a workgroup for every CU
    const int64_t all = (int64_t)a.b * a.t, heads = a.side[0].heads + a.side[1].heads;
    int64_t n = 4 * (256 / head_lanes(a)) / heads;
    if (n > (all + 1023) / 1024) n = (all + 1023) / 1024;
    const int64_t most = 4096 / (a.d / 2);       // 32 KB of angles
    if (n > most) n = most;
    if (n > HEAD_TOKENS) n = HEAD_TOKENS;
    return n < 1 ? 1 : (int)n;
}
static int head_groups(const HeadArgs &a) {
    const int64_t n = ((int64_t)a.b * a.t + head_tokens(a) - 1) / head_tokens(a);
    return n < 1024 ? (int)n : 1024;
}
size_t head_norm_workspace(const HeadArgs &a) { return (size_t)head_groups(a) * 2 * a.d * 4; }

template <typename F> static hipError_t by_head_form(const HeadArgs &a, F f) {
    auto v = [&](auto in, auto out) {
        auto of = [&](auto inter) {
            switch (head_vector(a)) {
            case 8: return f(in, out, std::integral_constant<int, 8>(), inter);
            case 4: return f(in, out, std::integral_constant<int, 4>(), inter);
            case 2: return f(in, out, std::integral_constant<int, 2>(), inter);
            default: return f(in, out, std::integral_constant<int, 1>(), inter);
            }
        };
        return a.interleaved ? of(std::true_type()) : of(std::false_type());
    };
    if (a.type == F16) return v(Tag<_Float16>(), Tag<_Float16>());
    if (a.type == BF16) return v(Tag<__bf16>(), Tag<__bf16>());
    if (a.ytype == F16) return v(Tag<float>(), Tag<_Float16>());
    if (a.ytype == BF16) return v(Tag<float>(), Tag<__bf16>());
    return v(Tag<float>(), Tag<float>());
}

hipError_t launch_head_norm(const HeadArgs &in, bool backward, hipStream_t st) {
    HeadArgs a = in;
    a.lanes = head_lanes(a);
    a.tokens = head_tokens(a);
    const int64_t all = (int64_t)a.b * a.t, groups = (all + a.tokens - 1) / a.tokens;
    size_t lds = a.turned ? (size_t)a.tokens * (a.d / 2) * 8 : 0;
    hipError_t e = hipSuccess;
    if (!backward) {
        if (!groups) return e;
        return by_head_form(a, [&](auto ti, auto to, auto v, auto inter) {
            typedef typename decltype(ti)::type T;
            typedef typename decltype(to)::type U;
            hipLaunchKernelGGL((head_norm_forward<T, U, decltype(v)::value, decltype(inter)::value>),
                               grid_of(groups), dim3(256), lds, st, a);
            return hipGetLastError();
        });
    }
    const int parts = head_groups(a);
    const size_t sums = (size_t)(256 / a.lanes) * a.d * 4;
    if (lds < sums) lds = sums;
    if (parts)
        e = by_head_form(a, [&](auto ti, auto to, auto v, auto inter) {
            typedef typename decltype(ti)::type T;
            typedef typename decltype(to)::type U;
            hipLaunchKernelGGL((head_norm_backward<T, U, decltype(v)::value, decltype(inter)::value>),
                               dim3(parts), dim3(256), lds, st, a);
            return hipGetLastError();
        });
    if (e != hipSuccess || (!a.side[0].dweight && !a.side[1].dweight)) return e;
    return start(head_norm_join, dim3((2 * a.d + 31) / 32), 1024, st, a, parts);
}

}  // namespace ops
}  // namespace ctc
