// Group norm with an activation on channels-last maps x [n][hw][c]:
//   xhat = (x - mean) rstd,  z = xhat gamma_c + beta_c (+ r),  y = act(z)
// with mean and rstd = 1 / sqrt(var + eps) over the pixels and channels of
// (image, group).  A carry-through checksum in the last channel takes no
// part in its group's statistics and passes: y = x (+ r).
// Backward, with dz = dy act'(z):
//   dr = dz,  dbeta_c = sum dz,  dgamma_c = sum dz xhat,
//   dx = rstd (dz gamma - (s1 + xhat s2) / count),
//   s1 = sum dz gamma,  s2 = sum dz gamma xhat  over (image, group).
//
// Sums are fp32.  A channel's sum and sum of squares are taken about the
// chunk's first pixel, which lies within a few deviations of the mean, and
// channels and chunks are joined as (count, mean, squared deviations), so a
// mean far from zero costs no digits.
//
// What bounds it: the bytes of the maps.
#pragma once
#include "ops_device.h"

namespace ctc {
namespace ops {

// How a map is cut: threads run along the channels (vectors of V), several
// pixels of a chunk at a time.
struct NormPlan {
    int v, tx, pl;               // channels a thread, threads and pixel lanes
    int ctiles, chunks;          // of a pixel row, of an image
    int64_t chunk;               // pixels
};
static NormPlan norm_plan(const NormArgs &a) {
    NormPlan p{};
    p.v = 16 / type_bytes(a.type);
    while (a.c % p.v) p.v /= 2;
    const int cv = a.c / p.v;
    p.tx = cv < 256 ? cv : 256;
    p.pl = 256 / p.tx;
    p.ctiles = (cv + p.tx - 1) / p.tx;
    // about 2048 workgroups, 8 pixels a thread at least
    int64_t chunks = 2048 / ((a.n < 1 ? 1 : a.n) * p.ctiles);
    const int64_t most = a.hw / (p.pl * 8);
    if (chunks > most) chunks = most;
    if (chunks < 1) chunks = 1;
    p.chunk = (a.hw + chunks - 1) / chunks;
    p.chunks = (int)((a.hw + p.chunk - 1) / p.chunk);
    return p;
}

// Position of a workgroup's threads in the map.
struct NormPos {
    int64_t img, p0, p1;         // image, pixels [p0, p1)
    int c0, pix;                 // first channel, first pixel's offset
    bool on;
    __device__ NormPos(const NormArgs &a, const NormPlan &p) {
        const int64_t t = blockIdx.x / p.ctiles;
        const int ct = blockIdx.x % p.ctiles;
        img = t / p.chunks;
        p0 = t % p.chunks * p.chunk;
        p1 = p0 + p.chunk < a.hw ? p0 + p.chunk : a.hw;
        c0 = (ct * p.tx + (int)threadIdx.x % p.tx) * p.v;
        pix = threadIdx.x / p.tx;
        on = pix < p.pl && c0 < a.c;
    }
};

// Sums two numbers per channel over a workgroup's pixel lanes; f(channel,
// sum1, sum2) for each.
template <int V, typename F>
__device__ __forceinline__ void norm_lanes(const NormArgs &a, const NormPlan &p,
                                           float (*sum)[256 * V], const NormPos &at,
                                           const float (&s1)[V], const float (&s2)[V], F f) {
    const int w = p.tx * V;
    if (at.pix < p.pl)
#pragma unroll
        for (int e = 0; e < V; e++) {
            const int i = at.pix * w + (int)threadIdx.x % p.tx * V + e;
            sum[0][i] = s1[e];
            sum[1][i] = s2[e];
        }
    __syncthreads();
    const int first = (int)(blockIdx.x % p.ctiles) * w;
    for (int i = threadIdx.x; i < w && first + i < a.c; i += 256) {
        float t1 = 0.f, t2 = 0.f;
        for (int l = 0; l < p.pl; l++) {
            t1 += sum[0][l * w + i];
            t2 += sum[1][l * w + i];
        }
        f(first + i, t1, t2);
    }
}

// Per chunk and channel: mean and squared deviations -> ws [n][chunks][c][2]
template <typename T, int V>
__global__ __launch_bounds__(256) void norm_stats(NormArgs a, NormPlan p) {
    __shared__ float sum[2][256 * V];
    const NormPos at(a, p);
    float s1[V] = {}, s2[V] = {}, k[V];
    const T *x = (const T *)a.x + at.img * a.hw * a.c;
    if (at.on) {
        load<T, V>(x + at.p0 * a.c + at.c0, k);
        for (int64_t q = at.p0 + at.pix; q < at.p1; q += p.pl) {
            float v[V];
            load<T, V>(x + q * a.c + at.c0, v);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float d = v[e] - k[e];
                s1[e] += d;
                s2[e] = __builtin_fmaf(d, d, s2[e]);
            }
        }
    }
    const float count = (float)(at.p1 - at.p0), inv = 1.f / count;
    float *out = a.ws + (at.img * p.chunks + at.p0 / p.chunk) * a.c * 2;
    norm_lanes<V>(a, p, sum, at, s1, s2, [&](int c, float t1, float t2) {
        const float k0 = widen(x[at.p0 * a.c + c]), d = t1 * inv;
        const float m2 = t2 - t1 * d;
        out[c * 2] = k0 + d;
        // (not fmaxf, which would drop a NaN)
        out[c * 2 + 1] = m2 < 0.f ? 0.f : m2;
    });
}

// Channels of group g that take part in its statistics.
__device__ __forceinline__ int norm_count(const NormArgs &a, int g) {
    return a.c / a.groups - (a.carry && g == a.groups - 1);
}

// Joins the chunks and channels of an (image, group): one wave each.
static __global__ __launch_bounds__(256) void norm_stats_join(NormArgs a, NormPlan p) {
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= a.n * a.groups) return;
    const int64_t img = t / a.groups;
    const int g = (int)(t % a.groups), per = a.c / a.groups, nc = norm_count(a, g);
    const int lane = threadIdx.x & 63;
    const float *part = a.ws + img * p.chunks * a.c * 2;
    const int entries = p.chunks * nc;
    float mean = 0.f, m2 = 0.f;
    const float total = (float)a.hw * nc;
    for (int i = lane; i < entries; i += 64) {
        const int ch = i / nc;
        const float *e = part + ((int64_t)ch * a.c + g * per + i % nc) * 2;
        const int64_t left = a.hw - ch * p.chunk;
        mean += e[0] * (float)(left < p.chunk ? left : p.chunk);
    }
    mean = nc ? wave_sum(mean) / total : 0.f;
    for (int i = lane; i < entries; i += 64) {
        const int ch = i / nc;
        const float *e = part + ((int64_t)ch * a.c + g * per + i % nc) * 2;
        const int64_t left = a.hw - ch * p.chunk;
        const float d = e[0] - mean;
        m2 += e[1] + d * d * (float)(left < p.chunk ? left : p.chunk);
    }
    m2 = nc ? wave_sum(m2) / total : 0.f;
    if (lane == 0) {
        a.mean[t] = mean;
        a.rstd[t] = 1.f / __builtin_sqrtf(m2 + a.eps);
    }
}

// The constants of V channels: mean, rstd, gamma, beta.
template <int V> struct NormChannels {
    float mean[V], rstd[V], gamma[V], beta[V];
    bool carry[V];
    __device__ NormChannels(const NormArgs &a, int64_t img, int c0) {
        const int per = a.c / a.groups;
#pragma unroll
        for (int e = 0; e < V; e++) {
            const int c = c0 + e;
            const int64_t g = img * a.groups + c / per;
            carry[e] = a.carry && c == a.c - 1;
            // the checksum passes: (x - 0) 1 + 0
            mean[e] = carry[e] ? 0.f : a.mean[g];
            rstd[e] = carry[e] ? 1.f : a.rstd[g];
            gamma[e] = carry[e] || !a.gamma ? 1.f : a.gamma[c];
            beta[e] = carry[e] || !a.beta ? 0.f : a.beta[c];
        }
    }
};

template <typename T, int V>
__global__ __launch_bounds__(256) void norm_apply(NormArgs a, NormPlan p) {
    const NormPos at(a, p);
    if (!at.on) return;
    const NormChannels<V> k(a, at.img, at.c0);
    const T *x = (const T *)a.x, *r = (const T *)a.residual;
    T *y = (T *)a.y;
    for (int64_t q = at.p0 + at.pix; q < at.p1; q += p.pl) {
        const int64_t o = (at.img * a.hw + q) * a.c + at.c0;
        float v[V], rv[V] = {};
        load<T, V>(x + o, v);
        if (r) load<T, V>(r + o, rv);
#pragma unroll
        for (int e = 0; e < V; e++) {
            const float z = __builtin_fmaf((v[e] - k.mean[e]) * k.rstd[e], k.gamma[e],
                                           k.beta[e]) + rv[e];
            v[e] = k.carry[e] ? z : act_of(a.act, z);
        }
        store<T, V>(y + o, v);
    }
}

// dz and xhat of one value.
template <int V>
__device__ __forceinline__ void norm_dz(const NormArgs &a, const NormChannels<V> &k,
                                        const float (&x)[V], const float (&dy)[V],
                                        const float (&r)[V], float (&dz)[V], float (&xh)[V]) {
#pragma unroll
    for (int e = 0; e < V; e++) {
        xh[e] = (x[e] - k.mean[e]) * k.rstd[e];
        const float z = __builtin_fmaf(xh[e], k.gamma[e], k.beta[e]) + r[e];
        dz[e] = k.carry[e] ? dy[e] : dy[e] * act_grad(a.act, z);
    }
}

// Per chunk and channel: sum dz, sum dz xhat -> ws [n][chunks][c][2]
template <typename T, int V>
__global__ __launch_bounds__(256) void norm_grad_sums(NormArgs a, NormPlan p) {
    __shared__ float sum[2][256 * V];
    const NormPos at(a, p);
    float s1[V] = {}, s2[V] = {};
    if (at.on) {
        const NormChannels<V> k(a, at.img, at.c0);
        const T *x = (const T *)a.x, *r = (const T *)a.residual, *dy = (const T *)a.dy;
        for (int64_t q = at.p0 + at.pix; q < at.p1; q += p.pl) {
            const int64_t o = (at.img * a.hw + q) * a.c + at.c0;
            float v[V], g[V], rv[V] = {}, dz[V], xh[V];
            load<T, V>(x + o, v);
            load<T, V>(dy + o, g);
            if (r) load<T, V>(r + o, rv);
            norm_dz<V>(a, k, v, g, rv, dz, xh);
#pragma unroll
            for (int e = 0; e < V; e++) {
                s1[e] += dz[e];
                s2[e] = __builtin_fmaf(dz[e], xh[e], s2[e]);
            }
        }
    }
    float *out = a.ws + (at.img * p.chunks + at.p0 / p.chunk) * a.c * 2;
    norm_lanes<V>(a, p, sum, at, s1, s2, [&](int c, float t1, float t2) {
        out[c * 2] = t1;
        out[c * 2 + 1] = t2;
    });
}

// Where the joined sums s1, s2 [n][groups][2] stand, behind the chunks'.
__host__ __device__ inline int64_t norm_sums_at(const NormArgs &a, const NormPlan &p) {
    return a.n * p.chunks * a.c * 2;
}
// Joins them: the first workgroups take four (image, group)s each, the
// others 16 channels each (dgamma, dbeta over all images).
static __global__ __launch_bounds__(256) void norm_grad_join(NormArgs a, NormPlan p,
                                                             int64_t group_blocks) {
    const int lane = threadIdx.x & 63;
    if (blockIdx.x < group_blocks) {
        const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
        if (t >= a.n * a.groups) return;
        const int64_t img = t / a.groups;
        const int g = (int)(t % a.groups), per = a.c / a.groups, nc = norm_count(a, g);
        const float *part = a.ws + img * p.chunks * a.c * 2;
        float s1 = 0.f, s2 = 0.f;
        for (int i = lane; i < p.chunks * nc; i += 64) {
            const int c = g * per + i % nc;
            const float *e = part + ((int64_t)(i / nc) * a.c + c) * 2;
            const float w = a.gamma ? a.gamma[c] : 1.f;
            s1 += e[0] * w;
            s2 += e[1] * w;
        }
        s1 = wave_sum(s1);
        s2 = wave_sum(s2);
        if (lane == 0) {
            float *out = a.ws + norm_sums_at(a, p) + t * 2;
            const float inv = nc ? 1.f / ((float)a.hw * nc) : 0.f;
            out[0] = s1 * inv;
            out[1] = s2 * inv;
        }
        return;
    }
    __shared__ float sum[2][16][17];
    const int cl = threadIdx.x & 15, row = threadIdx.x >> 4;
    const int c = (int)(blockIdx.x - group_blocks) * 16 + cl;
    float s1 = 0.f, s2 = 0.f;
    if (c < a.c && !(a.carry && c == a.c - 1))
        for (int64_t i = row; i < a.n * p.chunks; i += 16) {
            const float *e = a.ws + (i * a.c + c) * 2;
            s1 += e[0];
            s2 += e[1];
        }
    sum[0][row][cl] = s1;
    sum[1][row][cl] = s2;
    __syncthreads();
    if (row == 0 && c < a.c) {
        for (int i = 1; i < 16; i++) {
            s1 += sum[0][i][cl];
            s2 += sum[1][i][cl];
        }
        if (a.dbeta) a.dbeta[c] = s1;
        if (a.dgamma) a.dgamma[c] = s2;
    }
}

template <typename T, int V>
__global__ __launch_bounds__(256) void norm_grad_apply(NormArgs a, NormPlan p) {
    const NormPos at(a, p);
    if (!at.on) return;
    const NormChannels<V> k(a, at.img, at.c0);
    const int per = a.c / a.groups;
    float m1[V], m2[V];
#pragma unroll
    for (int e = 0; e < V; e++) {
        const float *s = a.ws + norm_sums_at(a, p) +
                         (at.img * a.groups + (at.c0 + e) / per) * 2;
        m1[e] = k.carry[e] ? 0.f : s[0];
        m2[e] = k.carry[e] ? 0.f : s[1];
    }
    const T *x = (const T *)a.x, *r = (const T *)a.residual, *dy = (const T *)a.dy;
    T *dx = (T *)a.dx, *dr = (T *)a.dresidual;
    for (int64_t q = at.p0 + at.pix; q < at.p1; q += p.pl) {
        const int64_t o = (at.img * a.hw + q) * a.c + at.c0;
        float v[V], g[V], rv[V] = {}, dz[V], xh[V];
        load<T, V>(x + o, v);
        load<T, V>(dy + o, g);
        if (r) load<T, V>(r + o, rv);
        norm_dz<V>(a, k, v, g, rv, dz, xh);
        if (dr) store<T, V>(dr + o, dz);
        if (dx) {
#pragma unroll
            for (int e = 0; e < V; e++)
                v[e] = k.rstd[e] * (dz[e] * k.gamma[e] - __builtin_fmaf(xh[e], m2[e], m1[e]));
            store<T, V>(dx + o, v);
        }
    }
}

size_t norm_workspace(const NormArgs &a, bool backward) {
    const NormPlan p = norm_plan(a);
    return 4 * (size_t)(norm_sums_at(a, p) + (backward ? a.n * a.groups * 2 : 0));
}

// f(Tag<T>, V) for a plan's vector width.
template <typename F> static hipError_t by_width(int type, int v, F f) {
    return by_type(type, [&](auto tag) {
        typedef typename decltype(tag)::type T;
        constexpr int W = 16 / (int)sizeof(T);
        if (v == W) return f(tag, std::integral_constant<int, W>());
        if constexpr (W == 8)
            if (v == 4) return f(tag, std::integral_constant<int, 4>());
        if (v == 2) return f(tag, std::integral_constant<int, 2>());
        return f(tag, std::integral_constant<int, 1>());
    });
}

hipError_t launch_norm_forward(const NormArgs &a, hipStream_t st) {
    if (a.n == 0) return hipSuccess;
    const NormPlan p = norm_plan(a);
    const dim3 grid((unsigned)(a.n * p.chunks * p.ctiles));
    return by_width(a.type, p.v, [&](auto tag, auto vc) {
        typedef typename decltype(tag)::type T;
        constexpr int V = decltype(vc)::value;
        hipError_t e = start(norm_stats<T, V>, grid, 256, st, a, p);
        if (e != hipSuccess) return e;
        e = start(norm_stats_join, dim3((unsigned)((a.n * a.groups + 3) / 4)), 256, st, a, p);
        if (e != hipSuccess) return e;
        return start(norm_apply<T, V>, grid, 256, st, a, p);
    });
}

hipError_t launch_norm_backward(const NormArgs &a, hipStream_t st) {
    if (a.n == 0 && !a.dgamma && !a.dbeta) return hipSuccess;
    const NormPlan p = norm_plan(a);
    const dim3 grid((unsigned)(a.n * p.chunks * p.ctiles));
    return by_width(a.type, p.v, [&](auto tag, auto vc) {
        typedef typename decltype(tag)::type T;
        constexpr int V = decltype(vc)::value;
        hipError_t e;
        if (a.n) {
            e = start(norm_grad_sums<T, V>, grid, 256, st, a, p);
            if (e != hipSuccess) return e;
        }
        const int64_t gb = (a.n * a.groups + 3) / 4;
        e = start(norm_grad_join, dim3((unsigned)(gb + (a.c + 15) / 16)), 256, st, a, p, gb);
        if (e != hipSuccess || !a.n || (!a.dx && !a.dresidual)) return e;
        return start(norm_grad_apply<T, V>, grid, 256, st, a, p);
    });
}

}  // namespace ops
}  // namespace ctc
