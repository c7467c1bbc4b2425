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
// Statistics of maps beyond a workgroup (norm_stats): a channel's sum and sum
// of squares over a chunk's pixels are fp64, about the chunk's first pixel, so
// neither a mean far from zero nor an outlier there costs digits; chunks and
// channels are joined as (count, mean, squared deviations), kept in fp32 and
// added in fp64.  Of maps held by a workgroup (norm_slab): the mean, then the
// squared deviations from it, summed in fp32 over up to 8 pixels of a thread
// and the pixel lanes, in fp64 over a group's channels; a mean far from zero
// is off by a few 2^-24 of itself, and the statistics with it.  Gradients' sums
// over a chunk's pixels are fp32, those over chunks, images and a group's
// channels fp64.
//
// What bounds it: the bytes of the maps.  Maps held by a workgroup are read
// once (norm_slab: 64 x 56 x 56 x 64 fp16 with a residual in 22.4 us, 3.4
// TB/s), others twice, by 2048 workgroups each pass (gradients of 32 x 112 x 112
// x 128 bf16 in 138 us: 48 for the sums at 4.3 TB/s, 6 for the joins, 65 for
// the rest at 4.7).
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
// Channels of a vector: 16 bytes, or what divides the channels.
static int norm_width(const NormArgs &a) {
    int v = 16 / type_bytes(a.type);
    while (a.c % v) v /= 2;
    return v;
}
static NormPlan norm_plan(const NormArgs &a) {
    NormPlan p{};
    p.v = norm_width(a);
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
    int ct, c0, pix;             // channel tile, first channel, first pixel's offset
    bool in, on;                 // the workgroup is one of the map's, the thread works
    __device__ NormPos(const NormArgs &a, const NormPlan &p) {
        const uint32_t wg = workgroup();
        const int64_t t = wg / p.ctiles;
        ct = wg % p.ctiles;
        img = t / p.chunks;
        in = img < a.n;
        p0 = t % p.chunks * p.chunk;
        p1 = p0 + p.chunk < a.hw ? p0 + p.chunk : a.hw;
        c0 = (ct * p.tx + (int)threadIdx.x % p.tx) * p.v;
        pix = threadIdx.x / p.tx;
        on = in && pix < p.pl && c0 < a.c;
    }
};

// Sums two numbers per channel over a workgroup's pixel lanes; f(channel,
// sum1, sum2) for each.  fp64 takes LDS for one number after the other (for
// both, 32 KB, a CU holds five workgroups instead of eight).
template <int V, typename N> constexpr int lanes_lds() { return 256 * V * (8 / sizeof(N)); }
template <int V, typename N, typename F>
__device__ __forceinline__ void norm_lanes(const NormArgs &a, const NormPlan &p, N *lds,
                                           const NormPos &at, const N (&s1)[V],
                                           const N (&s2)[V], F f) {
    const int w = p.tx * V;
    N t1[V] = {}, t2[V] = {};
    auto put = [&](N *to, const N (&s)[V]) {
        if (at.pix < p.pl)
#pragma unroll
            for (int e = 0; e < V; e++) to[at.pix * w + (int)threadIdx.x % p.tx * V + e] = s[e];
    };
    auto add = [&](const N *from, N (&t)[V]) {
#pragma unroll
        for (int e = 0; e < V; e++) {
            const int i = threadIdx.x + e * 256;
            if (i < w)
                for (int l = 0; l < p.pl; l++) t[e] += from[l * w + i];
        }
    };
    if constexpr (sizeof(N) == 4) {
        put(lds, s1);
        put(lds + 256 * V, s2);
        __syncthreads();
        add(lds, t1);
        add(lds + 256 * V, t2);
    } else {
        put(lds, s1);
        __syncthreads();
        add(lds, t1);
        __syncthreads();
        put(lds, s2);
        __syncthreads();
        add(lds, t2);
    }
    const int first = at.ct * w;
#pragma unroll
    for (int e = 0; e < V; e++) {
        const int i = threadIdx.x + e * 256;
        if (i < w && first + i < a.c) f(first + i, t1[e], t2[e]);
    }
}

// Per chunk and channel: mean and squared deviations -> ws [n][chunks][c][2].
// In fp64, about the chunk's first pixel: fp32 sums lose a chunk's length in
// digits where that pixel is an outlier (rstd of 12544 x 8 off by 7e-5).
template <typename T, int V>
__global__ __launch_bounds__(256, 8) void norm_stats(NormArgs a, NormPlan p) {
    __shared__ double sum[lanes_lds<V, double>()];
    const NormPos at(a, p);
    if (!at.in) return;
    double s1[V] = {}, s2[V] = {};
    float k[V];
    const T *x = (const T *)a.x + at.img * a.hw * a.c;
    if (at.on) {
        load<T, V>(x + at.p0 * a.c + at.c0, k);
        for (int64_t q = at.p0 + at.pix; q < at.p1; q += p.pl) {
            float v[V];
            load<T, V>(x + q * a.c + at.c0, v);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const double d = (double)v[e] - k[e];
                s1[e] += d;
                s2[e] = __builtin_fma(d, d, s2[e]);
            }
        }
    }
    const double inv = 1. / (double)(at.p1 - at.p0);
    float *out = a.ws + (at.img * p.chunks + at.p0 / p.chunk) * a.c * 2;
    norm_lanes<V>(a, p, sum, at, s1, s2, [&](int c, double t1, double t2) {
        const double d = t1 * inv, m2 = t2 - t1 * d;
        out[c * 2] = (float)(widen(x[at.p0 * a.c + c]) + d);
        // (not fmax, which would drop a NaN)
        out[c * 2 + 1] = m2 < 0 ? 0.f : (float)m2;
    });
}

// Channels of group g that take part in its statistics.
__device__ __forceinline__ int norm_count(const NormArgs &a, int g) {
    return a.c / a.groups - (a.carry && g == a.groups - 1);
}

// Joining an (image, group): W waves over its chunks and channels.
constexpr int JOIN_WAVES = 16;
template <int W> struct NormJoin {
    int64_t img, t;
    int g, per, nc, entries, at; // at: the thread's place among the W waves
    const float *part;
    // `t`th (image, group); part: [n][chunks][c][2]
    __device__ NormJoin(const NormArgs &a, const NormPlan &p, int64_t t_) : t(t_) {
        img = t / a.groups;
        g = (int)(t % a.groups);
        per = a.c / a.groups;
        nc = norm_count(a, g);
        entries = p.chunks * nc;
        part = a.ws + img * p.chunks * a.c * 2 + g * per * 2;
        at = threadIdx.x % (64 * W);
    }
    // f(entry, chunk, channel of the group), eight loads under way
    template <typename F> __device__ __forceinline__ void each(const NormArgs &a, F f) {
        if (nc == 0) return;
        const int step = 64 * W, dch = step / nc, dc = step % nc;
        int ch = at / nc, c = at % nc;
#pragma unroll 8
        for (int i = at; i < entries; i += step) {
            f(*(const float2 *)(part + ((int64_t)ch * a.c + c) * 2), ch, c);
            ch += dch;
            c += dc;
            if (c >= nc) {
                c -= nc;
                ch++;
            }
        }
    }
    // Sum over the W waves, for all of them.
    __device__ __forceinline__ double sum(double v, double *lds) {
        v = wave_sum(v);
        if constexpr (W > 1) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
            __syncthreads();
            v = 0;
#pragma unroll
            for (int i = 0; i < W; i++) v += lds[i];
        }
        return v;
    }
};
// A wave takes an (image, group) of up to 1024 entries, a workgroup of 16 a
// longer one (30690 entries: 247 us by one wave, 13 by 16).
static bool norm_join_wide(const NormArgs &a, const NormPlan &p) {
    return (int64_t)p.chunks * (a.c / a.groups) > 1024;
}
template <int W>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void norm_stats_join(NormArgs a, NormPlan p) {
    __shared__ double lds[W];
    const int64_t t = W == 1 ? (int64_t)workgroup() * 4 + (threadIdx.x >> 6) : workgroup();
    if (t >= a.n * a.groups) return;
    NormJoin<W> j(a, p, t);
    const double total = (double)a.hw * j.nc;
    // about the mean of the first entries (of up to 64 W channels), which lies
    // within the group's spread: one loop, and no digits lost
    const int some = j.entries < 64 * W ? j.entries : 64 * W;
    float at = 0.f;
    if (j.at < some) at = j.part[((int64_t)(j.at / j.nc) * a.c + j.at % j.nc) * 2];
    at = (float)(j.sum(at, lds) / (some ? some : 1));
    double s1 = 0, s2 = 0;
    j.each(a, [&](float2 e, int ch, int) {
        const int64_t left = a.hw - ch * p.chunk;
        const double d = (double)e.x - at, w = d * (double)(left < p.chunk ? left : p.chunk);
        s1 += w;
        s2 += d * w + e.y;
    });
    s1 = j.sum(s1, lds);
    s2 = j.sum(s2, lds);
    if (j.at == 0) {
        const double d = j.nc ? s1 / total : 0;
        double var = j.nc ? s2 / total - d * d : 0;
        var = var < 0 ? 0 : var;                 // (a NaN stays)
        a.mean[t] = (float)(at + d);
        a.rstd[t] = 1.f / __builtin_sqrtf((float)(var + a.eps));
    }
}

// The constants of V channels from c0 on, z = x scale' + ..: mean, rstd,
// gamma, beta; group g of an image by a count along the channels.
template <int V> struct NormChannels {
    float mean[V], rstd[V], gamma[V], beta[V];
    int ck;                      // the checksum's place among them, or -1
    // mean and rstd of the image's group g from where(g)
    template <typename W>
    __device__ __forceinline__ NormChannels(const NormArgs &a, int c0, W where) {
        const int per = a.c / a.groups;
        int g = c0 / per, left = per - c0 % per;
        ck = a.carry && a.c - 1 - c0 < V ? a.c - 1 - c0 : -1;
        float2 k = where(g);
#pragma unroll
        for (int e = 0; e < V; e++) {
            if (left == 0) {
                k = where(++g);
                left = per;
            }
            left--;
            // the checksum passes: (x - 0) 1 + 0
            mean[e] = e == ck ? 0.f : k.x;
            rstd[e] = e == ck ? 1.f : k.y;
            gamma[e] = e == ck || !a.gamma ? 1.f : a.gamma[c0 + e];
            beta[e] = e == ck || !a.beta ? 0.f : a.beta[c0 + e];
        }
    }
};
// ... from the arrays of the whole map
template <int V>
__device__ __forceinline__ NormChannels<V> norm_channels(const NormArgs &a, int64_t img, int c0) {
    return NormChannels<V>(a, c0, [&](int g) {
        return make_float2(a.mean[img * a.groups + g], a.rstd[img * a.groups + g]);
    });
}
// A number for each of V channels: that of its group.
template <int V, typename W>
__device__ __forceinline__ void per_group(const NormArgs &a, int c0, float (&v)[V], W where) {
    const int per = a.c / a.groups;
    int g = c0 / per, left = per - c0 % per;
    float k = where(g);
#pragma unroll
    for (int e = 0; e < V; e++) {
        if (left == 0) {
            k = where(++g);
            left = per;
        }
        left--;
        v[e] = k;
    }
}

// y of V values
template <int V>
__device__ __forceinline__ void norm_values(const NormArgs &a, const NormChannels<V> &k,
                                            float (&v)[V], const float (&r)[V]) {
#pragma unroll
    for (int e = 0; e < V; e++)
        v[e] = __builtin_fmaf(v[e] - k.mean[e], k.rstd[e] * k.gamma[e], k.beta[e]) + r[e];
    if (k.ck < 0) {
        act_of<V>(a.act, v);
    } else {
        float z[V];
#pragma unroll
        for (int e = 0; e < V; e++) z[e] = v[e];
        act_of<V>(a.act, v);
#pragma unroll
        for (int e = 0; e < V; e++) v[e] = e == k.ck ? z[e] : v[e];
    }
}

template <typename T, int V>
__global__ __launch_bounds__(256) void norm_apply(NormArgs a, NormPlan p) {
    const NormPos at(a, p);
    if (!at.on) return;
    const NormChannels<V> k = norm_channels<V>(a, at.img, at.c0);
    const T *x = (const T *)a.x, *r = (const T *)a.residual;
    T *y = (T *)a.y;
    for (int64_t q = at.p0 + at.pix; q < at.p1; q += p.pl) {
        const int64_t o = (at.img * a.hw + q) * a.c + at.c0;
        float v[V], rv[V] = {};
        load<T, V>(x + o, v);
        if (r) load<T, V>(r + o, rv);
        norm_values<V>(a, k, v, rv);
        store<T, V>(y + o, v);
    }
}

// dz and xhat of V values
template <int V>
__device__ __forceinline__ void norm_dz(const NormArgs &a, const NormChannels<V> &k,
                                        const float (&x)[V], const float (&dy)[V],
                                        const float (&r)[V], float (&dz)[V], float (&xh)[V]) {
    float z[V];
#pragma unroll
    for (int e = 0; e < V; e++) {
        xh[e] = (x[e] - k.mean[e]) * k.rstd[e];
        z[e] = __builtin_fmaf(xh[e], k.gamma[e], k.beta[e]) + r[e];
    }
    act_grad<V>(a.act, z);
#pragma unroll
    for (int e = 0; e < V; e++) dz[e] = e == k.ck ? dy[e] : dy[e] * z[e];
}

// Per chunk and channel: sum dz, sum dz xhat -> ws [n][chunks][c][2]
template <typename T, int V>
__global__ __launch_bounds__(256) void norm_grad_sums(NormArgs a, NormPlan p) {
    __shared__ float sum[lanes_lds<V, float>()];
    const NormPos at(a, p);
    if (!at.in) return;
    float s1[V] = {}, s2[V] = {};
    if (at.on) {
        const NormChannels<V> k = norm_channels<V>(a, at.img, at.c0);
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

// dx of V values from dz and xhat; m1, m2: the means over the group
template <int V>
__device__ __forceinline__ void norm_dx(const NormChannels<V> &k, const float (&dz)[V],
                                        const float (&xh)[V], const float (&m1)[V],
                                        const float (&m2)[V], float (&dx)[V]) {
#pragma unroll
    for (int e = 0; e < V; e++) {
        const float d = k.rstd[e] * (dz[e] * k.gamma[e] - __builtin_fmaf(xh[e], m2[e], m1[e]));
        dx[e] = e == k.ck ? dz[e] : d;
    }
}

// Where the joined sums s1, s2 [n][groups][2] stand, behind the chunks'.
__host__ __device__ inline int64_t norm_sums_at(const NormArgs &a, const NormPlan &p) {
    return a.n * p.chunks * a.c * 2;
}
// Joins them: the first workgroups take the (image, group)s, W waves each;
// the others 16 channels each (dgamma, dbeta over all images), by 64 rows of
// threads with eight loads in flight (16 rows took 17 us for 2048 chunks of
// 128 channels, these 6).
constexpr int JOIN_ROWS = 64;
template <int W>
__global__ __launch_bounds__(1024) void norm_grad_join(NormArgs a, NormPlan p,
                                                       int64_t group_blocks) {
    const uint32_t wg = workgroup();
    if (wg < group_blocks) {
        __shared__ double lds[W];
        const int64_t t = W == 1 ? (int64_t)wg * 16 + (threadIdx.x >> 6) : wg;
        if (t >= a.n * a.groups) return;
        NormJoin<W> j(a, p, t);
        double s1 = 0, s2 = 0;
        j.each(a, [&](float2 e, int, int c) {
            const double w = a.gamma ? a.gamma[j.g * j.per + c] : 1;
            s1 += e.x * w;
            s2 += e.y * w;
        });
        s1 = j.sum(s1, lds);
        s2 = j.sum(s2, lds);
        if (j.at == 0) {
            float *out = a.ws + norm_sums_at(a, p) + t * 2;
            const double total = j.nc ? (double)a.hw * j.nc : 1;
            out[0] = (float)(s1 / total);
            out[1] = (float)(s2 / total);
        }
        return;
    }
    __shared__ double sum[2][JOIN_ROWS / 4][16];
    const int cl = threadIdx.x & 15, row = threadIdx.x >> 4;
    const int64_t c = (wg - group_blocks) * 16 + cl;
    double s1 = 0, s2 = 0;
    if (c < a.c && !(a.carry && c == a.c - 1))
#pragma unroll 8
        for (int64_t i = row; i < a.n * p.chunks; i += JOIN_ROWS) {
            const float2 e = *(const float2 *)(a.ws + (i * a.c + c) * 2);
            s1 += e.x;
            s2 += e.y;
        }
    // the four rows of a wave, then the waves
#pragma unroll
    for (int o = 16; o < 64; o *= 2) {
        s1 += __shfl_xor(s1, o);
        s2 += __shfl_xor(s2, o);
    }
    if ((row & 3) == 0) {
        sum[0][row >> 2][cl] = s1;
        sum[1][row >> 2][cl] = s2;
    }
    __syncthreads();
    if (row == 0 && c < a.c) {
#pragma unroll
        for (int i = 1; i < JOIN_ROWS / 4; i++) {
            s1 += sum[0][i][cl];
            s2 += sum[1][i][cl];
        }
        if (a.dbeta) a.dbeta[c] = (float)s1;
        if (a.dgamma) a.dgamma[c] = (float)s2;
    }
}

template <typename T, int V>
__global__ __launch_bounds__(256) void norm_grad_apply(NormArgs a, NormPlan p) {
    const NormPos at(a, p);
    if (!at.on) return;
    const NormChannels<V> k = norm_channels<V>(a, at.img, at.c0);
    const float *sums = a.ws + norm_sums_at(a, p) + at.img * a.groups * 2;
    float m1[V], m2[V];
    per_group<V>(a, at.c0, m1, [&](int g) { return sums[g * 2]; });
    per_group<V>(a, at.c0, m2, [&](int g) { return sums[g * 2 + 1]; });
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
            norm_dx<V>(k, dz, xh, m1, m2, v);
            store<T, V>(dx + o, v);
        }
    }
}

// ---------------------------------------------------------------------------
// Maps of which a workgroup holds whole groups: it takes a slab of w channels
// (whole groups, whole vectors) of an image into its registers, R vectors a
// thread, and normalises from there, so the map is read once.  Threads run
// tx = w / V along the channels and NT / tx along the pixels.
// ---------------------------------------------------------------------------
// vectors a thread holds, of x (and of dy)
template <int NT> constexpr int slab_r() { return 4; }
template <int NT> constexpr int slab_r_forward() { return NT == 256 ? 4 : 8; }
// lanes: pixel lanes that hold pixels; slices: threads that add up a channel's
struct SlabPlan { int v, w, tx, pl, slabs, nt, lanes, slices; bool ok, by_xcd; };

template <typename T, int V, int NT, int N> struct Slab {
    static constexpr int NW = NT / 64;
    struct Lds {
        float v[N][NT * V];
        float chan[N][NT];                       // per channel, of w <= NT
        float a[NT], b[NT];                      // per group
    };
    int64_t img;
    int slab, px, cx, c0;        // c0: the thread's first channel
    bool on;
    __device__ bool place(const NormArgs &a, const SlabPlan &p) {
        const uint32_t wg = workgroup(), u = p.by_xcd ? wg >> 3 : wg;
        img = u / p.slabs;
        slab = (int)(u % p.slabs);
        // workgroups go round the eight XCDs: an image's slabs share the
        // lines that one XCD's L2 holds
        if (p.by_xcd) img = img * 8 + (wg & 7);
        cx = (int)threadIdx.x % p.tx;
        px = (int)threadIdx.x / p.tx;
        on = px < p.pl;
        c0 = slab * p.w + cx * V;
        return img < a.n;
    }
    // Sums of N numbers per channel over the pixel lanes -> l.chan.
    __device__ void channels(Lds &l, const SlabPlan &p, const float (&s)[N][V]) {
        if (on)
#pragma unroll
            for (int n = 0; n < N; n++)
#pragma unroll
                for (int e = 0; e < V; e++) l.v[n][(px * p.tx + cx) * V + e] = s[n][e];
        __syncthreads();
        // a channel's lanes in slices, then the slices: about as many slices
        // as lanes of one (as many as there are threads took 15 us, these 9,
        // for 12 images of 2 x 2 x 4)
        const int slices = p.slices, i = threadIdx.x, c = i % p.w, q = i / p.w;
        float t[N] = {};
        if (q < slices)
            for (int x = q; x < p.lanes; x += slices)
#pragma unroll
                for (int n = 0; n < N; n++) t[n] += l.v[n][x * p.w + c];
        __syncthreads();
        if (q < slices)
#pragma unroll
            for (int n = 0; n < N; n++) l.v[n][i] = t[n];
        __syncthreads();
        if (i < p.w)
#pragma unroll
            for (int n = 0; n < N; n++) {
                float u = 0.f;
                for (int x = 0; x < slices; x++) u += l.v[n][x * p.w + i];
                l.chan[n][i] = u;
            }
        __syncthreads();
    }
    // f(g, wave_sum over the group's channels of g(channel)) by a wave each.
    template <typename G, typename F>
    __device__ void groups(int gs, int per, G value, F f) {
        const int lane = threadIdx.x & 63;
        for (int g = threadIdx.x >> 6; g < gs; g += NW) {
            double t[2] = {};
            for (int c = lane; c < per; c += 64) value(g * per + c, t);
            t[0] = wave_sum(t[0]);
            t[1] = wave_sum(t[1]);
            if (lane == 0) f(g, t);
        }
        __syncthreads();
    }
};

template <typename T, int V, int NT>
__global__ __launch_bounds__(NT) void norm_slab(NormArgs a, SlabPlan p) {
    typedef Slab<T, V, NT, 1> S;
    constexpr int R = slab_r_forward<NT>();
    __shared__ typename S::Lds l;
    S s;
    if (!s.place(a, p)) return;
    const int per = a.c / a.groups, gs = p.w / per, g0 = s.slab * gs;
    const int64_t base = s.img * a.hw * a.c + s.c0;
    const T *x = (const T *)a.x + base;
    Raw<T, V> raw[R];
#pragma unroll
    for (int r = 0; r < R; r++) {
        const int64_t q = s.px + (int64_t)r * p.pl;
        if (s.on && q < a.hw) raw[r].load(x + q * a.c);
    }
    const int ck = a.carry ? a.c - 1 - s.slab * p.w : -1;   // its channel here
    auto count = [&](int g) { return (double)a.hw * (per - (ck >= 0 && ck / per == g)); };
    // the mean, then the squared deviations from it
    float sum[1][V] = {};
#pragma unroll
    for (int r = 0; r < R; r++)
        if (s.on && s.px + (int64_t)r * p.pl < a.hw) {
            float v[V];
            raw[r].values(v);
#pragma unroll
            for (int e = 0; e < V; e++) sum[0][e] += v[e];
            raw[r].hold();
        }
    s.channels(l, p, sum);
    s.groups(gs, per,
             [&](int c, double (&t)[2]) {
                 if (c != ck) t[0] += l.chan[0][c];
             },
             [&](int g, double (&t)[2]) {
                 const double n = count(g);
                 l.a[g] = n > 0 ? (float)(t[0] / n) : 0.f;
             });
    float mean[V], sq[1][V] = {};
    per_group<V>(a, s.cx * V, mean, [&](int g) { return l.a[g]; });
#pragma unroll
    for (int r = 0; r < R; r++)
        if (s.on && s.px + (int64_t)r * p.pl < a.hw) {
            float v[V];
            raw[r].values(v);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float d = v[e] - mean[e];
                sq[0][e] = __builtin_fmaf(d, d, sq[0][e]);
            }
            raw[r].hold();
        }
    s.channels(l, p, sq);
    s.groups(gs, per,
             [&](int c, double (&t)[2]) {
                 if (c != ck) t[0] += l.chan[0][c];
             },
             [&](int g, double (&t)[2]) {
                 const double n = count(g);
                 const float rs =
                     1.f / __builtin_sqrtf((float)((n > 0 ? t[0] / n : 0) + a.eps));
                 l.b[g] = rs;
                 a.mean[s.img * a.groups + g0 + g] = l.a[g];
                 a.rstd[s.img * a.groups + g0 + g] = rs;
             });
    if (!s.on) return;
    const NormChannels<V> k(a, s.c0, [&](int g) { return make_float2(l.a[g - g0], l.b[g - g0]); });
    const T *res = (const T *)a.residual + base;
    T *y = (T *)a.y + base;
#pragma unroll
    for (int r = 0; r < R; r++) {
        const int64_t q = s.px + (int64_t)r * p.pl;
        if (q < a.hw) {
            float v[V], rv[V] = {};
            if (a.residual) load<T, V>(res + q * a.c, rv);
            raw[r].values(v);
            norm_values<V>(a, k, v, rv);
            store<T, V>(y + q * a.c, v);
        }
    }
}

// The same for the gradients: x and dy in registers; the channels' sums over
// the image go to ws [n][c][2] for norm_grad_join (a plan of one chunk), or,
// of a single image, where they belong.
template <typename T, int V, int NT>
__global__ __launch_bounds__(NT) void norm_grad_slab(NormArgs a, SlabPlan p) {
    typedef Slab<T, V, NT, 2> S;
    constexpr int R = slab_r<NT>();
    __shared__ typename S::Lds l;
    S s;
    if (!s.place(a, p)) return;
    const int per = a.c / a.groups, gs = p.w / per;
    const int64_t base = s.img * a.hw * a.c + s.c0;
    const T *x = (const T *)a.x + base, *dy = (const T *)a.dy + base;
    const T *res = (const T *)a.residual + base;
    Raw<T, V> xr[R], dr[R];
#pragma unroll
    for (int r = 0; r < R; r++) {
        const int64_t q = s.px + (int64_t)r * p.pl;
        if (s.on && q < a.hw) {
            xr[r].load(x + q * a.c);
            dr[r].load(dy + q * a.c);
        }
    }
    const NormChannels<V> k = norm_channels<V>(a, s.img, s.on ? s.c0 : 0);
    auto values = [&](int r, int64_t q, float (&dz)[V], float (&xh)[V]) {
        float v[V], g[V], rv[V] = {};
        if (a.residual) load<T, V>(res + q * a.c, rv);
        xr[r].values(v);
        dr[r].values(g);
        norm_dz<V>(a, k, v, g, rv, dz, xh);
    };
    float sum[2][V] = {};
#pragma unroll
    for (int r = 0; r < R; r++) {
        const int64_t q = s.px + (int64_t)r * p.pl;
        if (s.on && q < a.hw) {
            float dz[V], xh[V];
            values(r, q, dz, xh);
#pragma unroll
            for (int e = 0; e < V; e++) {
                sum[0][e] += dz[e];
                sum[1][e] = __builtin_fmaf(dz[e], xh[e], sum[1][e]);
            }
            xr[r].hold();
            dr[r].hold();
        }
    }
    s.channels(l, p, sum);
    const int ck = a.carry ? a.c - 1 - s.slab * p.w : -1;
    for (int c = threadIdx.x; c < p.w; c += NT) {
        if (a.n == 1) {
            if (a.dbeta) a.dbeta[s.slab * p.w + c] = c == ck ? 0.f : l.chan[0][c];
            if (a.dgamma) a.dgamma[s.slab * p.w + c] = c == ck ? 0.f : l.chan[1][c];
        } else {
            float *out = a.ws + (s.img * a.c + s.slab * p.w + c) * 2;
            out[0] = l.chan[0][c];
            out[1] = l.chan[1][c];
        }
    }
    s.groups(gs, per,
             [&](int c, double (&t)[2]) {
                 const double w = a.gamma ? a.gamma[s.slab * p.w + c] : 1;
                 if (c != ck) {
                     t[0] += l.chan[0][c] * w;
                     t[1] += l.chan[1][c] * w;
                 }
             },
             [&](int g, double (&t)[2]) {
                 const double n = (double)a.hw * (per - (ck >= 0 && ck / per == g));
                 l.a[g] = n > 0 ? (float)(t[0] / n) : 0.f;
                 l.b[g] = n > 0 ? (float)(t[1] / n) : 0.f;
             });
    if (!s.on) return;
    float m1[V], m2[V];
    per_group<V>(a, s.cx * V, m1, [&](int g) { return l.a[g]; });
    per_group<V>(a, s.cx * V, m2, [&](int g) { return l.b[g]; });
    T *dx = (T *)a.dx + base, *dres = (T *)a.dresidual + base;
#pragma unroll
    for (int r = 0; r < R; r++) {
        const int64_t q = s.px + (int64_t)r * p.pl;
        if (q < a.hw) {
            float dz[V], xh[V], v[V];
            values(r, q, dz, xh);
            if (a.dresidual) store<T, V>(dres + q * a.c, dz);
            if (a.dx) {
                norm_dx<V>(k, dz, xh, m1, m2, v);
                store<T, V>(dx + q * a.c, v);
            }
        }
    }
}

// Whether and how a map is taken in slabs.
static SlabPlan slab_plan(const NormArgs &a, bool backward) {
    SlabPlan p{};
    const int v = norm_width(a), full = 16 / type_bytes(a.type), per = a.c / a.groups;
    if (a.n < 1) return p;
    int g = per, b = v;                          // least common multiple
    while (b) {
        const int t = g % b;
        g = b;
        b = t;
    }
    const int64_t least = (int64_t)per * v / g;
    if (a.c % least || least > a.c) return p;
    const int k = (int)(a.c / least);
    for (int m = 1; m <= k; m++) {
        if (k % m) continue;
        const int64_t w = least * m;
        auto fits = [&](int nt, int r) {
            if (w > nt) return false;
            const int pl = nt / (int)(w / v);
            return (a.hw + pl - 1) / pl <= r;
        };
        const int nt = v == full && fits(256, 4) ? 256 : fits(1024, backward ? 4 : 8) ? 1024 : 0;
        if (!nt) break;
        // pieces of 16 bytes only where latency is all (gradients of 8 x 3136
        // x 64 fp16 in 8 groups 18 us, as chunks 22; of 64 x 3136 x 64 43.5 us,
        // as chunks 36)
        if (w * type_bytes(a.type) < 32 && a.c * type_bytes(a.type) >= 32 &&
            (double)a.n * a.hw * a.c * type_bytes(a.type) > (4 << 20))
            continue;
        // wider slabs read longer pieces of a row, down to one workgroup a CU,
        // and up to the 128 bytes of a line (64 x 49 x 512 fp16 9.0 us, gradients
        // 11.6; up to 64 bytes 9.6 and 16.5, to 256 10.2 and 12.7.  Where the
        // slab then needs 1024 threads instead of 256 less is better: 64 x 196
        // x 256 fp16 13.2 us, up to 64 bytes 9.5)
        if (p.ok && (w * type_bytes(a.type) > 128 || a.n * (k / m) < 256)) break;
        p.ok = true;
        p.v = v;
        p.w = (int)w;
        p.nt = nt;
        p.tx = (int)(w / v);
        p.pl = nt / p.tx;
        p.slabs = k / m;
    }
    if (p.ok) {
        p.lanes = a.hw < p.pl ? (int)a.hw : p.pl;
        while (p.slices * p.slices < p.lanes && (p.slices + 1) * p.w <= p.nt) p.slices++;
    }
    p.by_xcd = a.n >= 8;
    return p;
}
static dim3 slab_grid(const NormArgs &a, const SlabPlan &p) {
    return grid_of((p.by_xcd ? (a.n + 7) / 8 * 8 : a.n) * p.slabs);
}

size_t norm_workspace(const NormArgs &a, bool backward) {
    const SlabPlan sp = slab_plan(a, backward);
    if (sp.ok) return backward && a.n > 1 ? (size_t)a.n * a.c * 2 * 4 : 0;
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
    const SlabPlan sp = slab_plan(a, false);
    if (sp.ok)
        return by_width(a.type, sp.v, [&](auto tag, auto vc) {
            typedef typename decltype(tag)::type T;
            constexpr int V = decltype(vc)::value;
            if constexpr (V * sizeof(T) == 16)
                if (sp.nt == 256)
                    return start(norm_slab<T, V, 256>, slab_grid(a, sp), 256, st, a, sp);
            return start(norm_slab<T, V, 1024>, slab_grid(a, sp), 1024, st, a, sp);
        });
    const NormPlan p = norm_plan(a);
    const dim3 grid = grid_of(a.n * p.chunks * p.ctiles);
    return by_width(a.type, p.v, [&](auto tag, auto vc) {
        typedef typename decltype(tag)::type T;
        constexpr int V = decltype(vc)::value;
        hipError_t e = start(norm_stats<T, V>, grid, 256, st, a, p);
        if (e != hipSuccess) return e;
        e = norm_join_wide(a, p)
                ? start(norm_stats_join<JOIN_WAVES>, grid_of(a.n * a.groups), 64 * JOIN_WAVES, st,
                        a, p)
                : start(norm_stats_join<1>, grid_of((a.n * a.groups + 3) / 4), 256, st, a, p);
        if (e != hipSuccess) return e;
        return start(norm_apply<T, V>, grid, 256, st, a, p);
    });
}

hipError_t launch_norm_backward(const NormArgs &a, hipStream_t st) {
    if (a.n == 0 && !a.dgamma && !a.dbeta) return hipSuccess;
    const SlabPlan sp = slab_plan(a, true);
    if (sp.ok) {
        hipError_t e = by_width(a.type, sp.v, [&](auto tag, auto vc) {
            typedef typename decltype(tag)::type T;
            constexpr int V = decltype(vc)::value;
            if constexpr (V * sizeof(T) == 16)
                if (sp.nt == 256)
                    return start(norm_grad_slab<T, V, 256>, slab_grid(a, sp), 256, st, a, sp);
            return start(norm_grad_slab<T, V, 1024>, slab_grid(a, sp), 1024, st, a, sp);
        });
        if (e != hipSuccess || a.n == 1 || (!a.dgamma && !a.dbeta)) return e;
        NormPlan one{};
        one.chunks = 1;
        one.chunk = a.hw;
        return start(norm_grad_join<1>, grid_of((a.c + 15) / 16), 1024, st, a, one,
                     (int64_t)0);
    }
    const NormPlan p = norm_plan(a);
    const dim3 grid = grid_of(a.n * p.chunks * p.ctiles);
    return by_width(a.type, p.v, [&](auto tag, auto vc) {
        typedef typename decltype(tag)::type T;
        constexpr int V = decltype(vc)::value;
        hipError_t e;
        if (a.n) {
            e = start(norm_grad_sums<T, V>, grid, 256, st, a, p);
            if (e != hipSuccess) return e;
        }
        const bool wide = norm_join_wide(a, p);
        const int64_t gb = wide ? a.n * a.groups : (a.n * a.groups + 15) / 16;
        const dim3 jg = grid_of(gb + (a.c + 15) / 16);
        e = wide ? start(norm_grad_join<JOIN_WAVES>, jg, 1024, st, a, p, gb)
                 : start(norm_grad_join<1>, jg, 1024, st, a, p, gb);
        if (e != hipSuccess || !a.n || (!a.dx && !a.dresidual)) return e;
        return start(norm_grad_apply<T, V>, grid, 256, st, a, p);
    });
}

}  // namespace ops
}  // namespace ctc
