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
        v[e] = __builtin_fmaf((v[e] - k.mean[e]) * k.rstd[e], k.gamma[e], k.beta[e]) + r[e];
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
    __shared__ float sum[2][256 * V];
    const NormPos at(a, p);
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
// Joins them: the first workgroups take 16 (image, group)s each, a wave each;
// the others 16 channels each (dgamma, dbeta over all images), by 64 rows of
// threads with eight loads in flight (16 rows took 17 us for 2048 chunks of
// 128 channels, these 6).
constexpr int JOIN_ROWS = 64;
static __global__ __launch_bounds__(1024) void norm_grad_join(NormArgs a, NormPlan p,
                                                              int64_t group_blocks) {
    const int lane = threadIdx.x & 63;
    if (blockIdx.x < group_blocks) {
        const int64_t t = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 6);
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
    __shared__ float sum[2][JOIN_ROWS][17];
    const int cl = threadIdx.x & 15, row = threadIdx.x >> 4;
    const int c = (int)(blockIdx.x - group_blocks) * 16 + cl;
    float s1 = 0.f, s2 = 0.f;
    if (c < a.c && !(a.carry && c == a.c - 1))
#pragma unroll 8
        for (int64_t i = row; i < a.n * p.chunks; i += JOIN_ROWS) {
            const float2 e = *(const float2 *)(a.ws + (i * a.c + c) * 2);
            s1 += e.x;
            s2 += e.y;
        }
    sum[0][row][cl] = s1;
    sum[1][row][cl] = s2;
    __syncthreads();
    if (row == 0 && c < a.c) {
        for (int i = 1; i < JOIN_ROWS; i++) {
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
struct SlabPlan { int w, tx, pl, slabs, nt; bool ok, by_xcd; };

template <typename T, int NT, int N> struct Slab {
    static constexpr int V = 16 / (int)sizeof(T), NW = NT / 64;
    struct Lds {
        float v[N][NT * V];
        float chan[N][NT];                       // per channel, of w <= NT
        float a[NT], b[NT];                      // per group
    };
    int64_t img;
    int slab, px, cx, c0;        // c0: the thread's first channel
    bool on;
    __device__ bool place(const NormArgs &a, const SlabPlan &p) {
        if (p.by_xcd) {
            // workgroups go round the eight XCDs: an image's slabs share the
            // lines that one XCD's L2 holds
            const int64_t u = blockIdx.x >> 3;
            img = u / p.slabs * 8 + (blockIdx.x & 7);
            slab = (int)(u % p.slabs);
        } else {
            img = blockIdx.x / p.slabs;
            slab = (int)(blockIdx.x % p.slabs);
        }
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
        // a channel's lanes in slices, then the slices
        const int slices = NT / p.w, i = threadIdx.x, c = i % p.w, q = i / p.w;
        float t[N] = {};
        if (q < slices)
            for (int x = q; x < p.pl; x += slices)
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
            float t[2] = {};
            for (int c = lane; c < per; c += 64) value(g * per + c, t);
            t[0] = wave_sum(t[0]);
            t[1] = wave_sum(t[1]);
            if (lane == 0) f(g, t);
        }
        __syncthreads();
    }
};

template <typename T, int NT>
__global__ __launch_bounds__(NT) void norm_slab(NormArgs a, SlabPlan p) {
    typedef Slab<T, NT, 1> S;
    constexpr int V = S::V, R = slab_r_forward<NT>();
    __shared__ typename S::Lds l;
    S s;
    if (!s.place(a, p)) return;
    const int per = a.c / a.groups, gs = p.w / per, g0 = s.slab * gs;
    const int64_t base = s.img * a.hw * a.c + s.c0;
    const T *x = (const T *)a.x + base;
    u4 raw[R];
#pragma unroll
    for (int r = 0; r < R; r++) {
        const int64_t q = s.px + (int64_t)r * p.pl;
        if (s.on && q < a.hw) __builtin_memcpy(&raw[r], x + q * a.c, 16);
    }
    const int ck = a.carry ? a.c - 1 - s.slab * p.w : -1;   // its channel here
    auto count = [&](int g) { return (float)a.hw * (per - (ck >= 0 && ck / per == g)); };
    // the mean, then the squared deviations from it
    float sum[1][V] = {};
#pragma unroll
    for (int r = 0; r < R; r++)
        if (s.on && s.px + (int64_t)r * p.pl < a.hw) {
            float v[V];
            values_of<T>(raw[r], v);
#pragma unroll
            for (int e = 0; e < V; e++) sum[0][e] += v[e];
            held(raw[r]);
        }
    s.channels(l, p, sum);
    s.groups(gs, per,
             [&](int c, float (&t)[2]) {
                 if (c != ck) t[0] += l.chan[0][c];
             },
             [&](int g, float (&t)[2]) {
                 const float n = count(g);
                 l.a[g] = n > 0.f ? t[0] / n : 0.f;
             });
    float mean[V], sq[1][V] = {};
    per_group<V>(a, s.cx * V, mean, [&](int g) { return l.a[g]; });
#pragma unroll
    for (int r = 0; r < R; r++)
        if (s.on && s.px + (int64_t)r * p.pl < a.hw) {
            float v[V];
            values_of<T>(raw[r], v);
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float d = v[e] - mean[e];
                sq[0][e] = __builtin_fmaf(d, d, sq[0][e]);
            }
            held(raw[r]);
        }
    s.channels(l, p, sq);
    s.groups(gs, per,
             [&](int c, float (&t)[2]) {
                 if (c != ck) t[0] += l.chan[0][c];
             },
             [&](int g, float (&t)[2]) {
                 const float n = count(g);
                 const float rs = 1.f / __builtin_sqrtf((n > 0.f ? t[0] / n : 0.f) + a.eps);
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
            values_of<T>(raw[r], v);
            norm_values<V>(a, k, v, rv);
            store<T, V>(y + q * a.c, v);
        }
    }
}

// The same for the gradients: x and dy in registers; the channels' sums over
// the image go to ws [n][c][2] for norm_grad_join (a plan of one chunk).
template <typename T, int NT>
__global__ __launch_bounds__(NT) void norm_grad_slab(NormArgs a, SlabPlan p) {
    typedef Slab<T, NT, 2> S;
    constexpr int V = S::V, R = slab_r<NT>();
    __shared__ typename S::Lds l;
    S s;
    if (!s.place(a, p)) return;
    const int per = a.c / a.groups, gs = p.w / per;
    const int64_t base = s.img * a.hw * a.c + s.c0;
    const T *x = (const T *)a.x + base, *dy = (const T *)a.dy + base;
    const T *res = (const T *)a.residual + base;
    u4 xr[R], dr[R];
#pragma unroll
    for (int r = 0; r < R; r++) {
        const int64_t q = s.px + (int64_t)r * p.pl;
        if (s.on && q < a.hw) {
            __builtin_memcpy(&xr[r], x + q * a.c, 16);
            __builtin_memcpy(&dr[r], dy + q * a.c, 16);
        }
    }
    const NormChannels<V> k = norm_channels<V>(a, s.img, s.on ? s.c0 : 0);
    auto values = [&](int r, int64_t q, float (&dz)[V], float (&xh)[V]) {
        float v[V], g[V], rv[V] = {};
        if (a.residual) load<T, V>(res + q * a.c, rv);
        values_of<T>(xr[r], v);
        values_of<T>(dr[r], g);
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
            held(xr[r]);
            held(dr[r]);
        }
    }
    s.channels(l, p, sum);
    for (int c = threadIdx.x; c < p.w; c += NT) {
        float *out = a.ws + (s.img * a.c + s.slab * p.w + c) * 2;
        out[0] = l.chan[0][c];
        out[1] = l.chan[1][c];
    }
    const int ck = a.carry ? a.c - 1 - s.slab * p.w : -1;
    s.groups(gs, per,
             [&](int c, float (&t)[2]) {
                 const float w = a.gamma ? a.gamma[s.slab * p.w + c] : 1.f;
                 if (c != ck) {
                     t[0] += l.chan[0][c] * w;
                     t[1] += l.chan[1][c] * w;
                 }
             },
             [&](int g, float (&t)[2]) {
                 const float n = (float)a.hw * (per - (ck >= 0 && ck / per == g));
                 l.a[g] = n > 0.f ? t[0] / n : 0.f;
                 l.b[g] = n > 0.f ? t[1] / n : 0.f;
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

// Whether and how a map is taken in slabs.  Vectors of 16 bytes only.
static SlabPlan slab_plan(const NormArgs &a, bool backward) {
    SlabPlan p{};
    const int v = 16 / type_bytes(a.type), per = a.c / a.groups;
    if (a.c % v || a.n < 1) return p;
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
        const int nt = fits(256, 4) ? 256 : fits(1024, backward ? 4 : 8) ? 1024 : 0;
        if (!nt) break;
        // pieces of 16 bytes only where latency is all
        if (w * type_bytes(a.type) < 32 && a.c * type_bytes(a.type) >= 32 &&
            (double)a.n * a.hw * a.c * type_bytes(a.type) > (4 << 20))
            continue;
        // wider slabs read longer pieces of a row, down to one workgroup a CU
        if (p.ok && (w * type_bytes(a.type) > 128 || a.n * (k / m) < 256)) break;
        p.ok = true;
        p.w = (int)w;
        p.nt = nt;
        p.tx = (int)(w / v);
        p.pl = nt / p.tx;
        p.slabs = k / m;
    }
    p.by_xcd = a.n >= 8;
    return p;
}
static dim3 slab_grid(const NormArgs &a, const SlabPlan &p) {
    return dim3((unsigned)((p.by_xcd ? (a.n + 7) / 8 * 8 : a.n) * p.slabs));
}

size_t norm_workspace(const NormArgs &a, bool backward) {
    const SlabPlan sp = slab_plan(a, backward);
    if (sp.ok) return backward ? (size_t)a.n * a.c * 2 * 4 : 0;
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
        return by_type(a.type, [&](auto tag) {
            typedef typename decltype(tag)::type T;
            return sp.nt == 256 ? start(norm_slab<T, 256>, slab_grid(a, sp), 256, st, a, sp)
                                : start(norm_slab<T, 1024>, slab_grid(a, sp), 1024, st, a, sp);
        });
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
    const SlabPlan sp = slab_plan(a, true);
    if (sp.ok) {
        hipError_t e = by_type(a.type, [&](auto tag) {
            typedef typename decltype(tag)::type T;
            return sp.nt == 256
                       ? start(norm_grad_slab<T, 256>, slab_grid(a, sp), 256, st, a, sp)
                       : start(norm_grad_slab<T, 1024>, slab_grid(a, sp), 1024, st, a, sp);
        });
        if (e != hipSuccess || (!a.dgamma && !a.dbeta)) return e;
        NormPlan one{};
        one.chunks = 1;
        one.chunk = a.hw;
        return start(norm_grad_join, dim3((unsigned)((a.c + 15) / 16)), 1024, st, a, one,
                     (int64_t)0);
    }
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
        const int64_t gb = (a.n * a.groups + 15) / 16;
        e = start(norm_grad_join, dim3((unsigned)(gb + (a.c + 15) / 16)), 1024, st, a, p, gb);
        if (e != hipSuccess || !a.n || (!a.dx && !a.dresidual)) return e;
        return start(norm_grad_apply<T, V>, grid, 256, st, a, p);
    });
}

}  // namespace ops
}  // namespace ctc
