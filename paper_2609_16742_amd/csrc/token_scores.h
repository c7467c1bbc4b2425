// Scores of given tokens (or classes) from rows of logits x:
//   lse = log sum_i exp x_i,   log p_i = x_i - lse,
//   H = -sum_i p_i log p_i = log s - t / s
// with the running maximum m, s = sum exp(x_i - m) and
// t = sum (x_i - m) exp(x_i - m), so one pass over the row gives all three
// (a new maximum m' scales s by f = exp(m - m') and turns t into
// f (t + (m - m') s)); in the same pass the rank of the target and every
// thread's largest value.
//
// Exponents are in powers of two, in a thread's pass about m2 = m log2(e)
// rounded: a value costs one multiply-add x log2(e) - m2, one exp2, and two
// more for s and t.  s belongs to m2 exactly, so what m2 was rounded by
// (soft_shift, up to 2^-8) comes off when the pass ends, and the joins are
// about m.  Maxima past fp16's range (rows of a type's lowest value or of a
// constant like -1e30; none yet, -inf), whose m2 would be rounded by more
// than exp2 can hold or overflow, take x - m first.
//
// Top alternatives: with the row dealt out to 64 groups of threads, the k-th
// largest group maximum is a lower bound T of the k-th largest value (k
// groups hold one at least), and for values in no order hardly more than k
// are >= T.  Threads whose maximum reaches T read their part again, the
// values >= T are collected and ordered by (value, lower index).  The order
// they are found in does not matter.
//
// What bounds it: the bytes of the logits (2048 x 131072 bf16 with 20
// alternatives in 122 us, 4.4 TB/s), and the vector instructions beside them
// (about ten a value, 72 us there).  A workgroup takes a row, or, of fewer
// than 512 long rows, a share of 4096 values or more of one (one row of 131072
// in 15 us instead of 55); rows of up to 4096 a wave.
#pragma once
#include "ops_device.h"

namespace ctc {
namespace ops {

constexpr int SC_CAP = 512;                      // collected alternatives
constexpr float SC_LOW = -200.f;                 // 2^ of it is 0 in fp32

// About m: s = sum p, t = sum d p with p = 2^d, d = (x - m) log2(e).  m = -inf
// marks an empty state (s = t = 0); s turns NaN with the first NaN or +inf and
// stays it.
struct SoftState { float m, s, t; };
// m2: the product in a register of its own, so that it is rounded the same
// wherever it is used (not contracted into a multiply-add)
__device__ __forceinline__ float soft_m2(float m) {
    float r = m * LOG2E;
    asm("" : "+v"(r));
    return r;
}
__device__ __forceinline__ bool soft_wide(float m) { return !(__builtin_fabsf(m) <= 65536.f); }
// What the pass adds to the exponents d: x LOG2E - m2 = (x - m) LOG2E +
// (m LOG2E - m2), with the same LOG2E in both.
__device__ __forceinline__ float soft_shift(float m) {
    return soft_wide(m) ? 0.f : __builtin_fmaf(m, LOG2E, -soft_m2(m));
}
// The state with every exponent larger by d.
__device__ __forceinline__ void soft_scale(SoftState &a, float d) {
    const float f = exp2_hw(d);
    a.t = (a.t + d * a.s) * f;
    a.s *= f;
}
// (No branches: the joins of a wave are a chain.  An empty state has the
// distance SC_LOW, or none from another empty one.)
__device__ __forceinline__ void soft_join(SoftState &a, SoftState b) {
    const float m = vmax(a.m, b.m);
    soft_scale(a, a.m == m ? 0.f : vmax((a.m - m) * LOG2E, SC_LOW));
    soft_scale(b, b.m == m ? 0.f : vmax((b.m - m) * LOG2E, SC_LOW));
    a.s += b.s;
    a.t += b.t;
    a.m = m;
}

// Total order: NaN above +inf, -0 as +0, equal values by the lower index.
__device__ __forceinline__ uint32_t order_bits(float x) {
    if (x != x) return 0xfffffffeu;              // (below the key ~0)
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t order_key(float x, int i) {
    return (uint64_t)order_bits(x) << 32 | (uint32_t)~i;
}
__device__ __forceinline__ int key_index(uint64_t k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ float key_value(uint64_t k) {
    const uint32_t b = (uint32_t)(k >> 32);
    return __builtin_bit_cast(float, b & 0x80000000u ? b ^ 0x80000000u : ~b);
}
// How many of keys[0 .. n) are larger (keys[n .. n + 3] have to be 0).
__device__ __forceinline__ int keys_above(const uint64_t *keys, int n, uint64_t mine) {
    int r = 0;
    for (int j = 0; j < n; j += 4)
#pragma unroll
        for (int e = 0; e < 4; e++) r += keys[j + e] > mine;
    return r;
}

// The next value below x; NaN (which !(y <= x) holds for every y) below -inf.
__device__ __forceinline__ float below(float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    if (x == -INF) return __builtin_nanf("");
    if (x == 0.f) return __builtin_bit_cast(float, 0x80000001u);
    return __builtin_bit_cast(float, x > 0.f ? b - 1 : b + 1);
}

__device__ __forceinline__ uint64_t shfl_xor_key(uint64_t k, int o) {
    const uint32_t lo = __shfl_xor((uint32_t)k, o), hi = __shfl_xor((uint32_t)(k >> 32), o);
    return (uint64_t)hi << 32 | lo;
}

// The k-th largest of the 64 lanes' values (k <= 64).
__device__ __forceinline__ float kth_of_lanes(float v, int k) {
    int above = 0;
#pragma unroll 8
    for (int j = 0; j < 64; j++) {
        const float o = __builtin_bit_cast(
            float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), j));
        above += o > v;
    }
    // lanes with fewer than k larger values: k of them at least
    float r = above < k ? v : INF;
#pragma unroll
    for (int o = 32; o; o >>= 1) r = fminf(r, __shfl_xor(r, o));
    return r;
}

// What a workgroup of NT threads finds in elements [lo, hi) of a row.
template <typename T, int NT> struct ScorePart {
    static constexpr int V = 16 / (int)sizeof(T);
    static constexpr int NW = NT / 64;
    struct Lds {
        float gmax[64];
        SoftState st[NW];
        int cnt[NW];
        int found, threads;
        uint16_t thread[NT];
        uint64_t key[SC_CAP + 4];
        uint64_t best[NW];
    };

    const T *x;
    int lo, hi;
    int target;                  // -1: no rank wanted
    float xt, thr_before;        // the target's value, and the next below it
    SoftState st;                // in scan(): exponents larger by `shift`
    float m2, shift;             // of st.m
    int cnt;

    // VALS elements from index i on.  The rank counts a wave at a time: `cnt`
    // is right in the lane that takes part longest, the first.
    template <int VALS> __device__ __forceinline__ void add(const float (&v)[VALS], int i) {
        float vm;
        if constexpr (VALS == 8)
            vm = vmax3(vmax3(vmax3(v[0], v[1], v[2]), v[3], v[4]), v[5],
                       vmax(v[6], v[7]));
        else if constexpr (VALS == 4)
            vm = vmax3(vmax(v[0], v[1]), v[2], v[3]);
        else vm = v[0];
        if (vm > st.m) {
            const float sh = soft_shift(vm);
            // (vmax drops the NaN of infinity from infinity)
            soft_scale(st, vmax(__builtin_fmaf(st.m - vm, LOG2E, sh - shift), SC_LOW));
            st.m = vm;
            m2 = soft_m2(vm);
            shift = sh;
        }
        if (!soft_wide(st.m)) {
#pragma unroll
            for (int e = 0; e < VALS; e++) {
                const float d = __builtin_fmaf(v[e], LOG2E, -m2);
                const float p = exp2_hw(d);
                st.s += p;
                st.t = __builtin_fmaf(vmax(d, SC_LOW), p, st.t);
            }
        } else {
            const float mu = st.m == -INF ? 0.f : st.m;
#pragma unroll
            for (int e = 0; e < VALS; e++) {
                const float d = (v[e] - mu) * LOG2E;
                const float p = exp2_hw(d);
                st.s += p;
                st.t = __builtin_fmaf(vmax(d, SC_LOW), p, st.t);
            }
        }
        if (target >= 0) {
            // (the target's own vector: scan() adds what stands before it)
            const float thr = i + VALS <= target ? thr_before : xt;
#pragma unroll
            for (int e = 0; e < VALS; e++)
                cnt += __builtin_popcountll(__ballot(!(v[e] <= thr)));
        }
    }
    __device__ void scan() {
        constexpr int U = 4;
        const int tid = threadIdx.x;
        const int nv = (hi - lo) / V;
        st = SoftState{-INF, 0.f, 0.f};
        m2 = shift = 0.f;
        cnt = 0;
        int i = tid;
        if (U * NT <= nv) thr_before = below(xt);
        // (all threads together: lane 0 stays to the end, see add)
        for (; i - tid + U * NT <= nv; i += U * NT) {
            float v[U][V];
#pragma unroll
            for (int u = 0; u < U; u++) load<T, V>(x + lo + (i + u * NT) * V, v[u]);
#pragma unroll
            for (int u = 0; u < U; u++) add(v[u], lo + (i + u * NT) * V);
        }
        // what is left: U vectors a thread at most and one value, sent for
        // together (and ahead of the wait for the target's value)
        {
            float v[U][V], w[1];
#pragma unroll
            for (int u = 0; u < U; u++)
                if (i + u * NT < nv) load<T, V>(x + lo + (i + u * NT) * V, v[u]);
            const int j = lo + nv * V + tid;
            if (j < hi) w[0] = widen(x[j]);
            thr_before = below(xt);
#pragma unroll
            for (int u = 0; u < U; u++)
                if (i + u * NT < nv) add(v[u], lo + (i + u * NT) * V);
            if (j < hi) add(w, j);
        }
        soft_scale(st, -shift);
        if (target >= 0 && xt != xt) {           // only NaN stands beside NaN
            cnt = 0;
            for (int j = lo + tid; j < hi && j < target; j += NT) {
                const float v = widen(x[j]);
                cnt += __builtin_popcountll(__ballot(v != v));
            }
        } else if (target >= lo && target < lo + nv * V && tid == 0) {
            // equal values before the target in its vector
            for (int j = target - (target - lo) % V; j < target; j++) cnt += widen(x[j]) == xt;
        }
    }
    // f(value, index) for every element this thread scanned
    template <typename F> __device__ __forceinline__ void again(F f) {
        const int nv = (hi - lo) / V;
        for (int i = threadIdx.x; i < nv; i += NT) {
            float v[V];
            load<T, V>(x + lo + i * V, v);
#pragma unroll
            for (int e = 0; e < V; e++) f(v[e], lo + i * V + e);
        }
        const int i = lo + nv * V + threadIdx.x;
        if (i < hi) f(widen(x[i]), i);
    }
    // Joins the threads' states; every thread returns with the whole.
    __device__ void join(Lds &l, SoftState &all, int &count) {
        SoftState a = st;
        int c = __builtin_amdgcn_readfirstlane(cnt);
#pragma unroll
        for (int o = 32; o; o >>= 1) {
            SoftState b{__shfl_xor(a.m, o), __shfl_xor(a.s, o), __shfl_xor(a.t, o)};
            soft_join(a, b);
        }
        if constexpr (NW > 1) {
            const int w = threadIdx.x >> 6;
            if ((threadIdx.x & 63) == 0) {
                l.st[w] = a;
                l.cnt[w] = c;
            }
            __syncthreads();
            a = l.st[0];
            c = l.cnt[0];
#pragma unroll
            for (int i = 1; i < NW; i++) {
                soft_join(a, l.st[i]);
                c += l.cnt[i];
            }
        }
        all = a;
        count = c;
    }
    // The k best entries in descending order to out(rank, key), fewer if the
    // range holds fewer that are not -inf; returns how many.
    template <typename F> __device__ int top(Lds &l, int k, F out) {
        const int tid = threadIdx.x, lane = tid & 63;
        // (a thread with a NaN or +inf takes part whatever its maximum)
        const bool odd = st.s != st.s;
        float g = st.m;
#pragma unroll
        for (int o = NW / 2; o; o >>= 1) g = vmax(g, __shfl_xor(g, o));
        if (tid == 0) l.found = l.threads = 0;
        if constexpr (NW > 1) {
            if (lane % NW == 0) l.gmax[tid / NW] = g;
            __syncthreads();
            g = l.gmax[lane];
        } else {
            __syncthreads();
        }
        const float T0 = kth_of_lanes(g, k);
        auto take = [&](float v, int i) {
            if (!(v < T0) && v != -INF) {
                const int at = atomicAdd(&l.found, 1);
                if (at < SC_CAP) l.key[at] = order_key(v, i);
            }
        };
        // The vectors of the threads that hold such values are dealt out to
        // all (each reading its own again, one after the other, was a fifth
        // of the kernel at 131072 tokens).
        const int nv = (hi - lo) / V, own = (nv + NT - 1) / NT;
        if (st.m >= T0 || odd) {
            l.thread[atomicAdd(&l.threads, 1)] = (uint16_t)tid;
            const int i = lo + nv * V + tid;
            if (i < hi) take(widen(x[i]), i);
        }
        __syncthreads();
        for (int q = tid; q < l.threads * own; q += NT) {
            const int i = l.thread[q / own] + q % own * NT;
            if (i < nv) {
                float v[V];
                load<T, V>(x + lo + i * V, v);
#pragma unroll
                for (int e = 0; e < V; e++) take(v[e], lo + i * V + e);
            }
        }
        __syncthreads();
        const int n = l.found;
        if (n <= SC_CAP) {
            if (tid < 4) l.key[n + tid] = 0;
            __syncthreads();
            for (int i = tid; i < n; i += NT) {
                const uint64_t mine = l.key[i];
                const int r = keys_above(l.key, n, mine);
                if (r < k) out(r, mine);
            }
            return n < k ? n : k;
        }
        // More values than places at or above T0 (many equal ones): the best
        // of what is left, one by one, the row read again for each (20
        // alternatives of 2048 x 131072 equal bf16 logits in 2242 us, of normal
        // ones in 129; 128 x 1000 36 and 9, one row of 131072 48 and 15).
        uint64_t last = ~0ull;
        for (int r = 0; r < k; r++) {
            uint64_t b = 0;
            again([&](float v, int i) {
                if (!(v < T0) && v != -INF) {
                    const uint64_t q = order_key(v, i);
                    if (q < last && q > b) b = q;
                }
            });
#pragma unroll
            for (int o = 32; o; o >>= 1) {
                const uint64_t q = shfl_xor_key(b, o);
                b = q > b ? q : b;
            }
            if constexpr (NW > 1) {
                if (lane == 0) l.best[tid >> 6] = b;
                __syncthreads();
                b = l.best[0];
                for (int i = 1; i < NW; i++) b = l.best[i] > b ? l.best[i] : b;
                __syncthreads();
            }
            last = b;
            if (tid == 0) out(r, b);
        }
        return k;
    }
};

// What the outputs of a row are, given its joined state.
__device__ __forceinline__ float soft_log(SoftState a) {
    return LN2 * __builtin_amdgcn_logf(a.s);
}
__device__ __forceinline__ float soft_lse(SoftState a) {
    return a.m == -INF && a.s == 0.f ? -INF : a.m + soft_log(a);
}
// log p of a logit: about the maximum, so a row far from zero (one of the
// type's lowest values, say) keeps its digits, which x - lse would lose.
__device__ __forceinline__ float soft_logprob(SoftState a, float x) {
    return (x - a.m) - soft_log(a);
}
__device__ __forceinline__ void write_scores(const ScoreArgs &a, int64_t row, SoftState s,
                                             int count, int target, float xt) {
    const bool empty = s.m == -INF && s.s == 0.f;
    const float lse = soft_lse(s);
    if (a.lse) a.lse[row] = lse;
    if (a.entropy)
        a.entropy[row] = empty ? 0.f : LN2 * (__builtin_amdgcn_logf(s.s) - s.t / s.s);
    if (a.logprob) a.logprob[row] = target < 0 ? 0.f : empty ? -INF : soft_logprob(s, xt);
    if (a.rank) a.rank[row] = target < 0 ? -1 : count;
}

struct ScorePlan { int splits, chunk; };
// A split's share in the workspace: m, s, t, rank count, then top_k keys.
__host__ __device__ inline size_t score_part_bytes(int k) { return 16 + 8 * (size_t)k; }

template <typename T, int NT>
__global__ __launch_bounds__(NT) void token_scores(ScoreArgs a, ScorePlan p) {
    typedef ScorePart<T, NT> Part;
    __shared__ typename Part::Lds l;
    const int64_t row = blockIdx.x / p.splits;
    const int split = blockIdx.x % p.splits;
    const int tid = threadIdx.x;
    Part w;
    w.x = (const T *)a.x + row * a.ld;
    w.lo = split * p.chunk;
    w.hi = a.vocab - w.lo < p.chunk ? a.vocab : w.lo + p.chunk;
    int target = a.target ? a.target[row] : -1;
    if (target >= a.vocab) target = -1;
    w.xt = target >= 0 ? widen(w.x[target]) : 0.f;
    w.target = a.rank ? target : -1;
    w.scan();
    SoftState all;
    int count;
    w.join(l, all, count);
    if (p.splits > 1) {
        char *part = (char *)a.ws + blockIdx.x * score_part_bytes(a.top_k);
        if (tid == 0) {
            float *f = (float *)part;
            f[0] = all.m;
            f[1] = all.s;
            f[2] = all.t;
            ((int *)part)[3] = count;
        }
        if (a.top_k) {
            uint64_t *keys = (uint64_t *)(part + 16);
            const int n = w.top(l, a.top_k, [&](int r, uint64_t q) { keys[r] = q; });
            for (int i = n + tid; i < a.top_k; i += NT) keys[i] = 0;
        }
        return;
    }
    if (tid == 0) write_scores(a, row, all, count, target, w.xt);
    if (a.top_k) {
        int32_t *ids = a.ids + row * a.top_k;
        float *tops = a.tops + row * a.top_k;
        const int n = w.top(l, a.top_k, [&](int r, uint64_t q) {
            ids[r] = key_index(q);
            tops[r] = soft_logprob(all, key_value(q));
        });
        for (int i = n + tid; i < a.top_k; i += NT) {
            ids[i] = -1;
            tops[i] = -INF;
        }
    }
}

// Joins the splits of a row (one workgroup a row).  Their lists are sorted,
// so with n lists the smallest of their ceil(k / n)-th entries, and for
// n >= k the k-th largest first entry, is a lower bound of the k-th best:
// hardly more than k entries are left to be ordered.
constexpr int SC_MAX_SPLITS = 64;
template <typename T>
__global__ __launch_bounds__(256) void token_scores_join(ScoreArgs a, ScorePlan p) {
    __shared__ uint64_t keys[SC_MAX_SPLITS * SCORES_MAX_K + 4];
    __shared__ uint64_t bound;
    __shared__ int found;
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, k = a.top_k, lane = tid & 63;
    const size_t bytes = score_part_bytes(k);
    const char *part = (const char *)a.ws + row * p.splits * bytes;
    auto entry = [&](int list, int i) {
        return ((const uint64_t *)(part + list * bytes + 16))[i];
    };
    SoftState all{-INF, 0.f, 0.f};
    int count = 0;
    if (lane < p.splits) {
        const float *f = (const float *)(part + lane * bytes);
        all = SoftState{f[0], f[1], f[2]};
        count = ((const int *)f)[3];
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        SoftState b{__shfl_xor(all.m, o), __shfl_xor(all.s, o), __shfl_xor(all.t, o)};
        soft_join(all, b);
        count += __shfl_xor(count, o);
    }
    const T *x = (const T *)a.x + row * a.ld;
    if (tid == 0) {
        int target = a.target ? a.target[row] : -1;
        if (target >= a.vocab) target = -1;
        write_scores(a, row, all, count, target, target >= 0 ? widen(x[target]) : 0.f);
    }
    if (!k) return;
    if (tid < 64) {
        const int at = (k + p.splits - 1) / p.splits - 1;
        const uint64_t mine = lane < p.splits ? entry(lane, at) : 0;
        int above = 0;
        for (int j = 0; j < p.splits; j++) {
            const uint64_t o = (uint64_t)__builtin_amdgcn_readlane((int)(mine >> 32), j) << 32 |
                               (uint32_t)__builtin_amdgcn_readlane((int)mine, j);
            above += o > mine;
        }
        if (tid == 0) bound = found = 0;
        // (equal entries are empty ones, 0: any of them will do)
        if (lane < p.splits && above == (p.splits >= k ? k : p.splits) - 1) bound = mine;
    }
    __syncthreads();
    const uint64_t least = bound > 1 ? bound : 1;
    for (int i = tid; i < p.splits * k; i += 256) {
        const uint64_t q = entry(i / k, i % k);
        if (q >= least) keys[atomicAdd(&found, 1)] = q;
    }
    __syncthreads();
    const int n = found;
    if (tid < 4) keys[n + tid] = 0;
    __syncthreads();
    int32_t *ids = a.ids + row * k;
    float *tops = a.tops + row * k;
    for (int i = tid; i < n; i += 256) {
        const uint64_t mine = keys[i];
        const int r = keys_above(keys, n, mine);
        if (r < k) {
            ids[r] = key_index(mine);
            tops[r] = soft_logprob(all, key_value(mine));
        }
    }
    for (int i = n + tid; i < k; i += 256) {
        ids[i] = -1;
        tops[i] = -INF;
    }
}

// Threads of a row, by its length: many rows fill the card with a wave each
// (16384 x 4000 bf16 without alternatives 36 us, 256 threads a row 57; 4096 x
// 2000 10 and 13), few rows wait for the longest chain (64 x 16000 7.5 us, a
// wave a row 15.5, 512 threads 8.3).  The rule does not look at the rows: 64 x
// 4000 takes 7.0 us by a wave, 5.1 by 256 threads, 8192 x 8000 45 by 256, 35 by
// a wave, 4096 x 20000 48 by 512, 41 by 256.
static int score_threads(const ScoreArgs &a) {
    return a.vocab <= 4096 ? 64 : a.vocab <= 16384 ? 256 : 512;
}
static ScorePlan score_plan(const ScoreArgs &a) {
    ScorePlan p{1, a.vocab};
    if (score_threads(a) < 512) return p;
    // one workgroup a row leaves CUs idle below 512 rows: shares of 4096
    // elements at least
    const int64_t want = a.rows > 0 ? 512 / a.rows : 1;
    int64_t s = a.vocab / 4096;
    if (s > want) s = want;
    if (s > SC_MAX_SPLITS) s = SC_MAX_SPLITS;
    if (s < 2) return p;
    p.chunk = (int)((a.vocab + s - 1) / s + 7) / 8 * 8;
    p.splits = (a.vocab + p.chunk - 1) / p.chunk;
    return p;
}
size_t scores_workspace(const ScoreArgs &a) {
    const ScorePlan p = score_plan(a);
    return p.splits > 1 ? a.rows * p.splits * score_part_bytes(a.top_k) : 0;
}
hipError_t launch_scores(const ScoreArgs &a, hipStream_t st) {
    if (a.rows == 0) return hipSuccess;
    const ScorePlan p = score_plan(a);
    const dim3 grid((unsigned)(a.rows * p.splits));
    return by_type(a.type, [&](auto tag) {
        typedef typename decltype(tag)::type T;
        const int nt = score_threads(a);
        hipError_t e = nt == 64 ? start(token_scores<T, 64>, grid, 64, st, a, p)
                     : nt == 256 ? start(token_scores<T, 256>, grid, 256, st, a, p)
                                 : start(token_scores<T, 512>, grid, 512, st, a, p);
        if (e != hipSuccess || p.splits == 1) return e;
        return start(token_scores_join<T>, dim3((unsigned)a.rows), 256, st, a, p);
    });
}

// Gradient of the scores:
//   dx_i = p_i (g_lse - g_lp - g_H (log p_i + H)) + [i = target] g_lp
// one read and one write of the row; dx may be x.  Bound by the bytes: 4096 x
// 32001 fp16 in 103 us, 5.1 TB/s.
//
// exp(x - lse) is off by what lse was rounded by, 2^-17 up to |lse| = 256 (a
// row of fp32's lowest value has lse = max for every length).  Past it one
// workgroup takes the row and divides by the sum of exp(x - lse), which is
// neither 0 nor infinite: lse lies within log(vocab) and half its last place
// of the maximum, and is the maximum where half its last place is more than
// that.  No other workgroup can read a row that is written in place.  (4096 x
// 32001 fp16 at 10000: 418 us.)
constexpr float SC_FAR = 256.f;
template <typename T>
__global__ __launch_bounds__(256, 8) void token_scores_grad(ScoreArgs a, int parts) {
    constexpr int V = 16 / (int)sizeof(T), U = 4;
    const int64_t row = blockIdx.x / parts;
    const int lo = (int)(blockIdx.x % parts) * (256 * V * U);
    const T *x = (const T *)a.x + row * a.ld;
    T *dx = (T *)a.dx + row * a.ldd;
    int target = a.target ? a.target[row] : -1;
    if (target >= a.vocab) target = -1;
    const float lse0 = a.lse[row];
    const bool empty = lse0 == -INF;
    const float lse = empty ? 0.f : lse0;
    const float glp = target >= 0 && a.g_logprob && !empty ? a.g_logprob[row] : 0.f;
    const float gh = a.g_entropy ? a.g_entropy[row] : 0.f;
    const float c = (a.g_lse ? a.g_lse[row] : 0.f) - glp -
                    (a.g_entropy ? gh * a.entropy[row] : 0.f);
    auto grad = [&](float lp, int i) {
        const float g = exp_hw(lp) * __builtin_fmaf(-gh, vmax(lp, SC_LOW), c);
        return i == target ? g + glp : g;
    };
    if (__builtin_fabsf(lse) > SC_FAR) {
        if (lo) return;
        __shared__ float sum[4];
        const int nv = a.vocab / V, last = nv * V + threadIdx.x;
        // f(values, their first index) for the thread's vectors of the row,
        // four under way, and for its last value
        auto each = [&](auto f) {
            for (int j = threadIdx.x; j < nv; j += 256 * U) {
                float v[U][V];
#pragma unroll
                for (int u = 0; u < U; u++)
                    if (j + u * 256 < nv) load<T, V>(x + (j + u * 256) * V, v[u]);
#pragma unroll
                for (int u = 0; u < U; u++)
                    if (j + u * 256 < nv) f(v[u], (j + u * 256) * V);
            }
            if (last < a.vocab) {
                float v[1] = {widen(x[last])};
                f(v, last);
            }
        };
        float s = 0.f;
        each([&](auto &v, int) {
            for (float e : v) s += exp_hw(e - lse);
        });
        s = wave_sum(s);
        if ((threadIdx.x & 63) == 0) sum[threadIdx.x >> 6] = s;
        __syncthreads();                         // (the row is read)
        const float log_s = LN2 * __builtin_amdgcn_logf(sum[0] + sum[1] + sum[2] + sum[3]);
        each([&](auto &v, int i) {
            constexpr int N = sizeof(v) / 4;
#pragma unroll
            for (int e = 0; e < N; e++) v[e] = grad((v[e] - lse) - log_s, i + e);
            store<T, N>(dx + i, v);
        });
        return;
    }
    auto one = [&](float v, int i) { return grad(v - lse, i); };
    if (lo + 256 * V * U <= a.vocab) {
        float v[U][V];
#pragma unroll
        for (int u = 0; u < U; u++) load<T, V>(x + lo + (u * 256 + threadIdx.x) * V, v[u]);
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int i = lo + (u * 256 + threadIdx.x) * V;
#pragma unroll
            for (int e = 0; e < V; e++) v[u][e] = one(v[u][e], i + e);
            store<T, V>(dx + i, v[u]);
        }
        return;
    }
    const int nv = (a.vocab - lo) / V;
    for (int j = threadIdx.x; j < nv; j += 256) {
        float v[V];
        load<T, V>(x + lo + j * V, v);
#pragma unroll
        for (int e = 0; e < V; e++) v[e] = one(v[e], lo + j * V + e);
        store<T, V>(dx + lo + j * V, v);
    }
    const int i = lo + nv * V + threadIdx.x;
    if (i < a.vocab) dx[i] = narrow<T>(one(widen(x[i]), i));
}
hipError_t launch_scores_backward(const ScoreArgs &a, hipStream_t st) {
    if (a.rows == 0) return hipSuccess;
    return by_type(a.type, [&](auto tag) {
        typedef typename decltype(tag)::type T;
        constexpr int PER = 256 * 4 * (16 / (int)sizeof(T));
        const int parts = (a.vocab + PER - 1) / PER;
        return start(token_scores_grad<T>, dim3((unsigned)(a.rows * parts)), 256, st, a, parts);
    });
}

}  // namespace ops
}  // namespace ctc
