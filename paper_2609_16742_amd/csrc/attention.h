// Attention of queries over keys and its backward pass (part of ops.hip).
//
//   s_ij = scale q_i k_j,  p_ij = exp(s_ij - lse_i),  o_i = sum_j p_ij v_j
//
// over the keys j that query i sees: those before the sequence's length and,
// with `causal`, j <= i + keys - queries.  The G = hq / hkv query heads that
// share a key head are rows of one matrix: row r = t G + g is query t of head
// g, so one query of many heads fills a tile, and the gradients of shared keys
// are sums over rows.
#pragma once
#include "ops_device.h"

namespace ctc {
namespace ops {

typedef __attribute__((address_space(3))) void *AttnLds;
typedef float f16v __attribute__((ext_vector_type(16)));
typedef short s4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s4v *AttnTr;

// The 32 x 32 x 16 products.  Of an operand a lane holds 8 values of k, those
// of 8 (lane / 32) + 0 .. 7, in row or column lane % 32; of a result column
// lane % 32 and rows 8 (i / 4) + 4 (lane / 32) + i % 4.  What a product leaves
// in a lane is so what the next one takes there, with k counted as in `KEY`:
// values 0 .. 3 and 4 .. 7 of a lane are k = 4 (lane / 32) + 0 .. 3 and + 8.
template <typename T> struct Tile;
template <> struct Tile<_Float16> {
    typedef _Float16 V8 __attribute__((ext_vector_type(8)));
    typedef _Float16 V2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ f16v mul(V8 a, V8 b, f16v c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
    // p = 2^SHIFT relative to the maximum, up to 2^LIMIT: its smallest values
    // keep their bits in fp16.  (The backward pass's, at most 1, are 2^15 p.)
    static constexpr float SHIFT = 8.f, LIMIT = 15.f, BACK = 15.f;
};
template <> struct Tile<__bf16> {
    typedef __bf16 V8 __attribute__((ext_vector_type(8)));
    typedef __bf16 V2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ f16v mul(V8 a, V8 b, f16v c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    static constexpr float SHIFT = 0.f, LIMIT = 8.f, BACK = 0.f;
};

// Eight fp32 values in 16 bits (to nearest), as an operand.
template <typename T> __device__ __forceinline__ typename Tile<T>::V8 pack8(const float *v) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typename Tile<T>::V8 r;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const typename Tile<T>::V2 h =
            __builtin_convertvector(f2{v[2 * i], v[2 * i + 1]}, typename Tile<T>::V2);
        r[2 * i] = h[0];
        r[2 * i + 1] = h[1];
    }
    return r;
}

// Tiles in LDS: rows of PITCH elements in pieces of 16 bytes, piece c of row r
// in place c ^ swizzle(r).  LDS has 64 banks, 256 bytes: sixteen rows in a row
// have sixteen places in them for a piece (operands read along rows, 16 lanes
// at a time), and each four of them four places of 64 bytes (operands read
// along columns, 32 columns of 4 rows at a time).  Rows 8 apart differ in bit 1.
template <int PITCH> __device__ __forceinline__ int swizzle(int r) {
    return PITCH == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : ((r & 2) << 1) | ((r >> 2) & 3);
}

// Memory as a buffer of 2^31 - 1 bytes; what is asked for behind it reads as
// zeros.
constexpr uint32_t BEYOND = 0x80000000u;
__device__ __forceinline__ u4 attn_buffer(const void *p) {
    const uint64_t at = (uint64_t)p;
    return u4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at),
              (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32)) & 0xffffu,
              0x7fffffffu, 0x00020000u};
}
__device__ __forceinline__ uint32_t lds_address(const char *p) {
    return (uint32_t)(uintptr_t)(AttnLds)p;
}
// 16 (or 4) bytes a lane from byte `at` of the buffer, `past` bytes further
// (which the bounds do not see), to consecutive places in LDS.  As an
// instruction of its own: with the builtin, the compiler has all loads to LDS
// land before any read along columns, and an iteration's prefetch is waited
// for within it.  Nothing but attn_arrive waits for these.  (M0 is LDS's
// address.  The compiler is told that it is lost, and warns that it is one that
// it may use itself: it would write it anew for that.  A scalar register that
// the vector unit wrote, as readfirstlane does, may be read by a load five
// states later: the compiler sees no load here, so the states stand in it.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds16(const u4 &buf, uint32_t to, uint32_t at,
                                           uint32_t past) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(
                     __builtin_amdgcn_readfirstlane(to)),
                 "v"(at), "s"(buf), "s"(__builtin_amdgcn_readfirstlane(past))
                 : "memory", "m0");
}
__device__ __forceinline__ void load_lds4(const u4 &buf, uint32_t to, uint32_t at) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(
                     __builtin_amdgcn_readfirstlane(to)),
                 "v"(at), "s"(buf)
                 : "memory", "m0");
}
#pragma clang diagnostic pop

// t = r / G for r < 2^31 (G's multiplier and shift: see attn_group).
__device__ __forceinline__ int over_group(const AttnArgs &a, int r) {
    return a.group == 1 ? r : (int)(__umulhi((uint32_t)r, a.gmul) >> a.gshift);
}

// Rows r of the queries (or of what is laid out like them) as one lane sees
// them.
struct AttnRow { int t, g; };
__device__ __forceinline__ AttnRow attn_row(const AttnArgs &a, int r) {
    const int t = over_group(a, r);
    return AttnRow{t, r - t * a.group};
}
// What a lane asks for of a tile of ROWS rows that NW waves load.
template <int PITCH, int ROWS, int NW, bool KEEP = false> struct Loads {
    static constexpr int CH = PITCH / 8, RPI = 64 / CH, N = ROWS / (RPI * NW);
    static constexpr int PER = NW * RPI < 16 ? 16 / (NW * RPI) : 1;  // swizzles of a lane's rows
    static_assert(N * RPI * NW == ROWS, "whole loads");
    // The row of load 0 and the byte of its piece in load i.  Unless they are
    // to be kept they are computed where they are used: a loop's registers are
    // its operands'.
    struct Lane { int row; uint32_t piece[PER]; };
    int lane, wave, d;
    Lane kept;
    __device__ __forceinline__ void init(int l, int w, int head) {
        lane = l;
        wave = w;
        d = head;
        if (KEEP) kept = make(l);
    }
    __device__ __forceinline__ Lane place() const {
        if (KEEP) return kept;
        int l = lane;
        asm volatile("" : "+v"(l));
        return make(l);
    }
    __device__ __forceinline__ Lane make(int l) const {
        Lane p;
        p.row = wave * RPI + l / CH;
#pragma unroll
        for (int o = 0; o < PER; o++) {
            const int c = l % CH ^ swizzle<PITCH>(p.row + o * NW * RPI);
            p.piece[o] = c * 8 < d ? c * 16 : BEYOND;
        }
        return p;
    }
    // A causal tile that some rows see in part: a probability of zero times a
    // NaN or an infinity would be a NaN.  `odd`: whether there is one among the
    // pieces that the wave loaded (and that have landed); `mend` makes them
    // zeros and keeps, for each column, the least of sign * (first + row) of
    // such a value in `least`, if given.
    template <typename T> __device__ __forceinline__ bool odd(const char *tile) const {
        // (an exponent of all ones carries into the sign's place)
        constexpr uint32_t MASK = std::is_same<T, _Float16>::value ? 0x7c007c00u : 0x7f807f80u;
        constexpr uint32_t ADD = std::is_same<T, _Float16>::value ? 0x04000400u : 0x00800080u;
        uint32_t found = 0;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const u4 v = *(const u4 *)(tile + (i * NW + wave) * 1024 + lane * 16);
#pragma unroll
            for (int j = 0; j < 4; j++) found |= (v[j] & MASK) + ADD;
        }
        return __any((int)(found & 0x80008000u));
    }
    template <typename T>
    __device__ __forceinline__ void mend(char *tile, int *least, int sign, int first) const {
        constexpr uint32_t ONES = std::is_same<T, _Float16>::value ? 0x7c00u : 0x7f80u;
#pragma unroll 1
        for (int i = 0; i < N; i++) {
            const int row = wave * RPI + lane / CH + i * (NW * RPI);
            const int c = (lane % CH ^ swizzle<PITCH>(row)) * 8;
            uint16_t *v = (uint16_t *)(tile + (i * NW + wave) * 1024 + lane * 16);
#pragma unroll 1
            for (int j = 0; j < 8; j++)
                if ((v[j] & ONES) == ONES) {
                    v[j] = 0;
                    if (least) atomicMin(least + c + j, sign * (first + row));
                }
        }
    }
    // The wave's pieces of a tile, to another.
    __device__ __forceinline__ void copy(char *to, const char *tile) const {
#pragma unroll 1
        for (int i = 0; i < N; i++) {
            const int at = (i * NW + wave) * 1024 + lane * 16;
            *(u4 *)(to + at) = *(const u4 *)(tile + at);
        }
    }
    // Rows first .. first + ROWS - 1 of a matrix at `base` (rows `stride` bytes
    // apart, those from `end` on as zeros).
    __device__ __forceinline__ void rows(uint32_t tile, const char *base, int64_t stride,
                                         int first, int end) const {
        const u4 buf = attn_buffer(base + first * stride);
        const uint32_t s = (uint32_t)stride;
        const Lane p = place();
        tile += wave * 1024;
        if (first + ROWS <= end) {
#pragma unroll
            for (int i = 0; i < N; i++)
                load_lds16(buf, tile + i * NW * 1024, p.row * s + p.piece[i % PER],
                           i * (NW * RPI) * s);
        } else {
#pragma unroll
            for (int i = 0; i < N; i++) {
                const int r = p.row + i * (NW * RPI);
                load_lds16(buf, tile + i * NW * 1024,
                           first + r < end ? r * s + p.piece[i % PER] : BEYOND, 0);
            }
        }
    }
    // Rows of queries (tokens st, heads sh bytes apart); zeros outside lo .. hi - 1.
    __device__ __forceinline__ void queries(const AttnArgs &a, uint32_t tile, const char *base,
                                            int64_t st, int64_t sh, int first, int lo,
                                            int hi) const {
        if (a.group == 1 && first >= lo) {
            rows(tile, base, st, first, hi);
            return;
        }
        const int t0 = over_group(a, first);
        const u4 buf = attn_buffer(base + t0 * st);
        const Lane p = place();
        tile += wave * 1024;
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int r = first + p.row + i * (NW * RPI);
            const AttnRow q = attn_row(a, r);
            const uint32_t o = (uint32_t)(q.t - t0) * (uint32_t)st + (uint32_t)q.g * (uint32_t)sh;
            load_lds16(buf, tile + i * NW * 1024, r >= lo && r < hi ? o + p.piece[i % PER] : BEYOND,
                       0);
        }
    }
};

// Operands of a tile in LDS.  `rows` is where row lane % 32, piece lane / 32
// stands; `cols` where a lane's four values of columns begin.
template <typename T, int PITCH> struct Operands {
    typedef typename Tile<T>::V8 V8;
    uint32_t rows, x, cols, y;
    __device__ __forceinline__ void init(int lane) {
        const int h = lane >> 5, r = lane & 31;
        rows = r * (PITCH * 2);
        x = (h ^ swizzle<PITCH>(r)) << 4;
        const int k = 4 * h + ((lane >> 2) & 3);
        cols = k * (PITCH * 2) + (lane & 1) * 8;
        y = ((2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) ^ swizzle<PITCH>(k)) << 4;
    }
    // Has addresses computed again where they are used: kept over a loop, they
    // take the registers of its operands.
    __device__ __forceinline__ void refresh() {
        asm volatile("" : "+v"(rows), "+v"(x), "+v"(cols), "+v"(y));
    }
    // rows 32 b .. of k = 16 s ..
    __device__ __forceinline__ V8 along(const char *tile, int b, int s) const {
        return *(const V8 *)(tile + b * 32 * PITCH * 2 + rows + (x ^ (s << 5)));
    }
    // rows 32 b .. of k = 16 s .. (counted as results are, lane by lane)
    __device__ __forceinline__ V8 along_result(const char *tile, int b, int s, int h) const {
        const char *p = tile + b * 32 * PITCH * 2 + rows + 8 * h;
        const uint32_t f = x ^ (h << 4);         // (the piece's place without the half)
        u2 lo, hi;
        __builtin_memcpy(&lo, p + (f ^ (s << 5)), 8);
        __builtin_memcpy(&hi, p + (f ^ 16 ^ (s << 5)), 8);
        return __builtin_bit_cast(V8, u4{lo[0], lo[1], hi[0], hi[1]});
    }
    // columns 32 n .. of k = rows 16 b .. (counted as results are)
    __device__ __forceinline__ V8 across(const char *tile, int b, int n) const {
        const char *p = tile + b * 16 * PITCH * 2 + cols;
        const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((AttnTr)(p + (y ^ (n << 6))));
        const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (AttnTr)(p + 8 * PITCH * 2 + (y ^ 32 ^ (n << 6))));
        return __builtin_bit_cast(V8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// The same operand straight from memory: row `p` (null: zeros), k = 16 s ..
template <typename T> __device__ __forceinline__ typename Tile<T>::V8
row_operand(const T *p, int lane, int s, int d) {
    typename Tile<T>::V8 v{};
    const int e = 16 * s + 8 * (lane >> 5);
    if (p && e < d) v = *(const typename Tile<T>::V8 *)(p + e);
    return v;
}

// Has operands loaded from memory land here, not within the loop that uses
// them, where the wait would be for its prefetch too.
template <typename V, int N> __device__ __forceinline__ void settle(V (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i++) {
        u4 t = __builtin_bit_cast(u4, v[i]);
        asm volatile("" : "+v"(t));
        v[i] = __builtin_bit_cast(V, t);
    }
}

__device__ __forceinline__ float other_half(float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? r[0] : r[1]);
}

// A lane's part of a result's column times f, to the row at `o`.  The two lanes
// of a column hold alternate fours of its values: they exchange every other four,
// so each stores eight in a row.
template <typename T>
__device__ __forceinline__ void store_result(T *o, const f16v &acc, float f, int n, int h32,
                                             int d) {
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
        float v[8];
#pragma unroll
        for (int x = 0; x < 8; x++) v[x] = acc[4 * j + x] * f;
        const u4 p = __builtin_bit_cast(u4, pack8<T>(v));
        const auto lo = __builtin_amdgcn_permlane32_swap(p[0], p[2], false, false);
        const auto hi = __builtin_amdgcn_permlane32_swap(p[1], p[3], false, false);
        const int e = n * 32 + 8 * (j + h32);
        if (e < d) *(u4 *)(o + e) = u4{lo[0], hi[0], lo[1], hi[1]};
    }
}

__device__ __forceinline__ f16v zeros16() {
    f16v z;
#pragma unroll
    for (int i = 0; i < 16; i++) z[i] = 0.f;
    return z;
}

// What the compiler is to schedule next, within its block: reads of LDS well
// ahead of the products that take them.  (Left alone it has a read land just
// before each product: 150 clocks for one of 32.)
constexpr int GROUP_VALU = 0x2, GROUP_MFMA = 0x8, GROUP_READ = 0x100;
#define ATTN_GROUP(what, n) __builtin_amdgcn_sched_group_barrier(what, n, 0)

// Loads of the wave have landed, and so have those of the others.
__device__ __forceinline__ void attn_arrive() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
}

// LDS of what causal tiles with NaNs or infinities leave behind: for each column
// which row had one (see Loads::mend), and for either stage the tile that did.
struct Odd { int least[128], tile[2]; };
__device__ __forceinline__ void odd_init(Odd &odd) {
    for (int i = threadIdx.x; i < 130; i += blockDim.x)
        (i < 128 ? odd.least[i] : odd.tile[i - 128]) = i < 128 ? 0x7fffffff : -1;
    __syncthreads();
}
__device__ __forceinline__ void attn_landed() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}
// Results whose column's bound is below `bound`: they saw such a value.
template <int ND>
__device__ __forceinline__ void odd_results(const Odd &odd, int h32, int bound, f16v (&acc)[ND]) {
#pragma unroll
    for (int n = 0; n < ND; n++)
#pragma unroll
        for (int i = 0; i < 16; i++)
            if (odd.least[n * 32 + 8 * (i / 4) + 4 * h32 + i % 4] < bound)
                acc[n][i] = __builtin_nanf("");
}

// A value that all lanes hold, in a scalar register.
__device__ __forceinline__ float uniform(float v) {
    return __builtin_bit_cast(float,
                              __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
}

// Workgroup id as (sequence and key head, part of it).  Workgroup i runs on XCD
// i % 8, and each XCD has an L2 of its own: where that leaves none idle, what
// reads the same keys runs on the same XCD.
struct AttnPlace { int b, h, part; };
__device__ __forceinline__ AttnPlace attn_place(const AttnArgs &a, int parts, int id) {
    const int pairs = a.b * a.hkv;
    int pair, part;
    if (a.causal) {
        // (longest first, of all pairs)
        pair = id % pairs;
        part = id / pairs;
    } else if (pairs % 8 == 0) {
        pair = (id >> 3) / parts * 8 + (id & 7);
        part = (id >> 3) % parts;
    } else {
        pair = id / parts;
        part = id % parts;
    }
    return AttnPlace{pair / a.hkv, pair % a.hkv, part};
}
__device__ __forceinline__ int attn_length(const int32_t *lengths, int b, int most) {
    if (!lengths) return most;
    const int n = __builtin_amdgcn_readfirstlane(lengths[b]);
    return n < 0 ? 0 : n > most ? most : n;
}

// Rows of a sequence and key head, in tiles of 32: 32 first values, 32 -delta.
__device__ __forceinline__ int64_t attn_stats(const AttnArgs &a, int pair, int r) {
    return ((int64_t)pair * a.row_tiles + (r >> 5)) * 64 + (r & 31);
}

// Keys and values of 64 keys at a time, in one of two stages.
template <int PITCH, int NW, bool KEEP> struct KeyStages {
    static constexpr int TILE = 64 * PITCH * 2;
    Loads<PITCH, 64, NW, KEEP> ld;
    const char *k, *v;
    int64_t ks, vs;
    int end;
    uint32_t lds;
    template <typename T>
    __device__ __forceinline__ void init(const AttnArgs &a, const AttnPlace &at, int lane, int wave,
                                         int keys, const char *to) {
        ld.init(lane, wave, a.d);
        k = (const char *)((const T *)a.k + at.b * a.ks[0] + at.h * a.ks[2]);
        v = (const char *)((const T *)a.v + at.b * a.vs[0] + at.h * a.vs[2]);
        ks = a.ks[1] * 2;
        vs = a.vs[1] * 2;
        end = keys;
        lds = lds_address(to);
    }
    __device__ __forceinline__ void fetch(int key, int stage) const {
        ld.rows(lds + stage * 2 * TILE, k, ks, key, end);
        ld.rows(lds + stage * 2 * TILE + TILE, v, vs, key, end);
    }
};
// Queries and gradients of RT rows, and what attn_rows wrote of them.
template <int PITCH, int RT, int NW> struct RowStages {
    static constexpr int TILE = RT * PITCH * 2, STAGE = 2 * TILE + RT * 8;
    Loads<PITCH, RT, NW> ld;
    const char *q, *g;
    int wave, lane, lo, hi, pair;
    uint32_t lds;
    template <typename T>
    __device__ __forceinline__ void init(const AttnArgs &a, const AttnPlace &at, int l, int w,
                                         int from, int to_row, const char *to) {
        ld.init(l, w, a.d);
        q = (const char *)((const T *)a.q + at.b * a.qs[0] + at.h * a.group * a.qs[2]);
        g = (const char *)((const T *)a.dout + at.b * a.dos[0] + at.h * a.group * a.dos[2]);
        wave = w;
        lane = l;
        lo = from;
        hi = to_row;
        pair = at.b * a.hkv + at.h;
        lds = lds_address(to);
    }
    __device__ __forceinline__ void fetch(const AttnArgs &a, int r, int stage) const {
        const uint32_t to = lds + stage * STAGE;
        ld.queries(a, to, q, a.qs[1] * 2, a.qs[2] * 2, r, lo, hi);
        ld.queries(a, to + TILE, g, a.dos[1] * 2, a.dos[2] * 2, r, lo, hi);
        if (wave < RT / 32)
            load_lds4(attn_buffer(a.stats + attn_stats(a, pair, r) + wave * 64),
                      to + 2 * TILE + wave * 256, lane * 4);
    }
};

// ---------------------------------------------------------------------------
// Forward: a workgroup takes NW tiles of 32 rows, a wave each, and goes through
// the keys (or its range of them) 64 at a time, two stages of keys and values
// in LDS.  A wave computes S^T = K Q^T, so a lane holds 32 scores of one row
// and the softmax needs one exchange between two lanes; P^T then stands as the
// operand of O^T = V^T P^T.  The sums are about a reference that is moved only
// when a row's maximum has grown past it by LIMIT - SHIFT (in powers of two):
// o and l are scaled anew in few steps.
// What bounds it: the matrix unit beside the vector unit's exponentials, and the
// clocks that the power of both allows.  2 x 8192 causal, 16 heads on 2 of 128:
// 509 us, 1.08 PFLOP/s; heads of 64, where a score has half the products, 0.78.
// Waves in their products go before those in their softmax (s_setprio): 556 ->
// 510 us; heads up to 64 lose by it (64 x 14 x 14: 19.5 -> 20.2).  One wave a
// workgroup for up to 32 rows: bytes of keys, 4.3 to 4.9 TB/s.
// ---------------------------------------------------------------------------
template <typename T, int NK, int ND, int NW, bool CAUSAL>
__global__ __launch_bounds__(NW * 64, NW == 1 ? 1 : NK <= 2 ? 4 : NK <= 4 && CAUSAL ? 3 : 2)
void attend(AttnArgs a) {
    typedef typename Tile<T>::V8 V8;
    constexpr int PITCH = NK <= 4 ? 64 : 128, KT = 64, TILE = KT * PITCH * 2;
    __shared__ __attribute__((aligned(16))) char lds[4 * TILE];
    __shared__ Odd odd;
    const int lane = threadIdx.x & 63, h32 = lane >> 5;
    const int wave = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const AttnPlace at = attn_place(a, a.tiles * a.splits, blockIdx.x);
    const int split = at.part % a.splits;
    const int tile = CAUSAL ? a.tiles - 1 - at.part / a.splits : at.part / a.splits;
    const int qn = attn_length(a.qlen, at.b, a.tq), kn = attn_length(a.klen, at.b, a.tk);
    const int r0 = tile * (NW * 32), R = qn * a.group;
    const int first = r0 + wave * 32, r = first + (lane & 31);
    const AttnRow row = attn_row(a, r);
    const bool valid = r < R;
    // keys that the lane's row sees, the wave's first row, the workgroup's last
    auto sees = [&](int t) {
        if (!CAUSAL) return kn;
        const int n = t + kn - qn + 1;
        return n < 0 ? 0 : n > kn ? kn : n;
    };
    const int lim = valid ? sees(row.t) : 0;
    const int least = sees(over_group(a, first)), block_least = sees(over_group(a, r0));
    const int last_row = r0 + NW * 32 <= R ? r0 + NW * 32 - 1 : R - 1;
    const int most = r0 < R ? sees(over_group(a, last_row)) : 0;
    const int wave_last = first + 32 <= R ? first + 31 : R - 1;
    const int wave_most = first < R ? sees(over_group(a, wave_last)) : 0;
    int k0 = 0, k1 = most;
    if (a.splits > 1) {
        k0 = split * a.per;
        if (k1 > k0 + a.per) k1 = k0 + a.per;
    }

    V8 q[NK];
    const T *qp = valid ? (const T *)a.q + at.b * a.qs[0] + row.t * a.qs[1] +
                              (at.h * a.group + row.g) * a.qs[2]
                        : nullptr;
#pragma unroll
    for (int s = 0; s < NK; s++) q[s] = row_operand<T>(qp, lane, s, a.d);
    settle(q);
    f16v acc[ND];
#pragma unroll
    for (int n = 0; n < ND; n++) acc[n] = zeros16();
    float mc = -INF, l = 0.f;
    const float c = uniform(a.scale * LOG2E);

    KeyStages<PITCH, NW, true> in;
    in.template init<T>(a, at, lane, wave, kn, lds);
    Operands<T, PITCH> op;
    op.init(lane);
    if (CAUSAL) odd_init(odd);
    bool spoilt = false;
    if (k0 < k1) in.fetch(k0, 0);
    int stage = 0;
    for (int key = k0; key < k1; key += KT, stage ^= 1) {
        char *kt = lds + stage * 2 * TILE, *vt = kt + TILE;
        const bool look = CAUSAL && key + KT > block_least;
        if (look) {
            attn_landed();
            if (in.ld.template odd<T>(vt)) odd.tile[stage] = key;
        }
        attn_arrive();
        if (key + KT < k1) in.fetch(key + KT, stage ^ 1);
        if (look && odd.tile[stage] == key) {
            in.ld.template mend<T>(vt, odd.least, 1, key);
            spoilt = true;
            __syncthreads();
        }
        if (key >= wave_most) continue;
        f16v s[2];
        if (NK > 4) __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int b = 0; b < 2; b++) {
            s[b] = zeros16();
#pragma unroll
            for (int i = 0; i < NK; i++) s[b] = Tile<T>::mul(op.along(kt, b, i), q[i], s[b]);
        }
        ATTN_GROUP(GROUP_READ, NK);
#pragma unroll
        for (int i = 0; i < NK; i++) {
            ATTN_GROUP(GROUP_MFMA, 1);
            ATTN_GROUP(GROUP_READ, 1);
        }
        ATTN_GROUP(GROUP_MFMA, NK);
        if (NK > 4) __builtin_amdgcn_s_setprio(0);
        if (key + KT > least) {
#pragma unroll
            for (int b = 0; b < 2; b++)
#pragma unroll
                for (int i = 0; i < 16; i++)
                    if (key + b * 32 + 8 * (i / 4) + 4 * h32 + i % 4 >= lim) s[b][i] = -INF;
        }
        float m = vmax3(s[0][0], s[0][1], s[0][2]);
#pragma unroll
        for (int i = 3; i < 15; i += 2) m = vmax3(m, s[0][i], s[0][i + 1]);
        m = vmax3(m, s[0][15], s[1][0]);
#pragma unroll
        for (int i = 1; i < 15; i += 2) m = vmax3(m, s[1][i], s[1][i + 1]);
        m = vmax(m, s[1][15]);
        m = c * vmax(m, other_half(m));
        if (__any(m - mc > Tile<T>::LIMIT)) {
            if (m - mc > Tile<T>::LIMIT) {
                const float to = m - Tile<T>::SHIFT, f = exp2_hw(mc - to);
                mc = to;
                l *= f;
#pragma unroll
                for (int n = 0; n < ND; n++) acc[n] *= f;
            }
        }
        const float ref = mc == -INF ? 0.f : -mc;
        // Half of the values' operands are read while the first half of the
        // probabilities is taken, the rest beside the first products.
        V8 va[2][ND], pb[2];
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int n = 0; n < ND; n++) va[b][n] = op.across(vt, b, n);
        __builtin_amdgcn_sched_barrier(0);
        float p[32];
#pragma unroll
        for (int i = 0; i < 16; i++) p[i] = exp2_hw(__builtin_fmaf(s[0][i], c, ref));
#pragma unroll
        for (int i = 0; i < 16; i++) l += p[i];
#pragma unroll
        for (int b = 0; b < 2; b++) pb[b] = pack8<T>(p + 8 * b);
        __builtin_amdgcn_sched_barrier(0);
        if (NK > 4) __builtin_amdgcn_s_setprio(1);
        V8 vc[2][ND];
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int n = 0; n < ND; n++) {
                acc[n] = Tile<T>::mul(va[b][n], pb[b], acc[n]);
                vc[b][n] = op.across(vt, 2 + b, n);
            }
#pragma unroll
        for (int i = 16; i < 32; i++) p[i] = exp2_hw(__builtin_fmaf(s[1][i - 16], c, ref));
#pragma unroll
        for (int i = 16; i < 32; i++) l += p[i];
        V8 pc[2];
#pragma unroll
        for (int b = 0; b < 2; b++) pc[b] = pack8<T>(p + 16 + 8 * b);
#pragma unroll
        for (int i = 0; i < 2 * ND; i++) {
            ATTN_GROUP(GROUP_MFMA, 1);
            ATTN_GROUP(GROUP_READ, 2);
            ATTN_GROUP(GROUP_VALU, 8);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
            for (int n = 0; n < ND; n++) acc[n] = Tile<T>::mul(vc[b][n], pc[b], acc[n]);
        if (NK > 4) __builtin_amdgcn_s_setprio(0);
    }
    if (spoilt) odd_results<ND>(odd, h32, lim, acc);
    l += other_half(l);
    // (a row that sees nothing, or is none: zeros)
    if (!valid) l = 0.f;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const float lse2 = l == 0.f ? -INF : mc + __builtin_amdgcn_logf(l);
    if (r >= a.tq * a.group) return;
    if (a.splits > 1) {
        const int64_t i = (((int64_t)split * a.b + at.b) * a.hkv + at.h) * a.tq * a.group + r;
        float *o = a.part + i * a.d;
#pragma unroll
        for (int n = 0; n < ND; n++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int e = n * 32 + j * 8 + 4 * h32;
                if (e < a.d) {
                    f4 v;
#pragma unroll
                    for (int x = 0; x < 4; x++) v[x] = valid ? acc[n][4 * j + x] * inv : 0.f;
                    __builtin_memcpy(o + e, &v, 16);
                }
            }
        if (!h32) a.part_lse[i] = lse2;
        return;
    }
    const int head = at.h * a.group + row.g;
    T *o = (T *)a.o + at.b * a.os[0] + row.t * a.os[1] + head * a.os[2];
#pragma unroll
    for (int n = 0; n < ND; n++)
        store_result<T>(o, valid ? acc[n] : zeros16(), inv, n, h32, a.d);
    if (!h32) a.lse[((int64_t)at.b * a.hq + head) * a.tq + row.t] = lse2 * LN2;
}

// Joins the ranges of keys of a row: four values a lane.
template <typename T> __global__ __launch_bounds__(256) void attend_join(AttnArgs a) {
    const int per = a.d / 4;
    const int64_t rows = (int64_t)a.b * a.hkv * a.tq * a.group;
    const int64_t n = (int64_t)workgroup() * 256 + threadIdx.x, i = n / per;
    if (i >= rows) return;
    const int x = (int)(n - i * per) * 4;
    float m = -INF;
#pragma unroll 8
    for (int s = 0; s < a.splits; s++) {
        const float v = a.part_lse[s * rows + i];
        m = v > m ? v : m;
    }
    const float ref = m == -INF ? 0.f : m;
    float l = 0.f;
    f4 sum = (f4)(0.f);
#pragma unroll 8
    for (int s = 0; s < a.splits; s++) {
        f4 v;
        __builtin_memcpy(&v, a.part + (s * rows + i) * a.d + x, 16);
        const float w = exp2_hw(a.part_lse[s * rows + i] - ref);
        l += w;
        sum += w * v;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t pair = i / (a.tq * a.group);
    const AttnRow row = attn_row(a, (int)(i - pair * (a.tq * a.group)));
    const int64_t b = pair / a.hkv, head = (pair - b * a.hkv) * a.group + row.g;
    const float v[4] = {sum[0] * inv, sum[1] * inv, sum[2] * inv, sum[3] * inv};
    store<T, 4>((T *)a.o + b * a.os[0] + row.t * a.os[1] + head * a.os[2] + x, v);
    if (x == 0)
        a.lse[(b * a.hq + head) * a.tq + row.t] =
            l == 0.f ? -INF : (ref + __builtin_amdgcn_logf(l)) * LN2;
}

// ---------------------------------------------------------------------------
// Backward.  With delta_i = do_i o_i,
//   ds_ij = p_ij (do_i v_j - delta_i),
//   dv_j = sum_i p_ij do_i,  dk_j = scale sum_i ds_ij q_i,
//   dq_i = scale sum_j ds_ij k_j.
// `attn_rows` writes what each row needs: -lse as the products' first value
// (so p = exp2(c s), -infinity where the row is no row) and -delta.  fp16 takes
// p for dv as 2^15 p, whatever the gradients are, and ds as 2^e ds with the
// largest e for which 2 |do| |v| 2^e, a bound of it, is at most 2^14 (attn_rows
// finds the sizes).  |v| is the largest of the sequence's key head, since delta
// has a part of each.  |do| is the row's own for dq; for dk, whose sums go over
// rows, it is the largest of those that the workgroup goes through, so a row
// 2^24 times smaller than another in the sum for a key has few bits left there.
// The probabilities are computed twice, once with a lane's key fixed (dk, dv)
// and once with its row fixed (dq): seven products instead of five, and no
// sums between workgroups, whose order would change the result's bits.
// What bounds it: the matrix unit, 0.93 to 0.97 PFLOP/s of those seven (2 x 3136,
// 16 heads of 128: 580 to 605 us).
// ---------------------------------------------------------------------------
template <typename T> __global__ __launch_bounds__(256) void attn_rows(AttnArgs a) {
    __shared__ float most[4];
    const AttnPlace at = attn_place(a, a.q_chunks + a.v_chunks, blockIdx.x);
    const int lane = threadIdx.x & 15, sub = threadIdx.x >> 4, pair = at.b * a.hkv + at.h;
    const int qn = attn_length(a.qlen, at.b, a.tq), kn = attn_length(a.klen, at.b, a.tk);
    const bool queries = at.part < a.q_chunks;
    float top = 0.f;
    if (queries) {
        const int lo = a.causal && qn > kn ? (qn - kn) * a.group : 0, hi = kn ? qn * a.group : 0;
        const float over = -1.f / a.scale;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int r = at.part * 64 + i * 16 + sub;
            const bool valid = r >= lo && r < hi;
            float dot = 0.f, size = 0.f, first = -INF;
            if (valid) {
                const AttnRow row = attn_row(a, r);
                const int head = at.h * a.group + row.g;
                if (8 * lane < a.d) {
                    float x[8], y[8];
                    load<T, 8>((const T *)a.dout + at.b * a.dos[0] + row.t * a.dos[1] +
                                   head * a.dos[2] + 8 * lane, x);
                    load<T, 8>((const T *)a.o + at.b * a.os[0] + row.t * a.os[1] +
                                   head * a.os[2] + 8 * lane, y);
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        dot += x[e] * y[e];
                        size += x[e] * x[e];
                    }
                }
                const float lse = a.lse[((int64_t)at.b * a.hq + head) * a.tq + row.t];
                if (!(lse == -INF)) first = lse * over;
            }
#pragma unroll
            for (int o = 8; o; o >>= 1) {
                dot += __shfl_xor(dot, o);
                size += __shfl_xor(size, o);
            }
            if (lane == 0 && r < a.row_tiles * 32) {
                float *st = a.stats + attn_stats(a, pair, r);
                st[0] = first;
                st[32] = first == -INF ? 0.f : -dot;
            }
            if (size < INF) top = vmax(top, size);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int j = (at.part - a.q_chunks) * 64 + i * 16 + sub;
            float size = 0.f;
            if (j < kn && 8 * lane < a.d) {
                float x[8];
                load<T, 8>((const T *)a.v + at.b * a.vs[0] + j * a.vs[1] + at.h * a.vs[2] +
                               8 * lane, x);
#pragma unroll
                for (int e = 0; e < 8; e++) size += x[e] * x[e];
            }
#pragma unroll
            for (int o = 8; o; o >>= 1) size += __shfl_xor(size, o);
            if (size < INF) top = vmax(top, size);
        }
    }
    if (a.type != F16) return;
    top = vmax(top, __shfl_xor(top, 16));
    top = vmax(top, __shfl_xor(top, 32));
    if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x == 0)
        a.bounds[(int64_t)pair * (a.q_chunks + a.v_chunks) + at.part] =
            vmax(vmax(most[0], most[1]), vmax(most[2], most[3]));
}

// The largest of all lanes' values.
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v = vmax(v, __shfl_xor(v, o));
    return v;
}
// e for squared sizes of do and v.  (60: gradients of zeros)
__device__ __forceinline__ float attn_exponent(float q, float v) {
    // log2 of 2 |do| |v|, rounded up
    const float e = 14.f - __builtin_ceilf(1.f + 0.5f * (__builtin_amdgcn_logf(q) +
                                                       __builtin_amdgcn_logf(v)));
    return e > 60.f ? 60.f : e;
}
// The largest squared size of v of the sequence and key head, and of do in
// chunks q0 .. q1 - 1 of 64 rows.
__device__ __forceinline__ float attn_value_size(const AttnArgs &a, int pair) {
    const float *b = a.bounds + (int64_t)pair * (a.q_chunks + a.v_chunks) + a.q_chunks;
    float v = 0.f;
    for (int i = threadIdx.x & 63; i < a.v_chunks; i += 64) v = vmax(v, b[i]);
    return wave_max(v);
}
__device__ __forceinline__ float attn_row_size(const AttnArgs &a, int pair, int q0, int q1) {
    const float *b = a.bounds + (int64_t)pair * (a.q_chunks + a.v_chunks);
    float q = 0.f;
    for (int i = q0 + (threadIdx.x & 63); i < q1; i += 64) q = vmax(q, b[i]);
    return wave_max(q);
}

// Where a workgroup of attend_keys stands: its keys, and the rows it goes
// through.
template <bool CAUSAL> struct KeyPlace {
    AttnPlace at;
    int pair, split, qn, kn, key0, lo, hi, row, end, shift;
    // first row that sees key j
    __device__ __forceinline__ int seen(const AttnArgs &a, int j) const {
        if (!CAUSAL) return 0;
        const int t = j - shift;
        return t < 0 ? 0 : t * a.group;
    }
    __device__ __forceinline__ KeyPlace(const AttnArgs &a, int rt) {
        at = attn_place(a, a.key_tiles * a.row_splits, blockIdx.x);
        pair = at.b * a.hkv + at.h;
        split = at.part % a.row_splits;
        qn = attn_length(a.qlen, at.b, a.tq);
        kn = attn_length(a.klen, at.b, a.tk);
        shift = kn - qn;
        key0 = at.part / a.row_splits * 128;
        lo = CAUSAL && qn > kn ? (qn - kn) * a.group : 0;
        hi = key0 < kn ? qn * a.group : 0;
        const int first = seen(a, key0);
        row = (first > lo ? first : lo) & ~(rt - 1);
        end = hi;
        if (a.row_splits > 1 && row < hi) {
            const int steps = (hi - row + rt - 1) / rt;
            const int per = (steps + a.row_splits - 1) / a.row_splits;
            row += split * per * rt;
            if (end > row + per * rt) end = row + per * rt;
        }
    }
};
// Stores a wave's dk or dv, times `f` (of a range of rows: as partial sums).
template <typename T, int ND, typename Place>
__device__ __forceinline__ void store_keys(const AttnArgs &a, const Place &p, int key, int h32,
                                           const f16v (&acc)[ND], float f, bool values) {
    if (key >= a.tk) return;
    const bool valid = key < p.kn;
    if (a.row_splits > 1) {
        const int64_t i = ((int64_t)p.split * a.b * a.hkv + p.pair) * a.tk + key;
        float *o = a.part + (i * 2 + values) * a.d;
#pragma unroll
        for (int n = 0; n < ND; n++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int x = n * 32 + j * 8 + 4 * h32;
                f4 u;
#pragma unroll
                for (int z = 0; z < 4; z++) u[z] = valid ? acc[n][4 * j + z] * f : 0.f;
                if (x < a.d) __builtin_memcpy(o + x, &u, 16);
            }
        return;
    }
    T *o = values ? (T *)a.dv + p.at.b * a.dvs[0] + key * a.dvs[1] + p.at.h * a.dvs[2]
                  : (T *)a.dk + p.at.b * a.dks[0] + key * a.dks[1] + p.at.h * a.dks[2];
#pragma unroll
    for (int n = 0; n < ND; n++)
        store_result<T>(o, valid ? acc[n] : zeros16(), f, n, h32, a.d);
}
// Sixteen first values of a block of rows (as a result holds them).
__device__ __forceinline__ f16v first_values(const float *st, int h32) {
    f16v s;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const f4 x = *(const f4 *)(st + 4 * h32 + 8 * j);
#pragma unroll
        for (int i = 0; i < 4; i++) s[4 * j + i] = x[i];
    }
    return s;
}

// dk and dv: a workgroup takes 128 keys, 32 a wave, and goes through the rows
// (or its range of them) RT at a time.  K stays in registers as operands; so
// does V for heads up to 64; V of wider ones is read from LDS, since the sums
// leave no more registers to two waves a SIMD.
template <int NK> struct KeyTiles {
    static constexpr bool WIDE = NK > 4;
    static constexpr int PITCH = WIDE ? 128 : 64, RT = WIDE ? 32 : 64, TILE = RT * PITCH * 2;
    static constexpr int STAGE = RowStages<PITCH, RT, 4>::STAGE;
    static constexpr int BYTES = 2 * STAGE + (WIDE ? 128 * PITCH * 2 : 0);
};
template <typename T, int NK, int ND, bool CAUSAL>
__device__ __forceinline__ void attend_keys(const AttnArgs &a, char *lds, Odd &odd) {
    typedef typename Tile<T>::V8 V8;
    constexpr bool WIDE = KeyTiles<NK>::WIDE;
    constexpr int PITCH = KeyTiles<NK>::PITCH, RT = KeyTiles<NK>::RT, TILE = KeyTiles<NK>::TILE;
    constexpr int STAGE = KeyTiles<NK>::STAGE;
    const int lane = threadIdx.x & 63, h32 = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const KeyPlace<CAUSAL> p(a, RT);
    const int key = p.key0 + wave * 32 + (lane & 31), from = p.seen(a, key);
    const int wave_from = p.seen(a, p.key0 + wave * 32 + 31);
    const int wave_first = p.seen(a, p.key0 + wave * 32);

    const T *vb = (const T *)a.v + p.at.b * a.vs[0] + p.at.h * a.vs[2];
    const T *kp = nullptr, *vp = nullptr;
    if (key < p.kn) {
        kp = (const T *)a.k + p.at.b * a.ks[0] + key * a.ks[1] + p.at.h * a.ks[2];
        vp = vb + key * a.vs[1];
    }
    const char *vt = lds + 2 * STAGE + wave * 32 * PITCH * 2;
    V8 kf[NK], vf[WIDE ? 1 : NK];
#pragma unroll
    for (int s = 0; s < NK; s++) kf[s] = row_operand<T>(kp, lane, s, a.d);
    if constexpr (WIDE) {
        Loads<PITCH, 128, 4> ld;
        ld.init(lane, wave, a.d);
        ld.rows(lds_address(lds + 2 * STAGE), (const char *)vb, a.vs[1] * 2, p.key0, p.kn);
    } else {
#pragma unroll
        for (int s = 0; s < NK; s++) vf[s] = row_operand<T>(vp, lane, s, a.d);
        settle(vf);
    }
    settle(kf);
    f16v dk[ND], dv[ND];
#pragma unroll
    for (int n = 0; n < ND; n++) dk[n] = dv[n] = zeros16();
    constexpr bool HALF = std::is_same<T, _Float16>::value;
    constexpr float BACK = Tile<T>::BACK;
    const float c = uniform(a.scale * LOG2E);
    float e = 0.f;
    if (HALF)
        e = uniform(attn_exponent(attn_row_size(a, p.pair, p.row / 64, (p.end + 63) / 64),
                                  attn_value_size(a, p.pair)));
    const float to_ds = exp2_hw(e - BACK);       // ds = (2^BACK p) (dp - delta) times this
    Operands<T, PITCH> op;
    op.init(lane);

    RowStages<PITCH, RT, 4> in;
    in.template init<T>(a, p.at, lane, wave, p.lo, p.hi, lds);
    // (a row with a NaN or an infinite query has it in its lse; one in its
    // gradient, in delta, but of dv only in its own column)
    if (CAUSAL) odd_init(odd);
    bool spoilt = false;
    const int block_from = p.seen(a, p.key0 + 127);
    if (p.row < p.end) in.fetch(a, p.row, 0);
    int stage = 0;
    for (int row = p.row; row < p.end; row += RT, stage ^= 1) {
        char *qt = lds + stage * STAGE, *ot = qt + TILE;
        const bool look = CAUSAL && row < block_from;
        if (look) {
            attn_landed();
            if (in.ld.template odd<T>(qt) || in.ld.template odd<T>(ot)) odd.tile[stage] = row;
        }
        attn_arrive();
        if (row + RT < p.end) in.fetch(a, row + RT, stage ^ 1);
        if (look && odd.tile[stage] == row) {
            in.ld.template mend<T>(qt, nullptr, 1, 0);
            in.ld.template mend<T>(ot, odd.least, -1, row);
            spoilt = true;
            __syncthreads();
        }
        if (WIDE) op.refresh();
#pragma unroll
        for (int b = 0; b < RT / 32; b++) {
            const int r = row + 32 * b;
            if (r + 32 <= wave_first) continue;
            if (WIDE) __builtin_amdgcn_s_setprio(1);
            f16v s = first_values((const float *)(ot + TILE) + b * 64, h32);
#pragma unroll
            for (int i = 0; i < NK; i++) s = Tile<T>::mul(op.along(qt, b, i), kf[i], s);
            f16v dp = first_values((const float *)(ot + TILE) + b * 64 + 32, h32);
#pragma unroll
            for (int i = 0; i < NK; i++)
                dp = Tile<T>::mul(op.along(ot, b, i), WIDE ? op.along(vt, 0, i) : vf[WIDE ? 0 : i],
                                  dp);
            float x[16], y[16];
#pragma unroll
            for (int i = 0; i < 16; i++) x[i] = exp2_hw(__builtin_fmaf(s[i], c, BACK));
            if (WIDE) {
                // 8 + 3 NK reads
                ATTN_GROUP(GROUP_READ, 4 + NK);
#pragma unroll
                for (int i = 0; i < NK / 2; i++) {
                    ATTN_GROUP(GROUP_MFMA, 1);
                    ATTN_GROUP(GROUP_READ, 1);
                }
#pragma unroll
                for (int i = 0; i < NK / 2; i++) {
                    ATTN_GROUP(GROUP_MFMA, 1);
                    ATTN_GROUP(GROUP_READ, 2);
                }
#pragma unroll
                for (int i = 0; i < NK; i++) {
                    ATTN_GROUP(GROUP_MFMA, 1);
                    ATTN_GROUP(GROUP_READ, 1);
                    ATTN_GROUP(GROUP_VALU, 4);
                }
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_setprio(0);
            }
#pragma unroll
            for (int i = 0; i < 16; i++) y[i] = x[i] * (HALF ? dp[i] * to_ds : dp[i]);
            if (r < wave_from) {
#pragma unroll
                for (int i = 0; i < 16; i++)
                    if (r + 8 * (i / 4) + 4 * h32 + i % 4 < from) x[i] = y[i] = 0.f;
            }
            // (rows behind the last, zeros, times an infinite key are NaNs)
            if (r + 32 > p.hi) {
#pragma unroll
                for (int i = 0; i < 16; i++)
                    if (r + 8 * (i / 4) + 4 * h32 + i % 4 >= p.hi) x[i] = y[i] = 0.f;
            }
            if (WIDE) __builtin_amdgcn_s_setprio(1);
            V8 pb[2], sb[2];
#pragma unroll
            for (int k = 0; k < 2; k++) {
                pb[k] = pack8<T>(x + 8 * k);
                sb[k] = pack8<T>(y + 8 * k);
            }
#pragma unroll
            for (int k = 0; k < 2; k++)
#pragma unroll
                for (int n = 0; n < ND; n++)
                    dv[n] = Tile<T>::mul(op.across(ot, 2 * b + k, n), pb[k], dv[n]);
#pragma unroll
            for (int k = 0; k < 2; k++)
#pragma unroll
                for (int n = 0; n < ND; n++)
                    dk[n] = Tile<T>::mul(op.across(qt, 2 * b + k, n), sb[k], dk[n]);
            if (WIDE) {
                ATTN_GROUP(GROUP_READ, 8);
#pragma unroll
                for (int i = 0; i < 4 * ND - 4; i++) {
                    ATTN_GROUP(GROUP_MFMA, 1);
                    ATTN_GROUP(GROUP_READ, 2);
                }
                ATTN_GROUP(GROUP_MFMA, 4);
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_setprio(0);
            }
        }
    }
    if (spoilt) odd_results<ND>(odd, h32, 1 - from, dv);
    store_keys<T, ND>(a, p, key, h32, dk, a.scale * exp2_hw(-e), false);
    store_keys<T, ND>(a, p, key, h32, dv, exp2_hw(-BACK), true);
}
// Adds up the ranges' gradients, always in the same order: four values a lane,
// dq's rows first, then dk and dv of each key.
template <typename T> __global__ __launch_bounds__(256) void attend_sums(AttnArgs a) {
    const int64_t pairs = (int64_t)a.b * a.hkv, rows = pairs * a.tq * a.group;
    const int64_t keys = pairs * a.tk;
    int64_t n = (int64_t)workgroup() * 256 + threadIdx.x;
    const int64_t dq = a.q_splits > 1 ? rows * (a.d / 4) : 0;
    const bool query = n < dq;
    if (!query) n -= dq;
    const int per = query ? a.d / 4 : a.d / 2, splits = query ? a.q_splits : a.row_splits;
    const int64_t i = n / per;
    if (!query && (a.row_splits < 2 || i >= keys)) return;
    int x = (int)(n - i * per) * 4;
    const float *p = (query ? a.part_q : a.part) + i * (4 * per) + x;
    const int64_t step = (query ? rows : keys) * (4 * per);
    f4 sum = (f4)(0.f);
#pragma unroll 8
    for (int s = 0; s < splits; s++) {
        f4 v;
        __builtin_memcpy(&v, p + s * step, 16);
        sum += v;
    }
    const float v[4] = {sum[0], sum[1], sum[2], sum[3]};
    const int64_t of = query ? a.tq * a.group : a.tk, pair = i / of, j = i - pair * of;
    const int64_t b = pair / a.hkv, h = pair - b * a.hkv;
    T *o;
    if (query) {
        const AttnRow row = attn_row(a, (int)j);
        o = (T *)a.dq + b * a.dqs[0] + row.t * a.dqs[1] + (h * a.group + row.g) * a.dqs[2];
    } else if (x < a.d) {
        o = (T *)a.dk + b * a.dks[0] + j * a.dks[1] + h * a.dks[2];
    } else {
        o = (T *)a.dv + b * a.dvs[0] + j * a.dvs[1] + h * a.dvs[2];
        x -= a.d;
    }
    store<T, 4>(o + x, v);
}

// dq: like the forward pass, 32 rows a wave, the keys 64 at a time.
template <typename T, int NK, int ND, bool CAUSAL>
__device__ __forceinline__ void attend_queries(const AttnArgs &a, char *lds, Odd &odd, int id) {
    typedef typename Tile<T>::V8 V8;
    constexpr int PITCH = NK <= 4 ? 64 : 128, KT = 64, TILE = KT * PITCH * 2;
    const int lane = threadIdx.x & 63, h32 = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const AttnPlace at = attn_place(a, a.tiles * a.q_splits, id);
    const int split = at.part % a.q_splits;
    const int tile = CAUSAL ? a.tiles - 1 - at.part / a.q_splits : at.part / a.q_splits;
    const int pair = at.b * a.hkv + at.h;
    const int qn = attn_length(a.qlen, at.b, a.tq), kn = attn_length(a.klen, at.b, a.tk);
    const int r0 = tile * 128, R = qn * a.group;
    const int first = r0 + wave * 32, r = first + (lane & 31);
    const AttnRow row = attn_row(a, r);
    auto sees = [&](int t) {
        if (!CAUSAL) return kn;
        const int n = t + kn - qn + 1;
        return n < 0 ? 0 : n > kn ? kn : n;
    };
    const int lim = r < R ? sees(row.t) : 0;
    const bool valid = lim > 0;
    const int least = sees(over_group(a, first)), block_least = sees(over_group(a, r0));
    const int last_row = r0 + 128 <= R ? r0 + 127 : R - 1;
    const int most = r0 < R ? sees(over_group(a, last_row)) : 0;
    const int wave_last = first + 32 <= R ? first + 31 : R - 1;
    const int wave_most = first < R ? sees(over_group(a, wave_last)) : 0;

    const int head = at.h * a.group + row.g;
    const T *qp = valid ? (const T *)a.q + at.b * a.qs[0] + row.t * a.qs[1] + head * a.qs[2]
                        : nullptr;
    const T *op_ = valid ? (const T *)a.dout + at.b * a.dos[0] + row.t * a.dos[1] +
                               head * a.dos[2]
                         : nullptr;
    V8 q[NK], g[NK];
#pragma unroll
    for (int s = 0; s < NK; s++) q[s] = row_operand<T>(qp, lane, s, a.d);
#pragma unroll
    for (int s = 0; s < NK; s++) g[s] = row_operand<T>(op_, lane, s, a.d);
    settle(q);
    settle(g);
    const float c = uniform(a.scale * LOG2E);
    float e = 0.f;
    if (std::is_same<T, _Float16>::value) {
        float size = 0.f;
#pragma unroll
        for (int s = 0; s < NK; s++)
#pragma unroll
            for (int i = 0; i < 8; i++) size += (float)g[s][i] * (float)g[s][i];
        size += other_half(size);
        e = attn_exponent(size < INF ? size : 0.f, attn_value_size(a, pair));
    }
    f16v acc[ND];
#pragma unroll
    for (int n = 0; n < ND; n++) acc[n] = zeros16();
    const float *st = a.stats + attn_stats(a, pair, r < a.row_tiles * 32 ? r : 0);
    const float first_s = valid ? st[0] : -INF, first_dp = valid ? st[32] : 0.f;

    KeyStages<PITCH, 4, false> in;
    in.template init<T>(a, at, lane, wave, kn, lds);
    Operands<T, PITCH> op;
    op.init(lane);
    int k0 = 0, k1 = most;
    if (a.q_splits > 1) {
        const int per = ((most + KT - 1) / KT + a.q_splits - 1) / a.q_splits * KT;
        k0 = split * per;
        if (k1 > k0 + per) k1 = k0 + per;
    }
    // A causal tile with a NaN or an infinity: a row that sees a NaN has it in
    // its lse, but an infinite key whose score is -infinity shows in nothing, so
    // scores are taken from the tile as it is, and the product with ds from a
    // copy with zeros.  (The copy stands in the other stage, whose tile is
    // loaded when all are done with it.)
    if (CAUSAL) odd_init(odd);
    bool spoilt = false;
    if (k0 < k1) in.fetch(k0, 0);
    int stage = 0;
    for (int key = k0; key < k1; key += KT, stage ^= 1) {
        char *kt = lds + stage * 2 * TILE, *vt = kt + TILE;
        const bool look = CAUSAL && key + KT > block_least;
        if (look) {
            attn_landed();
            if (in.ld.template odd<T>(kt)) odd.tile[stage] = key;
        }
        attn_arrive();
        const char *kc = kt;
        const bool apart = look && __builtin_amdgcn_readfirstlane(odd.tile[stage]) == key;
        if (apart) {
            char *copy = lds + (stage ^ 1) * 2 * TILE;
            in.ld.copy(copy, kt);
            in.ld.template mend<T>(copy, odd.least, 1, key);
            kc = copy;
            spoilt = true;
            __syncthreads();
        } else if (key + KT < k1) {
            in.fetch(key + KT, stage ^ 1);
        }
        if (key < wave_most) {
#pragma unroll
            for (int b = 0; b < 2; b++) {
                f16v s, dp;
                if (NK > 4) op.refresh();
                if (NK > 4) __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int i = 0; i < 16; i++) s[i] = first_s, dp[i] = first_dp;
#pragma unroll
                for (int i = 0; i < NK; i++) s = Tile<T>::mul(op.along(kt, b, i), q[i], s);
#pragma unroll
                for (int i = 0; i < NK; i++) dp = Tile<T>::mul(op.along(vt, b, i), g[i], dp);
                float ds[16];
#pragma unroll
                for (int i = 0; i < 16; i++) ds[i] = exp2_hw(__builtin_fmaf(s[i], c, e));
                if (NK > 4) {
                    ATTN_GROUP(GROUP_READ, 6);
#pragma unroll
                    for (int i = 0; i < NK; i++) {
                        ATTN_GROUP(GROUP_MFMA, 1);
                        ATTN_GROUP(GROUP_READ, 1);
                    }
#pragma unroll
                    for (int i = 0; i < NK; i++) {
                        ATTN_GROUP(GROUP_MFMA, 1);
                        ATTN_GROUP(GROUP_READ, 1);
                        ATTN_GROUP(GROUP_VALU, 4);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    __builtin_amdgcn_s_setprio(0);
                }
#pragma unroll
                for (int i = 0; i < 16; i++) ds[i] *= dp[i];
                if (key + KT > least) {
#pragma unroll
                    for (int i = 0; i < 16; i++)
                        if (key + b * 32 + 8 * (i / 4) + 4 * h32 + i % 4 >= lim) ds[i] = 0.f;
                }
                if (NK > 4) __builtin_amdgcn_s_setprio(1);
                V8 sb[2];
#pragma unroll
                for (int k = 0; k < 2; k++) sb[k] = pack8<T>(ds + 8 * k);
#pragma unroll
                for (int k = 0; k < 2; k++)
#pragma unroll
                    for (int n = 0; n < ND; n++)
                        acc[n] = Tile<T>::mul(op.across(kc, 2 * b + k, n), sb[k], acc[n]);
                if (NK > 4) {
                    ATTN_GROUP(GROUP_READ, 8);
#pragma unroll
                    for (int i = 0; i < 2 * ND - 4; i++) {
                        ATTN_GROUP(GROUP_MFMA, 1);
                        ATTN_GROUP(GROUP_READ, 2);
                    }
                    ATTN_GROUP(GROUP_MFMA, 4);
                    __builtin_amdgcn_sched_barrier(0);
                    __builtin_amdgcn_s_setprio(0);
                }
            }
        }
        if (apart) {
            __syncthreads();
            if (key + KT < k1) in.fetch(key + KT, stage ^ 1);
        }
    }
    if (spoilt) odd_results<ND>(odd, h32, lim, acc);
    if (r >= a.tq * a.group) return;
    const float back = a.scale * exp2_hw(-e);
    if (a.q_splits > 1) {
        float *o = a.part_q + (((int64_t)split * a.b * a.hkv + pair) * a.tq * a.group + r) * a.d;
#pragma unroll
        for (int n = 0; n < ND; n++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int i = n * 32 + j * 8 + 4 * h32;
                f4 v;
#pragma unroll
                for (int x = 0; x < 4; x++) v[x] = valid ? acc[n][4 * j + x] * back : 0.f;
                if (i < a.d) __builtin_memcpy(o + i, &v, 16);
            }
        return;
    }
    T *o = (T *)a.dq + at.b * a.dqs[0] + row.t * a.dqs[1] + head * a.dqs[2];
#pragma unroll
    for (int n = 0; n < ND; n++)
        store_result<T>(o, valid ? acc[n] : zeros16(), back, n, h32, a.d);
}

// Few rows and keys, up to 64 each (a map of 7 x 7): a workgroup takes a
// sequence's key head whole.  Four waves take 32 rows by 32 keys of p and ds
// each, and with both in LDS as operands every product of the gradients: five
// in all, and what attn_rows finds is found on the way, so one launch does it.
// Its chain is one load, two exchanges of the workgroup and the stores.  64 maps
// of 7 x 7, 8 heads of 64: 20 us by the general kernels, 10 by this.
template <typename T, int NK, int ND>
__global__ __launch_bounds__(256, NK <= 4 ? 2 : 1) void attend_backward_small(AttnArgs a) {
    typedef typename Tile<T>::V8 V8;
    constexpr int PITCH = NK <= 4 ? 64 : 128, TILE = 64 * PITCH * 2, PT = 64 * 64 * 2;
    constexpr bool HALF = std::is_same<T, _Float16>::value;
    constexpr float BACK = Tile<T>::BACK;
    __shared__ __attribute__((aligned(16))) char lds[4 * TILE + 3 * PT + 2048];
    __shared__ Odd odd, odd_keys;
    char *qt = lds, *ot = lds + TILE, *kt = lds + 2 * TILE, *vt = lds + 3 * TILE;
    char *pt = lds + 4 * TILE, *st = pt + PT, *dt = st + PT;    // p^T, ds^T, ds
    float *first = (float *)(dt + PT), *delta = first + 64, *dsize = first + 128,
          *vsize = first + 192, *to_dq = first + 256;
    const int lane = threadIdx.x & 63, h32 = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const AttnPlace at = attn_place(a, 1, blockIdx.x);
    const int qn = attn_length(a.qlen, at.b, a.tq), kn = attn_length(a.klen, at.b, a.tk);
    const int lo = a.causal && qn > kn ? (qn - kn) * a.group : 0, hi = kn ? qn * a.group : 0;
    const T *kb = (const T *)a.k + at.b * a.ks[0] + at.h * a.ks[2];
    const T *vb = (const T *)a.v + at.b * a.vs[0] + at.h * a.vs[2];
    const T *qb = (const T *)a.q + at.b * a.qs[0] + at.h * a.group * a.qs[2];
    const T *gb = (const T *)a.dout + at.b * a.dos[0] + at.h * a.group * a.dos[2];
    const T *ob = (const T *)a.o + at.b * a.os[0] + at.h * a.group * a.os[2];
    if (a.causal) {
        odd_init(odd);
        odd_init(odd_keys);
    }
    Loads<PITCH, 64, 4> ld;
    ld.init(lane, wave, a.d);
    ld.queries(a, lds_address(qt), (const char *)qb, a.qs[1] * 2, a.qs[2] * 2, 0, lo, hi);
    ld.queries(a, lds_address(ot), (const char *)gb, a.dos[1] * 2, a.dos[2] * 2, 0, lo, hi);
    ld.rows(lds_address(kt), (const char *)kb, a.ks[1] * 2, 0, kn);
    ld.rows(lds_address(vt), (const char *)vb, a.vs[1] * 2, 0, kn);
    {
        // four lanes a row and a key
        const int r = threadIdx.x >> 2, part = threadIdx.x & 3;
        const AttnRow row = attn_row(a, r);
        const bool valid = r >= lo && r < hi;
        float dot = 0.f, size = 0.f, value = 0.f, lse = -INF;
        if (valid)
            lse = a.lse[((int64_t)at.b * a.hq + at.h * a.group + row.g) * a.tq + row.t];
#pragma unroll
        for (int i = 0; i < PITCH / 32; i++) {
            const int e = (part + 4 * i) * 8;
            if (e < a.d && valid) {
                float x[8], y[8];
                load<T, 8>(gb + row.t * a.dos[1] + row.g * a.dos[2] + e, x);
                load<T, 8>(ob + row.t * a.os[1] + row.g * a.os[2] + e, y);
#pragma unroll
                for (int j = 0; j < 8; j++) dot += x[j] * y[j], size += x[j] * x[j];
            }
            if (HALF && e < a.d && r < kn) {
                float x[8];
                load<T, 8>(vb + r * a.vs[1] + e, x);
#pragma unroll
                for (int j = 0; j < 8; j++) value += x[j] * x[j];
            }
        }
#pragma unroll
        for (int o = 1; o < 4; o *= 2) {
            dot += __shfl_xor(dot, o);
            size += __shfl_xor(size, o);
            value += __shfl_xor(value, o);
        }
        if (part == 0) {
            const bool in = !(lse == -INF);
            first[r] = in ? -lse / a.scale : -INF;
            delta[r] = in ? -dot : 0.f;
            dsize[r] = size < INF ? size : 0.f;
            vsize[r] = value < INF ? value : 0.f;
        }
    }
    if (a.causal) {
        attn_landed();
        if (ld.template odd<T>(qt) || ld.template odd<T>(ot) || ld.template odd<T>(kt))
            odd.tile[0] = 0;
    }
    attn_arrive();
    const bool spoilt = a.causal && odd.tile[0] == 0;
    // exponents of the sequence's ds, and of row `lane`'s for dq (what the
    // products take from 2^BACK p, for each wave by itself)
    float e = 0.f, row_e = 0.f, to_dk = 1.f;
    if (HALF) {
        const float size = dsize[lane], value = wave_max(vsize[lane]);
        e = uniform(attn_exponent(wave_max(size), value));
        row_e = attn_exponent(size, value);
        to_dk = exp2_hw(e - BACK);
        to_dq += wave * 64;
        to_dq[lane] = exp2_hw(row_e - BACK);
    }
    const float c = uniform(a.scale * LOG2E);
    Operands<T, PITCH> op;
    Operands<T, 64> pop;
    op.init(lane);
    pop.init(lane);
    {
        const int kblock = wave & 1, rblock = wave >> 1;
        f16v s = first_values(first + 32 * rblock, h32);
        f16v dp = first_values(delta + 32 * rblock, h32);
#pragma unroll
        for (int i = 0; i < NK; i++)
            s = Tile<T>::mul(op.along(qt, rblock, i), op.along(kt, kblock, i), s);
#pragma unroll
        for (int i = 0; i < NK; i++)
            dp = Tile<T>::mul(op.along(ot, rblock, i), op.along(vt, kblock, i), dp);
        const int key = 32 * kblock + (lane & 31);
        int from = 0;
        if (a.causal) {
            const int t = key - (kn - qn);
            from = t < 0 ? 0 : t * a.group;
        }
        if (key >= kn) from = 64;
        float x[16], y[16], z[16];
        f16v rows;
        if (HALF) rows = first_values(to_dq + 32 * rblock, h32);
#pragma unroll
        for (int i = 0; i < 16; i++) {
            x[i] = exp2_hw(__builtin_fmaf(s[i], c, BACK));
            const int at = 32 * rblock + 8 * (i / 4) + 4 * h32 + i % 4;
            // (rows behind the last, zeros, times an infinite key are NaNs)
            if (at < from || at >= hi) x[i] = 0.f;
            const float none = x[i] == 0.f ? 0.f : dp[i];
            y[i] = x[i] * (HALF ? none * to_dk : none);
            z[i] = HALF ? x[i] * (none * rows[i]) : y[i];
        }
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const V8 p = pack8<T>(x + 8 * k), d = pack8<T>(y + 8 * k), r8 = pack8<T>(z + 8 * k);
            const u4 pu = __builtin_bit_cast(u4, p), du = __builtin_bit_cast(u4, d);
#pragma unroll
            for (int j = 0; j < 2; j++) {
                // rows 32 rblock + 16 k + 8 j + 4 h32 ..
                const int piece = 4 * rblock + 2 * k + j;
                const int to = key * 128 + ((piece ^ swizzle<64>(key)) << 4) + 8 * h32;
                *(u2 *)(pt + to) = u2{pu[2 * j], pu[2 * j + 1]};
                *(u2 *)(st + to) = u2{du[2 * j], du[2 * j + 1]};
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int r = 32 * rblock + 16 * k + 8 * j + 4 * h32 + i;
                    *(T *)(dt + r * 128 + ((key / 8 ^ swizzle<64>(r)) << 4) + key % 8 * 2) =
                        r8[4 * j + i];
                }
            }
        }
    }
    if (spoilt) {
        __syncthreads();
        ld.template mend<T>(qt, nullptr, 1, 0);
        ld.template mend<T>(ot, odd.least, -1, 0);
        ld.template mend<T>(kt, odd_keys.least, 1, 0);
    }
    __syncthreads();
    const int block = wave & 1, half = wave >> 1;
    const int x = 32 * block + (lane & 31);      // the lane's key, and row
    const float row_back = HALF ? exp2_hw(-__shfl(row_e, x)) : 1.f;
    const AttnRow row = attn_row(a, x);
    V8 pf[4], sf[4], df[4];
#pragma unroll
    for (int s = 0; s < 4; s++) {
        pf[s] = pop.along_result(pt, block, s, h32);
        sf[s] = pop.along_result(st, block, s, h32);
        df[s] = pop.along_result(dt, block, s, h32);
    }
    const bool valid = x >= lo && x < hi;
    T *dkp = (T *)a.dk + at.b * a.dks[0] + x * a.dks[1] + at.h * a.dks[2];
    T *dvp = (T *)a.dv + at.b * a.dvs[0] + x * a.dvs[1] + at.h * a.dvs[2];
    T *dqp = (T *)a.dq + at.b * a.dqs[0] + row.t * a.dqs[1] +
             (at.h * a.group + row.g) * a.dqs[2];
#pragma unroll
    for (int n = 0; n < ND; n++) {
        if ((n & 1) != half) continue;
        f16v dv = zeros16(), dk = zeros16(), dq = zeros16();
#pragma unroll
        for (int s = 0; s < 4; s++) {
            dv = Tile<T>::mul(op.across(ot, s, n), pf[s], dv);
            dk = Tile<T>::mul(op.across(qt, s, n), sf[s], dk);
            dq = Tile<T>::mul(op.across(kt, s, n), df[s], dq);
        }
        if (spoilt) {
            const int t = x - (kn - qn), from = t < 0 ? 0 : t * a.group;
            const int lim = row.t + kn - qn + 1;
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int e = n * 32 + 8 * (i / 4) + 4 * h32 + i % 4;
                if (odd.least[e] < 1 - from) dv[i] = __builtin_nanf("");
                if (odd_keys.least[e] < lim) dq[i] = __builtin_nanf("");
            }
        }
        if (x < a.tk) {
            store_result<T>(dvp, x < kn ? dv : zeros16(), exp2_hw(-BACK), n, h32, a.d);
            store_result<T>(dkp, x < kn ? dk : zeros16(), a.scale * exp2_hw(-e), n, h32, a.d);
        }
        if (x < a.tq * a.group)
            store_result<T>(dqp, valid ? dq : zeros16(), a.scale * row_back, n, h32, a.d);
    }
}

// Both in one launch, so that workgroups of the second kind fill the CUs that
// those of the first, which take longer, leave idle at their end.  800 of each
// kind on 512 places (2 x 3136, 16 heads of 128): 400 and 270 us apart, 590 to 620
// together.  (Apart, dq first, where dk or dv is written over the keys or
// values: those of the second kind read all of them, those of the first their
// own.)
template <typename T, int NK, int ND, bool CAUSAL>
__global__ __launch_bounds__(256, 2) void attend_backward(AttnArgs a) {
    constexpr int Q = 256 * (NK <= 4 ? 64 : 128) * 2, K = KeyTiles<NK>::BYTES;
    __shared__ __attribute__((aligned(16))) char lds[Q > K ? Q : K];
    __shared__ Odd odd;
    const int keys = a.b * a.hkv * a.key_tiles * a.row_splits;
    if ((int)blockIdx.x < keys) attend_keys<T, NK, ND, CAUSAL>(a, lds, odd);
    else attend_queries<T, NK, ND, CAUSAL>(a, lds, odd, blockIdx.x - keys);
}

// ------------------------------------------------------------------- host

static int64_t ceil_of(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Multiplier and shift of the group: r / G = (r * gmul >> 32) >> gshift for
// r < 2^31, with gmul = ceil(2^(31 + l) / G), 2^l >= G.
static void attn_group(AttnArgs &a) {
    a.group = a.hq / a.hkv;
    int l = 0;
    while ((1 << l) < a.group) l++;
    a.gmul = l ? (uint32_t)((((uint64_t)1 << (31 + l)) + a.group - 1) / a.group) : 0;
    a.gshift = l ? l - 1 : 0;
}
// Gradients of which a workgroup takes a sequence's key head whole.
static bool attn_small(const AttnArgs &a) {
    return (int64_t)a.tq * a.group <= 64 && a.tk <= 64;
}
// How a call is cut up.  Ranges of keys or rows, where the tiles alone would
// leave CUs idle: as many as give two workgroups a CU, of four steps of 64 at
// least (a range writes sums of fp32, which a second launch adds up).
static int64_t attn_ranges(int64_t workgroups, int64_t steps) {
    const int64_t s = workgroups ? 512 / workgroups : 1;
    const int64_t n = s < steps / 4 ? s : steps / 4;
    return n < 1 ? 1 : n;
}
// waves of a workgroup; forward: tiles of rows, ranges of keys of `per`;
// backward: tiles of rows and keys, their ranges of keys and rows
struct AttnPlan { int waves, tiles, splits, per, row_splits, q_splits; };
static AttnPlan attn_plan(const AttnArgs &a, bool backward) {
    AttnPlan p;
    const int64_t rows = (int64_t)a.tq * a.group, pairs = (int64_t)a.b * a.hkv;
    p.waves = rows <= 32 && !backward ? 1 : 4;
    p.tiles = (int)ceil_of(rows, p.waves * 32);
    const int64_t steps = ceil_of(a.tk, 64), n = attn_ranges(pairs * p.tiles, steps);
    p.per = (int)(ceil_of(steps, n) * 64);
    p.splits = a.tk ? (int)ceil_of(a.tk, p.per) : 1;
    p.q_splits = (int)n;
    p.row_splits = (int)attn_ranges(pairs * ceil_of(a.tk, 128), ceil_of(rows, 64));
    return p;
}
// Floats of the backward pass's workspace: what attn_rows writes, sums of dk
// and dv, sums of dq.
struct AttnSpace { int64_t stats, bounds, keys, queries; };
static AttnSpace attn_space(const AttnArgs &a, const AttnPlan &p) {
    const int64_t rows = (int64_t)a.tq * a.group, pairs = (int64_t)a.b * a.hkv;
    AttnSpace s;
    s.stats = pairs * ceil_of(rows, 64) * 128;
    s.bounds = (pairs * (ceil_of(rows, 64) + ceil_of(a.tk, 64)) + 3) / 4 * 4;
    s.keys = p.row_splits > 1 ? p.row_splits * pairs * a.tk * 2 * a.d : 0;
    s.queries = p.q_splits > 1 ? p.q_splits * pairs * rows * a.d : 0;
    return s;
}
size_t attention_workspace(const AttnArgs &in, bool backward) {
    AttnArgs a = in;
    attn_group(a);
    const int64_t rows = (int64_t)a.tq * a.group, pairs = (int64_t)a.b * a.hkv;
    const AttnPlan p = attn_plan(a, backward);
    if (backward) {
        if (attn_small(a)) return 0;
        const AttnSpace s = attn_space(a, p);
        return (size_t)((s.stats + s.bounds + s.keys + s.queries) * 4);
    }
    if (p.splits == 1) return 0;
    return (size_t)(p.splits * pairs * rows * (a.d + 1) * 4);
}

// A head's size in steps of 16 and 32 values, as the kernels are compiled.
template <template <typename, int, int> class L, typename T>
static hipError_t by_head(const AttnArgs &a, hipStream_t st) {
    if (a.d <= 32) return L<T, 2, 1>::go(a, st);
    if (a.d <= 64) return L<T, 4, 2>::go(a, st);
    if (a.d <= 96) return L<T, 6, 3>::go(a, st);
    return L<T, 8, 4>::go(a, st);
}
template <template <typename, int, int> class L>
static hipError_t by_form(const AttnArgs &a, hipStream_t st) {
    return a.type == F16 ? by_head<L, _Float16>(a, st) : by_head<L, __bf16>(a, st);
}

template <typename T, int NK, int ND> struct Attend {
    static hipError_t go(const AttnArgs &a, hipStream_t st) {
        const dim3 grid((unsigned)((int64_t)a.b * a.hkv * a.tiles * a.splits));
        return a.causal ? go<true>(a, grid, st) : go<false>(a, grid, st);
    }
    template <bool C> static hipError_t go(const AttnArgs &a, dim3 grid, hipStream_t st) {
        if (a.waves == 1) return start(attend<T, NK, ND, 1, C>, grid, 64, st, a);
        return start(attend<T, NK, ND, 4, C>, grid, 256, st, a);
    }
};
template <typename T, int NK, int ND> struct AttendBackward {
    static hipError_t go(const AttnArgs &a, hipStream_t st) {
        const int64_t pairs = (int64_t)a.b * a.hkv;
        if (attn_small(a))
            return start(attend_backward_small<T, NK, ND>, dim3((unsigned)pairs), 256, st, a);
        const int64_t keys = pairs * a.key_tiles * a.row_splits;
        const int64_t queries = pairs * a.tiles * a.q_splits;
        hipError_t e = hipSuccess;
        if (a.keys_last) {
            AttnArgs first = a;
            first.key_tiles = 0;
            e = both(first, queries, st);
            if (e == hipSuccess) e = both(a, keys, st);
        } else {
            e = both(a, keys + queries, st);
        }
        const int64_t lanes = (a.q_splits > 1 ? pairs * a.tq * a.group * (a.d / 4) : 0) +
                              (a.row_splits > 1 ? pairs * a.tk * (a.d / 2) : 0);
        if (e == hipSuccess && lanes)
            e = start(attend_sums<T>, grid_of(ceil_of(lanes, 256)), 256, st, a);
        return e;
    }
    static hipError_t both(const AttnArgs &a, int64_t wgs, hipStream_t st) {
        const dim3 grid((unsigned)wgs);
        if (!wgs) return hipSuccess;
        return a.causal ? start(attend_backward<T, NK, ND, true>, grid, 256, st, a)
                        : start(attend_backward<T, NK, ND, false>, grid, 256, st, a);
    }
};

hipError_t launch_attention(const AttnArgs &in, hipStream_t st) {
    AttnArgs a = in;
    attn_group(a);
    const AttnPlan p = attn_plan(a, false);
    const int64_t rows = (int64_t)a.tq * a.group, pairs = (int64_t)a.b * a.hkv;
    a.waves = p.waves; a.tiles = p.tiles; a.splits = p.splits; a.per = p.per;
    a.part = a.ws;
    a.part_lse = a.ws + p.splits * pairs * rows * a.d;
    const hipError_t e = by_form<Attend>(a, st);
    if (e != hipSuccess || p.splits == 1) return e;
    const dim3 join = grid_of(ceil_of(pairs * rows * (a.d / 4), 256));
    return a.type == F16 ? start(attend_join<_Float16>, join, 256, st, a)
                         : start(attend_join<__bf16>, join, 256, st, a);
}

hipError_t launch_attention_backward(const AttnArgs &in, hipStream_t st) {
    AttnArgs a = in;
    attn_group(a);
    const int64_t rows = (int64_t)a.tq * a.group, pairs = (int64_t)a.b * a.hkv;
    a.row_tiles = (int)ceil_of(rows, 64) * 2;
    a.q_chunks = (int)ceil_of(rows, 64);
    a.v_chunks = a.type == F16 ? (int)ceil_of(a.tk, 64) : 0;
    a.tiles = (int)ceil_of(rows, 128);
    a.key_tiles = (int)ceil_of(a.tk, 128);
    const AttnPlan p = attn_plan(a, true);
    const AttnSpace s = attn_space(a, p);
    a.row_splits = p.row_splits;
    a.q_splits = p.q_splits;
    a.stats = a.ws;
    a.bounds = a.stats + s.stats;
    a.part = a.bounds + s.bounds;
    a.part_q = a.part + s.keys;
    hipError_t e = hipSuccess;
    if (!attn_small(a) && a.q_chunks + a.v_chunks) {
        const dim3 grid((unsigned)(pairs * (a.q_chunks + a.v_chunks)));
        e = a.type == F16 ? start(attn_rows<_Float16>, grid, 256, st, a)
                          : start(attn_rows<__bf16>, grid, 256, st, a);
    }
    return e == hipSuccess ? by_form<AttendBackward>(a, st) : e;
}

}  // namespace ops
}  // namespace ctc
