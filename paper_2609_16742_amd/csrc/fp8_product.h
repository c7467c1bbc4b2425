// Matrix product in 8-bit floating point with a scale for each block of 128:
//   y[m][n] = act(sum over blocks kb of sa[kb][m'] sb[kb][n'] *
//                 sum over k in kb of a[m][k] b[n][k]  + bias[n])
// with m' = m or m / 128, n' = n or n / 128.  A block is summed on the matrix
// unit, its result scaled and added in fp32, so every scale counts exactly
// where it belongs.  Two ways to sum a block:
//  - one 16x16x128 8-bit MFMA.  The unit lines eight products (of eight
//    values of k in a row) up with the largest exponent among them and drops,
//    towards zero, what lies more than 13 bits below it (measured: 2^16 + 2^3
//    arrives, of 2^16 + 2^2 only 2^16; the eights are added in 24 bits).  An
//    eight so loses less than 7 * 2^-13 of its largest product.  Error of 512
//    x 512 x 4096 against what rounding the exact result leaves: normal values
//    2.08e-4 of 2.08e-4 (fp16), one outlier of 300 deviations in each block
//    2.13e-4 of 2.05e-4, of 1000 2.17e-4 of 2.06e-4; bf16 1.65e-3 of 1.65e-3
//    in all of them.  The 8-bit values themselves stand for others to 2^-4, so
//    16-bit results are summed like this, at the 8-bit rate;
//  - four 16x16x32 bf16 MFMAs on the widened values (exact, as are their
//    products), at half the rate but with fp32 sums: fp32 results.
//
// b's rows (filters) are the MFMA's first operand: a lane ends up with four
// consecutive n of one m.  A lane's 32 values of k are two 16-byte chunks g
// and g + 4 (g = lane / 16) of the block's 128 bytes, the same in a and b.
#pragma once
#include "ops_device.h"

namespace ctc {
namespace ops {

typedef __amdgpu_buffer_rsrc_t Buf;
constexpr int PAST = (int)0x80000000u;           // past every buffer: reads 0
typedef __attribute__((address_space(3))) void *LdsAt;

// One MFMA over a block of 128: rows from b (type FB), columns from a (FA).
template <int FA, int FB>
__device__ __forceinline__ f4 mfma_block(i8v b, i8v a) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
        b, a, (f4)(0.f), FB == E5M2 ? 1 : 0, FA == E5M2 ? 1 : 0, 0, 0, 0, 0);
}
// Two 16-byte chunks as one operand.
__device__ __forceinline__ i8v chunks(u4 lo, u4 hi) {
    i8v r;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        r[e] = (int)lo[e];
        r[e + 4] = (int)hi[e];
    }
    return r;
}
// The same sum in fp32: operands widened to bf16.
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
struct Wide { bf8v q[4]; };
template <int F> __device__ __forceinline__ Wide widen_block(i8v v) {
    Wide r;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        bf2 lo, hi;
        if constexpr (F == E4M3) {
            lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[i], 1.f, false);
            hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[i], 1.f, true);
        } else {
            lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(v[i], 1.f, false);
            hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(v[i], 1.f, true);
        }
        const int at = (i & 1) * 4;
        r.q[i >> 1][at] = lo[0];
        r.q[i >> 1][at + 1] = lo[1];
        r.q[i >> 1][at + 2] = hi[0];
        r.q[i >> 1][at + 3] = hi[1];
    }
    return r;
}
__device__ __forceinline__ f4 mfma_wide(const Wide &b, const Wide &a) {
    f4 d = (f4)(0.f);
#pragma unroll
    for (int i = 0; i < 4; i++)
        d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.q[i], a.q[i], d, 0, 0, 0);
    return d;
}
// The first `n` bytes of a chunk, the others zero (n may be < 0 or > 16).
__device__ __forceinline__ u4 first_bytes(u4 v, int n) {
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const int b = n - 4 * e;
        v[e] = b >= 4 ? v[e] : b <= 0 ? 0 : v[e] & ((1u << (8 * (b & 3))) - 1);
    }
    return v;
}

// The bias of four columns.
__device__ __forceinline__ f4 bias_of(const ProductArgs &p, int64_t n) {
    f4 b = (f4)(0.f);
#pragma unroll
    for (int e = 0; e < 4; e++)
        if (p.bias && n + e < p.n) b[e] = p.bias[n + e];
    return b;
}
// Four results of row m from column n on.
__device__ __forceinline__ void product_out(const ProductArgs &p, int64_t m, int64_t n, f4 v,
                                            f4 bias) {
    if (m >= p.m) return;
    v += bias;
    float w[4] = {v[0], v[1], v[2], v[3]};
    act_of<4>(p.act, w);
    const int64_t o = m * p.ldy + n;
    auto put = [&](auto *y) {
        typedef typename std::remove_pointer<decltype(y)>::type T;
        if (n + 4 <= p.n) store<T, 4>(y + o, w);
        else
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (n + e < p.n) y[o + e] = narrow<T>(w[e]);
    };
    if (p.ytype == F32) put((float *)p.y);
    else if (p.ytype == F16) put((_Float16 *)p.y);
    else put((__bf16 *)p.y);
}
// ... or as partial sums of range `split`.
__device__ __forceinline__ void partial_out(const ProductArgs &p, int split, int64_t m,
                                            int64_t n, f4 v) {
    if (m >= p.m) return;
    float *o = p.ws + ((int64_t)split * p.m + m) * p.n + n;
    if (n + 4 <= p.n) __builtin_memcpy(o, &v, 16);
    else
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (n + e < p.n) o[e] = v[e];
}

// ---------------------------------------------------------------------------
// Few rows of a: the filters are streamed once (for each 64 rows).  A
// workgroup of NW waves takes 16 filters and MT tiles of 16 rows; its waves
// take every NW-th block of k, each through a ring of R stages in LDS of its
// own (no barrier: a wave waits for its own loads), and add up at the end.  A
// stage holds the block's rows as product_tile's do, filters first, then
// their scales.
// What bounds it: the bytes of the filters, and how many are under way (R - 1
// stages of each wave): 32 rows, 4096 filters, k = 25088 in 21 to 28 us (4 to 5
// TB/s of filters).  Loading fragments straight into registers took as
// long for one row, but 41 us instead of 23 for 32 (k = 25088, 4096 filters):
// a load whose neighbouring lanes are in different rows keeps the address
// unit four times as long.
// ---------------------------------------------------------------------------
template <int MT, int FA, int FB, bool WIDE>
__global__ __launch_bounds__(MT < 4 ? 512 : 256) void product_rows(ProductArgs p, int nt,
                                                                   int splits, int per) {
    constexpr int NW = MT < 4 ? 8 : 4, R = MT == 1 ? 4 : 3;
    constexpr int ROWS = 16 * (1 + MT), STAGE = ROWS * 128 + 512;
    constexpr int LOADS = ROWS / 8 + 2;          // of a stage
    static_assert(NW * R * STAGE <= 160 * 1024 && NW * MT * 1024 <= NW * R * STAGE, "LDS");
    __shared__ __attribute__((aligned(16))) char lds[NW * R * STAGE];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int fr = lane & 15, fg = lane >> 4;
    const int split = blockIdx.x % splits, tile = blockIdx.x / splits;
    const int64_t n0 = (int64_t)(tile % nt) * 16, m0 = (int64_t)(tile / nt) * (16 * MT);
    const int nblocks = (int)((p.k + 127) / 128);
    const int kb0 = split * per, kb1 = kb0 + per < nblocks ? kb0 + per : nblocks;
    const int kend = (int)p.k;
    const int ma = p.m - m0 < 16 * MT ? (int)(p.m - m0) : 16 * MT;
    const int nb = p.n - n0 < 16 ? (int)(p.n - n0) : 16;
    const Buf ar = __builtin_amdgcn_make_buffer_rsrc((void *)(p.a + m0 * p.lda), 0,
                                                     (int)(ma * p.lda), 0x00020000);
    const Buf br = __builtin_amdgcn_make_buffer_rsrc((void *)(p.b + n0 * p.ldb), 0,
                                                     (int)(nb * p.ldb), 0x00020000);
    const int ash = p.a_block == 1 ? 0 : 7, bsh = p.b_block == 1 ? 0 : 7;
    const float *sab = p.sa + (m0 >> ash), *sbb = p.sb + (n0 >> bsh);
    // the scales' places: lane l for row l of a and filter l
    const int sai = lane < ma ? (int)(((m0 + lane) >> ash) - (m0 >> ash)) * 4 : 0;
    const int sbi = lane < nb ? (int)(((n0 + lane) >> bsh) - (n0 >> bsh)) * 4 : 0;
    const int lrow = lane >> 3, lchunk = ((lane & 7) ^ lrow) * 16;
    const int ao = lrow * (int)p.lda + lchunk, bo = lrow * (int)p.ldb + lchunk;
    char *ring = lds + wave * R * STAGE;
    auto issue = [&](int kb, int slot) {
        const bool on = kb < kb1;                // past the range: zeros
        const int k0 = kb * 128;
        const bool ok = on && k0 + lchunk < kend;
        const int av = ok ? ao + k0 : PAST, bv = ok ? bo + k0 : PAST;
        char *to = ring + slot * STAGE;
#pragma unroll
        for (int i = 0; i < 2; i++)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(br, (LdsAt)(to + i * 1024), 16,
                                                     bv + i * 8 * (int)p.ldb, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 2 * MT; i++)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ar, (LdsAt)(to + (i + 2) * 1024), 16,
                                                     av + i * 8 * (int)p.lda, 0, 0, 0);
        const int64_t q = on ? kb : 0;
        const Buf sar = __builtin_amdgcn_make_buffer_rsrc(
            (void *)(sab + q * p.ldsa), 0,
            on ? (int)(((m0 + ma - 1) >> ash) - (m0 >> ash) + 1) * 4 : 0, 0x00020000);
        const Buf sbr = __builtin_amdgcn_make_buffer_rsrc(
            (void *)(sbb + q * p.ldsb), 0,
            on ? (int)(((n0 + nb - 1) >> bsh) - (n0 >> bsh) + 1) * 4 : 0, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(sar, (LdsAt)(to + ROWS * 128), 4, sai, 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(sbr, (LdsAt)(to + ROWS * 128 + 256), 4, sbi, 0,
                                                 0, 0);
    };
    f4 acc[MT];
#pragma unroll
    for (int j = 0; j < MT; j++) acc[j] = (f4)(0.f);
    const int c0 = (fg ^ (fr & 7)) * 16, c1 = ((fg + 4) ^ (fr & 7)) * 16;
    auto block = [&](int kb, int slot) {
        const char *at = ring + slot * STAGE + fr * 128;
        // the block k ends in, in the middle of 16 bytes
        const bool ragged = (kb + 1) * 128 > kend && (kend & 15);
        const int left = kend - kb * 128 - fg * 16;
        auto frag = [&](int tile) {
            u4 lo = *(const u4 *)(at + tile * 2048 + c0), hi = *(const u4 *)(at + tile * 2048 + c1);
            if (ragged) {
                lo = first_bytes(lo, left);
                hi = first_bytes(hi, left - 64);
            }
            return chunks(lo, hi);
        };
        const float *sc = (const float *)(ring + slot * STAGE + ROWS * 128);
        const f4 sb = *(const f4 *)(sc + 64 + fg * 4);
        const i8v w = frag(0);
#pragma unroll
        for (int j = 0; j < MT; j++) {
            const i8v x = frag(1 + j);
            const float s = sc[j * 16 + fr];
            if constexpr (WIDE)
                acc[j] += mfma_wide(widen_block<FB>(w), widen_block<FA>(x)) * (sb * s);
            else
                acc[j] += mfma_block<FA, FB>(w, x) * (sb * s);
        }
    };
    int kb = kb0 + wave;
#pragma unroll
    for (int r = 0; r < R - 1; r++) issue(kb + r * NW, r);
    int slot = 0;
    for (; kb < kb1; kb += NW) {
        const int fill = slot == 0 ? R - 1 : slot - 1;   // the one read last
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        issue(kb + (R - 1) * NW, fill);
        // all but the loads of the R - 1 later stages
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((R - 1) * LOADS) : "memory");
        __builtin_amdgcn_sched_barrier(0);
        block(kb, slot);
        slot = slot == R - 1 ? 0 : slot + 1;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
    f4 *sum = (f4 *)lds;                         // [NW][MT][64]
#pragma unroll
    for (int j = 0; j < MT; j++) sum[(wave * MT + j) * 64 + lane] = acc[j];
    __syncthreads();
    for (int j = wave; j < MT; j += NW) {
        f4 t = sum[j * 64 + lane];
        for (int i = 1; i < NW; i++) t += sum[(i * MT + j) * 64 + lane];
        const int64_t m = m0 + j * 16 + fr;
        if (splits > 1) partial_out(p, split, m, n0 + fg * 4, t);
        else product_out(p, m, n0 + fg * 4, t, bias_of(p, n0 + fg * 4));
    }
}

// ---------------------------------------------------------------------------
// Tiles of BM rows of a by BN filters, WM x WN waves.  A step is one block
// of 128: its rows go from HBM into one of two LDS stages by the buffer
// unit (16 bytes a lane, 1 KB a wave instruction: eight rows back to back),
// the next step's while this one's MFMAs run.  Chunk g of row r is kept in
// slot g ^ (r & 7), which spreads the fragment reads over the banks.
// What bounds it: the matrix unit where the tiles fill the card (8192 x 4096 x
// 8192 to 16 bits in 234 us, 2.34 PFLOP/s, up to 260 us among launches of the
// same; to fp32, by 128 x 128 tiles, in 453; with a scale for each filter to
// fp32 in 555, to 16 bits in 452).
// ---------------------------------------------------------------------------
template <int BM, int BN, int WM, int WN, int FA, int FB, bool SB1, bool WIDE>
__global__ __launch_bounds__(64 * WM * WN, 2) void product_tile(ProductArgs p, int mt, int nt,
                                                             int splits, int per) {
    constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN;
    constexpr int IM = TM / 16, IN = TN / 16;
    constexpr int AR = BM / 8 / NW, BR = BN / 8 / NW;    // loads of a wave a step
    constexpr int STAGE = (BM + BN) * 128;
    constexpr int DQ = IN >= 8 ? 2 : 4;          // loads sent between two groups
    static_assert((AR + BR) % DQ == 0 && (AR + BR) / DQ <= IN, "loads");
    static_assert(AR * 8 * NW == BM && BR * 8 * NW == BN && 128 % TN == 0 && IN % 2 == 0, "tile");
    __shared__ __attribute__((aligned(16))) char lds[2 * STAGE];
    __shared__ __attribute__((aligned(16))) float sbl[3][SB1 ? BN : 4];
    // each XCD runs a contiguous range of tiles (workgroups go round the
    // eight XCDs), which goes down four tiles of rows, then along the filters:
    // 32 tiles at a time share 4 and 8 panels
    const int total = mt * nt * splits, share = (total + 7) / 8;
    int t = (blockIdx.x & 7) * share + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= share || t >= total) return;
    const int split = t / (mt * nt);
    t -= split * (mt * nt);
    const int group = t / (4 * nt), rows = mt - 4 * group < 4 ? mt - 4 * group : 4;
    t -= group * 4 * nt;
    const int64_t m0 = (int64_t)(4 * group + t % rows) * BM, n0 = (int64_t)(t / rows) * BN;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    const int fr = lane & 15, fg = lane >> 4;

    const int64_t ma = p.m - m0 < BM ? p.m - m0 : BM, nb = p.n - n0 < BN ? p.n - n0 : BN;
    const Buf ar = __builtin_amdgcn_make_buffer_rsrc((void *)(p.a + m0 * p.lda), 0,
                                                     (int)(ma * p.lda), 0x00020000);
    const Buf br = __builtin_amdgcn_make_buffer_rsrc((void *)(p.b + n0 * p.ldb), 0,
                                                     (int)(nb * p.ldb), 0x00020000);
    const int nblocks = (int)((p.k + 127) / 128);
    const int first = split * per;
    const int last = first + per < nblocks ? first + per : nblocks;
    const int lrow = wave * 8 + (lane >> 3);
    const int lchunk = ((lane & 7) ^ (lane >> 3)) * 16;
    const int ao = lrow * (int)p.lda + lchunk, bo = lrow * (int)p.ldb + lchunk;
    const int kend = (int)p.k;
    // Loads q0 .. q1 - 1 of a wave's AR + BR for a step (a tile's rows span
    // less than 2^31 bytes: PAST stays past the end with a row offset added)
    auto issue = [&](int step, int st, int q0, int q1) {
        const int k0 = step * 128;
        const bool ok = step < last && k0 + lchunk < kend;
        const int av = ok ? ao + k0 : PAST, bv = ok ? bo + k0 : PAST;
        const int arow = NW * 8 * (int)p.lda, brow = NW * 8 * (int)p.ldb;
#pragma unroll
        for (int q = q0; q < q1; q++) {
            char *to = lds + st * STAGE + (q * NW + wave) * 1024;
            if (q < AR)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(ar, (LdsAt)to, 16, av + q * arow, 0, 0,
                                                         0);
            else
                __builtin_amdgcn_raw_ptr_buffer_load_lds(br, (LdsAt)to, 16,
                                                         bv + (q - AR) * brow, 0, 0, 0);
        }
    };
    // scales: a's of a lane's IM columns; b's one of the wave's filters (a
    // wave's lie in one block of 128), or, SB1, the tile's through LDS
    const int ash = p.a_block == 1 ? 0 : 7, bsh = p.b_block == 1 ? 0 : 7;
    const float *sab = p.sa + (m0 >> ash), *sbb = p.sb + (n0 >> bsh);
    uint32_t sai[IM], sbi;
#pragma unroll
    for (int j = 0; j < IM; j++) {
        const int r = wm * TM + j * 16 + fr;
        sai[j] = (uint32_t)((((int64_t)(r < ma ? r : ma - 1) + m0) >> ash) - (m0 >> ash));
    }
    {
        const int r = SB1 ? (int)threadIdx.x % BN : wn * TN;
        sbi = (uint32_t)((((int64_t)(r < nb ? r : nb - 1) + n0) >> bsh) - (n0 >> bsh));
    }
    f4 acc[IN][IM], d[2][IM];
#pragma unroll
    for (int j = 0; j < IM; j++) {
#pragma unroll
        for (int i = 0; i < IN; i++) acc[i][j] = (f4)(0.f);
        d[1][j] = (f4)(0.f);
    }
    float sa[IM] = {}, san[IM] = {}, sbn = 0.f;
    auto scales = [&](int step) {
#pragma unroll
        for (int j = 0; j < IM; j++) san[j] = (sab + step * p.ldsa)[sai[j]];
        sbn = (sbb + step * p.ldsb)[sbi];
    };
    // The last block of a k that is no multiple of 16: zeros behind the end
    // in the 16 bytes it lies in (a and b: what stands there may be NaN).
    auto blank = [&](int st) {
        const int c = (kend & 127) >> 4;
        for (int r = threadIdx.x; r < BM + BN; r += 64 * NW) {
            u4 *v = (u4 *)(lds + st * STAGE + r * 128 + ((c ^ (r & 7)) << 4));
            *v = first_bytes(*v, kend & 15);
        }
        __syncthreads();
    };
    auto arrived = [&]() {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
    };
    const int c0 = (fg ^ (fr & 7)) * 16, c1 = ((fg + 4) ^ (fr & 7)) * 16;
    const int abase = (wm * TM + fr) * 128, bbase = BM * 128 + (wn * TN + fr) * 128;
    auto frag = [&](int at) {
        return chunks(*(const u4 *)(lds + at + c0), *(const u4 *)(lds + at + c1));
    };
    typedef typename std::conditional<WIDE, Wide, i8v>::type Frag;
    auto afrag = [&](int at) -> Frag {
        if constexpr (WIDE) return widen_block<FA>(frag(at));
        else return frag(at);
    };
    auto bfrag = [&](i8v v) -> Frag {
        if constexpr (WIDE) return widen_block<FB>(v);
        else return v;
    };
    Frag x[IM];
    i8v w;
    // A step: IN groups of IM MFMAs.  The results of a group are scaled and
    // added while the next group's MFMAs run, and the next filter fragment
    // is read.  The one barrier stands before the last group: by then every
    // wave has read this stage out, so the step after next goes into it, and
    // the next step's rows have arrived; the last group's MFMAs hide the
    // reads of the next step's first fragments.  Loads go out a few at a time
    // between the groups: a wave's MFMAs wait behind a load that finds the
    // address unit busy (16 clocks for each load of eight waves).
    if (first < last) {
        issue(first, 0, 0, AR + BR);
        scales(first);
        if constexpr (SB1)
            if (threadIdx.x < BN) {
                sbl[0][threadIdx.x] = sbn;
                // (the scales of no step, which the first step multiplies its
                // zeros by: what LDS held may be NaN)
                sbl[2][threadIdx.x] = 0.f;
            }
        arrived();
        issue(first + 1, 1, 0, DQ);
    }
    auto begin = [&](int cur) {
#pragma unroll
        for (int j = 0; j < IM; j++) x[j] = afrag(cur + abase + j * 2048);
        w = frag(cur + bbase);
    };
    begin(0);
    int slot = 0;                                // of sbl: step modulo 3
    const bool ragged = (kend & 15) && last == nblocks && first < last;
    int step = first, stop = ragged ? last - 1 : last;
    for (;;) {
    for (; step < stop; step++) {
        const int cur = ((step - first) & 1) * STAGE, nxt = STAGE - cur;
        const int before = slot == 0 ? 2 : slot - 1, after = slot == 2 ? 0 : slot + 1;
        float sp[IM];                            // the scales of the step before
#pragma unroll
        for (int j = 0; j < IM; j++) {
            sp[j] = sa[j];
            sa[j] = SB1 ? san[j] : san[j] * sbn;
        }
        scales(step + 1 < last ? step + 1 : step);
#pragma unroll
        for (int i = 0; i < IN; i++) {
            const bool end = i == IN - 1;
            if (end) {
                if constexpr (SB1)
                    if (threadIdx.x < BN) sbl[after][threadIdx.x] = sbn;
                arrived();
            }
            // the stage that the barrier freed: DQ loads a group
            const int q = end ? 0 : (i + 1) * DQ;
            if (q < AR + BR) issue(step + (end ? 2 : 1), end == (cur != 0), q, q + DQ);
            const Frag wf = bfrag(w);
            if (!end) w = frag(cur + bbase + (i + 1) * 2048);
            f4 s4 = (f4)(1.f);
            if constexpr (SB1)
                s4 = *(const f4 *)(sbl[i ? slot : before] + wn * TN + (i ? i - 1 : IN - 1) * 16 +
                                   fg * 4);
#pragma unroll
            for (int j = 0; j < IM; j++) {
                if constexpr (WIDE) d[i & 1][j] = mfma_wide(wf, x[j]);
                else d[i & 1][j] = mfma_block<FA, FB>(wf, x[j]);
                if (end) x[j] = afrag(nxt + abase + j * 2048);
            }
            if (end) w = frag(nxt + bbase);
#pragma unroll
            for (int j = 0; j < IM; j++) {
                f4 &r = d[(i & 1) ^ 1][j];
                if constexpr (SB1) r *= s4;
                acc[i ? i - 1 : IN - 1][j] += r * (i ? sa[j] : sp[j]);
            }
            if constexpr (WIDE) {
                __builtin_amdgcn_sched_barrier(0);
            } else {
#pragma unroll
                for (int j = 0; j < IM; j++) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // MFMA
                    if (end) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);   // LDS reads
                    __builtin_amdgcn_sched_group_barrier(0x002, SB1 ? 8 : 4, 0);   // VALU
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        slot = after;
    }
    if (stop == last) break;
    // (its stage has arrived; its first fragments are read again)
    blank((step - first) & 1);
    begin(((step - first) & 1) * STAGE);
    stop = last;
    }
    {
        const int before = slot == 0 ? 2 : slot - 1;
        f4 s4 = (f4)(1.f);
        if constexpr (SB1) s4 = *(const f4 *)(sbl[before] + wn * TN + (IN - 1) * 16 + fg * 4);
#pragma unroll
        for (int j = 0; j < IM; j++) {
            if constexpr (SB1) d[1][j] *= s4;
            if (first < last) acc[IN - 1][j] += d[1][j] * sa[j];
        }
    }
    // The results go through LDS, each wave's through its own part of the
    // stages, piece g of row r in place g ^ (r & 15): a lane holds four
    // columns of one of 16 rows, from where a store would write 16 pieces of
    // a line, and the code that writes would stand here IN x IM times.
    constexpr int PART = 2 * STAGE / NW, LINE = TN / 4;   // bytes; pieces of a row
    constexpr int HELD = PART / (TN * 4) < TM ? PART / (TN * 4) : TM;
    static_assert(HELD % 16 == 0 && TM % HELD == 0 && LINE <= 64, "rows held");
    arrived();                                   // (loads past the range wrote zeros)
    f4 *held = (f4 *)(lds + wave * PART);
    const int64_t n = n0 + wn * TN + lane % LINE * 4;
    const f4 bias = splits > 1 ? (f4)(0.f) : bias_of(p, n);
#pragma unroll
    for (int h = 0; h < TM / HELD; h++) {
#pragma unroll
        for (int j = 0; j < HELD / 16; j++)
#pragma unroll
            for (int i = 0; i < IN; i++)
                held[(j * 16 + fr) * LINE + ((i * 4 + fg) ^ fr)] = acc[i][h * (HELD / 16) + j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll 2
        for (int t = 0; t < HELD * LINE / 64; t++) {
            const int q = t * (64 / LINE) + lane / LINE;
            const f4 v = held[q * LINE + (lane % LINE ^ (q & 15))];
            const int64_t m = m0 + wm * TM + h * HELD + q;
            if (n >= p.n) continue;
            if (splits > 1) partial_out(p, split, m, n, v);
            else product_out(p, m, n, v, bias);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// ---------------------------------------------------------------------------
// 128 x 128 tiles with three steps of loads under way: a ring of four LDS
// stages (rows as in product_tile, then the scales of the 128 rows and the
// 128 filters), one workgroup of 2 x 4 waves a CU.  Every wave sends as many
// loads a step, so a wait for all but the last two steps' is a count.
// What bounds it: a step takes 0.75 us (to fp32 1.15), more than half of it to
// fill and read 128 KB of LDS at 128 bytes a clock, and the latency of the
// first loads.  2048 x 2048 x 2048 to 16 bits in 20 us, to fp32 in 29.
// ---------------------------------------------------------------------------
template <int FA, int FB, bool WIDE>
__global__ __launch_bounds__(512) void product_ring(ProductArgs p, int mt, int nt, int splits,
                                                    int per) {
    constexpr int B = 128, S = 4, IM = 4, IN = 2, TM = 64, TN = 32;
    constexpr int STAGE = 2 * B * 128 + 2 * B * 4, LOADS = 5;
    __shared__ __attribute__((aligned(16))) char lds[S * STAGE];
    static_assert(B * B * 4 <= S * STAGE, "results");
    // each XCD runs a contiguous range of tiles (workgroups go round them)
    const int total = mt * nt * splits, share = (total + 7) / 8;
    int t = (blockIdx.x & 7) * share + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= share || t >= total) return;
    const int split = t / (mt * nt);
    t -= split * (mt * nt);
    const int64_t m0 = (int64_t)(t % mt) * B, n0 = (int64_t)(t / mt) * B;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave & 1, wn = wave >> 1;
    const int fr = lane & 15, fg = lane >> 4;
    const int ma = p.m - m0 < B ? (int)(p.m - m0) : B, nb = p.n - n0 < B ? (int)(p.n - n0) : B;
    const Buf ar = __builtin_amdgcn_make_buffer_rsrc((void *)(p.a + m0 * p.lda), 0,
                                                     (int)(ma * p.lda), 0x00020000);
    const Buf br = __builtin_amdgcn_make_buffer_rsrc((void *)(p.b + n0 * p.ldb), 0,
                                                     (int)(nb * p.ldb), 0x00020000);
    const int nblocks = (int)((p.k + 127) / 128), kend = (int)p.k;
    const int first = split * per, last = first + per < nblocks ? first + per : nblocks;
    const int lrow = wave * 8 + (lane >> 3), lchunk = ((lane & 7) ^ (lane >> 3)) * 16;
    const int ao = lrow * (int)p.lda + lchunk, bo = lrow * (int)p.ldb + lchunk;
    // the scales' quarter of this wave (waves 4 .. 7 send the same again):
    // rows 0 .. 63, 64 .. 127, filters 0 .. 63, 64 .. 127
    const int part = wave & 3, srow = (part & 1) * 64 + lane;
    const int sh = (part < 2 ? p.a_block : p.b_block) == 1 ? 0 : 7;
    const int64_t s0 = part < 2 ? m0 : n0;
    const int rows = part < 2 ? ma : nb;
    const float *sbase = (part < 2 ? p.sa : p.sb) + (s0 >> sh);
    const int64_t sld = part < 2 ? p.ldsa : p.ldsb;
    const int sbytes = (int)(((s0 + rows - 1) >> sh) - (s0 >> sh) + 1) * 4;
    const int si = srow < rows ? (int)(((s0 + srow) >> sh) - (s0 >> sh)) * 4 : 0;
    auto issue = [&](int step, int slot) {
        const bool on = step < last;             // past the range: zeros
        const int k0 = step * 128;
        const bool ok = on && k0 + lchunk < kend;
        const int av = ok ? ao + k0 : PAST, bv = ok ? bo + k0 : PAST;
        char *to = lds + slot * STAGE;
#pragma unroll
        for (int q = 0; q < 2; q++)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ar, (LdsAt)(to + (q * 8 + wave) * 1024), 16,
                                                     av + q * 64 * (int)p.lda, 0, 0, 0);
#pragma unroll
        for (int q = 0; q < 2; q++)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                br, (LdsAt)(to + B * 128 + (q * 8 + wave) * 1024), 16,
                bv + q * 64 * (int)p.ldb, 0, 0, 0);
        const Buf sr = __builtin_amdgcn_make_buffer_rsrc(
            (void *)(sbase + (on ? step : 0) * sld), 0, on ? sbytes : 0, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(sr, (LdsAt)(to + 2 * B * 128 + part * 256), 4,
                                                 si, 0, 0, 0);
    };
    f4 acc[IN][IM];
#pragma unroll
    for (int i = 0; i < IN; i++)
#pragma unroll
        for (int j = 0; j < IM; j++) acc[i][j] = (f4)(0.f);
    const int c0 = (fg ^ (fr & 7)) * 16, c1 = ((fg + 4) ^ (fr & 7)) * 16;
    typedef typename std::conditional<WIDE, Wide, i8v>::type Frag;
#pragma unroll
    for (int q = 0; q < S - 1; q++) issue(first + q, q);
    int slot = 0;
    for (int step = first; step < last; step++) {
        __builtin_amdgcn_sched_barrier(0);
        // this step's loads of the wave have arrived, and its reads of the
        // step before, whose stage is filled next
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((S - 2) * LOADS) : "memory");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        issue(step + S - 1, (slot + S - 1) % S);
        char *at = lds + slot * STAGE;
        if ((step + 1) * 128 > kend && (kend & 15)) {
            // k ends in the middle of 16 bytes: zeros behind it
            if (threadIdx.x < 2 * B) {
                const int row = threadIdx.x, c = (kend & 127) >> 4;
                u4 *v = (u4 *)(at + row * 128 + ((c ^ (row & 7)) << 4));
                *v = first_bytes(*v, kend & 15);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
        }
        auto frag = [&](int row) {
            return chunks(*(const u4 *)(at + row * 128 + c0), *(const u4 *)(at + row * 128 + c1));
        };
        const float *sc = (const float *)(at + 2 * B * 128);
        Frag x[IM];
        float sa[IM];
#pragma unroll
        for (int j = 0; j < IM; j++) {
            const i8v v = frag(wm * TM + j * 16 + fr);
            if constexpr (WIDE) x[j] = widen_block<FA>(v);
            else x[j] = v;
            sa[j] = sc[wm * TM + j * 16 + fr];
        }
#pragma unroll
        for (int i = 0; i < IN; i++) {
            const i8v w = frag(B + wn * TN + i * 16 + fr);
            const f4 sb = *(const f4 *)(sc + B + wn * TN + i * 16 + fg * 4);
            if constexpr (WIDE) {
                const Wide ww = widen_block<FB>(w);
#pragma unroll
                for (int j = 0; j < IM; j++) acc[i][j] += mfma_wide(ww, x[j]) * (sb * sa[j]);
            } else {
#pragma unroll
                for (int j = 0; j < IM; j++)
                    acc[i][j] += mfma_block<FA, FB>(w, x[j]) * (sb * sa[j]);
            }
        }
        slot = (slot + 1) % S;
    }
    // The results through LDS, for whole lines (see product_tile)
    constexpr int LINE = B / 4;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
    f4 *held = (f4 *)lds;
#pragma unroll
    for (int j = 0; j < IM; j++)
#pragma unroll
        for (int i = 0; i < IN; i++)
            held[(wm * TM + j * 16 + fr) * LINE + ((wn * (TN / 4) + i * 4 + fg) ^ fr)] =
                acc[i][j];
    __syncthreads();
    const int64_t n = n0 + threadIdx.x % LINE * 4;
    if (n >= p.n) return;
    const f4 bias = splits > 1 ? (f4)(0.f) : bias_of(p, n);
#pragma unroll 2
    for (int h = 0; h < B * LINE / 512; h++) {
        const int q = h * (512 / LINE) + (int)threadIdx.x / LINE;
        const f4 v = held[q * LINE + ((int)threadIdx.x % LINE ^ (q & 15))];
        if (splits > 1) partial_out(p, split, m0 + q, n, v);
        else product_out(p, m0 + q, n, v, bias);
    }
}

// Adds the ranges' partial sums, in order: four results a thread.
static __global__ __launch_bounds__(256) void product_join(ProductArgs p, int splits) {
    const int64_t nq = (p.n + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= p.m * nq) return;
    const int64_t m = i / nq, n = i % nq * 4;
    f4 t = (f4)(0.f);
    for (int s = 0; s < splits; s++) {
        const float *o = p.ws + ((int64_t)s * p.m + m) * p.n + n;
        f4 v = (f4)(0.f);
        if (n + 4 <= p.n) __builtin_memcpy(&v, o, 16);
        else
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (n + e < p.n) v[e] = o[e];
        t += v;
    }
    product_out(p, m, n, t, bias_of(p, n));
}

// How a product runs.  Kinds: product_rows; product_tile of 128 x 128 or of
// 256 x 256; product_ring.
enum { ROWS, TILE, BIG_TILE, RING };
struct ProductPlan { int kind, mt, nt, splits, per; };
static ProductPlan product_plan(const ProductArgs &a) {
    ProductPlan r{};
    const int64_t nb = (a.k + 127) / 128;
    auto done = [&](int64_t s) {
        s = s < 1 ? 1 : s > 16 ? 16 : s;
        r.per = (int)((nb + s - 1) / s);
        r.splits = r.per ? (int)((nb + r.per - 1) / r.per) : 1;
        return r;
    };
    // Short products too go to product_rows, whose waves have several blocks
    // under way: 214 x 102 x 2912 in 8 us instead of 14, 10807 x 10 x 5933 in
    // 15 instead of 22; at 3467 x 120 x 4227 (14520 below) it takes 26, tiles 18.
    const int64_t few = ((a.m + 63) / 64) * ((a.n + 15) / 16);
    if (a.m <= 64 || (few <= 512 && few * nb <= 8192)) {
        r.kind = ROWS;
        r.mt = a.m <= 16 ? 1 : a.m <= 32 ? 2 : 4;
        r.nt = (int)((a.n + 15) / 16);
        // blocks of a range: eight a wave, joining costs as much as reading
        // them
        const int64_t s = few ? 256 / few : 1, most = nb / (r.mt < 4 ? 64 : 32);
        return done(s < most ? s : most);
    }
    const bool wide = a.ytype == F32;
    // 256 x 256 tiles, one a CU, from 192 on (bf16, k = 4096: 3584 x 3584, 196
    // tiles, 58 us, in 128 x 128 tiles 75; 4096 x 4096 66 and 81; 8192 x 4096
    // 133 and 163; below, 2816 x 2816, 121 tiles, 54 and 43).  Near the limit
    // and just past a whole round the others win or lose by more than the rule
    // sees: 3328 x 3328, 169 tiles, 56 and 66; 4352 x 4096, 272, 112 and 100.
    const int64_t big = ((a.m + 255) / 256) * ((a.n + 255) / 256);
    if (!wide && a.b_block > 1 && big >= 192) {
        r.kind = BIG_TILE;
        r.mt = (int)((a.m + 255) / 256);
        r.nt = (int)((a.n + 255) / 256);
        return done(1);
    }
    r.mt = (int)((a.m + 127) / 128);
    r.nt = (int)((a.n + 127) / 128);
    const int64_t tiles = (int64_t)r.mt * r.nt;
    // Ranges of k: a step takes `one` us where a CU has one workgroup, `two`
    // where it has two; adding the ranges up takes 4 us and the time of
    // writing and reading them at 4 TB/s.  (Within 10% of the times of 1 to
    // 16 ranges at sizes from 1024 x 1024 x 1024 to 256 x 4096 x 25088.)
    const double one = wide ? 1.15 : a.b_block > 1 ? 0.75 : 1.25;
    const double two = wide ? 1.9 : a.b_block > 1 ? 0.75 : 1.3;
    double best = 0;
    int64_t s = 1;
    for (int64_t t = 1; t <= 16 && t * 2 <= nb + 1; t++) {
        const int64_t wgs = tiles * t;
        const double us =
            (double)((nb + t - 1) / t) *
                (wgs <= 256 ? one : two * (double)((wgs + 511) / 512)) +
            (t > 1 ? 4 + (double)t * (double)a.m * (double)a.n * 8 / 4e6 : 0);
        if (t == 1 || us < best) {
            best = us;
            s = t;
        }
    }
    // product_ring where a CU has one workgroup (fp32: 1280 x 320 x 6272 in
    // 23 us, tiles 25; 2048 x 2048 x 2048 in 29, tiles 32), for 16-bit results
    // only of the whole k (16384 x 64 x 576 in 9.4 us, tiles 10.5; 3467 x 120 x
    // 4227 in four ranges 18.0, tiles 17.2)
    r.kind = tiles * s <= 256 && (wide || s == 1) ? RING : TILE;
    return done(s);
}
size_t product_workspace(const ProductArgs &a) {
    const ProductPlan r = product_plan(a);
    return r.splits > 1 ? (size_t)r.splits * a.m * a.n * 4 : 0;
}

template <int FA, int FB> static hipError_t product_go(const ProductArgs &a, hipStream_t st) {
    const ProductPlan r = product_plan(a);
    hipError_t e;
    if (r.kind == ROWS) {
        const dim3 grid((unsigned)((a.m + 16 * r.mt - 1) / (16 * r.mt) * r.nt * r.splits));
        auto rows = [&](auto wide) {
            constexpr bool W = decltype(wide)::value;
            auto go = [&](auto kernel, int threads) {
                return start(kernel, grid, threads, st, a, r.nt, r.splits, r.per);
            };
            return r.mt == 1   ? go(product_rows<1, FA, FB, W>, 512)
                   : r.mt == 2 ? go(product_rows<2, FA, FB, W>, 512)
                               : go(product_rows<4, FA, FB, W>, 256);
        };
        e = a.ytype == F32 ? rows(std::true_type()) : rows(std::false_type());
    } else {
        const unsigned g = ((unsigned)(r.mt * r.nt * r.splits) + 7) / 8 * 8;
        const bool s1 = a.b_block == 1;
        auto tile = [&](auto big, auto sb1, auto wide) {
            constexpr bool B = decltype(big)::value, S = decltype(sb1)::value,
                           W = decltype(wide)::value;
            if constexpr (B)
                return start(product_tile<256, 256, 4, 2, FA, FB, S, W>, dim3(g), 512, st, a,
                             r.mt, r.nt, r.splits, r.per);
            else
                return start(product_tile<128, 128, 2, 2, FA, FB, S, W>, dim3(g), 256, st, a,
                             r.mt, r.nt, r.splits, r.per);
        };
        typedef std::true_type Y;
        typedef std::false_type N;
        if (r.kind == RING) {
            auto ring = [&](auto wide) {
                return start(product_ring<FA, FB, decltype(wide)::value>, dim3(g), 512, st, a,
                             r.mt, r.nt, r.splits, r.per);
            };
            e = a.ytype == F32 ? ring(Y()) : ring(N());
        } else if (r.kind == BIG_TILE) {
            e = tile(Y(), N(), N());
        } else if (a.ytype == F32) {
            e = s1 ? tile(N(), Y(), Y()) : tile(N(), N(), Y());
        } else {
            e = s1 ? tile(N(), Y(), N()) : tile(N(), N(), N());
        }
    }
    if (e != hipSuccess || r.splits == 1) return e;
    const int64_t items = a.m * ((a.n + 3) / 4);
    return start(product_join, dim3((unsigned)((items + 255) / 256)), 256, st, a, r.splits);
}
hipError_t launch_product(const ProductArgs &a, hipStream_t st) {
    if (a.m == 0 || a.n == 0) return hipSuccess;
    if (a.atype == E4M3)
        return a.btype == E4M3 ? product_go<E4M3, E4M3>(a, st) : product_go<E4M3, E5M2>(a, st);
    return a.btype == E4M3 ? product_go<E5M2, E4M3>(a, st) : product_go<E5M2, E5M2>(a, st);
}

}  // namespace ops
}  // namespace ctc
