// 8-bit floating point (e4m3, e5m2) with a scale for each block: 1 or 128
// rows by 128 columns of the matrix as the product reads it,
//   s = max(amax, 2^-100) / MAX,   q = round(x * (MAX / max(amax, 2^-100))).
// 2^-100 keeps MAX / amax finite; a block of zeros gets zeros.  A NaN or an
// infinity spoils its whole block (its scale is NaN or infinite, and what
// is not NaN in it is 0), so the product shows it.
// What bounds it: the bytes (2 or 4 in and 1 out for each value).  6272 x 320
// fp16 takes 3.8 us, the transpose of 8192 x 4096 bf16 23.6 (4.3 TB/s).  A block
// stays in registers between its largest value and its rounding, so x is read
// once; a transpose turns in LDS as bytes, after the rounding.
#pragma once
#include "ops_device.h"

namespace ctc {
namespace ops {

// The largest magnitude of values, as fp32 bits: NaN above infinity above
// every number.
__device__ __forceinline__ uint32_t mag(float v) {
    return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu;
}
struct Scale { float s, inv; };
__device__ __forceinline__ Scale scale_of(uint32_t amax, float most) {
    constexpr uint32_t LEAST = 0x0d800000u;      // 2^-100
    const float a = __builtin_bit_cast(float, amax < LEAST ? LEAST : amax);
    return Scale{a / most, most / a};
}
template <int Q> __device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    int r = 0;
    if constexpr (Q == E4M3) {
        r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, r, false);
        r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
    } else {
        r = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, r, false);
        r = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, r, true);
    }
    return (uint32_t)r;
}
template <int Q> constexpr float most_of() { return Q == E4M3 ? 448.f : 57344.f; }

// V consecutive values of a row from column c on, zero past `cols`.
template <typename T, int V>
__device__ __forceinline__ void load_row(const T *row, int64_t c, int64_t cols, float (&v)[V]) {
    if (c + V <= cols) {
        load<T, V>(row + c, v);
        return;
    }
#pragma unroll
    for (int e = 0; e < V; e++) v[e] = c + e < cols ? widen(row[c + e]) : 0.f;
}

// Blocks of one row: eight values a thread, 16 threads a block, 16 rows of
// one block column a workgroup.
template <typename T, int Q>
__global__ __launch_bounds__(256) void quantize_rows(QuantArgs a, int64_t rtiles) {
    const int64_t kb = blockIdx.x / rtiles;
    const int64_t r = blockIdx.x % rtiles * 16 + (threadIdx.x >> 4);
    const int64_t c = kb * 128 + (threadIdx.x & 15) * 8;
    float v[8] = {};
    if (r < a.rows) load_row<T, 8>((const T *)a.x + r * a.ldx, c, a.cols, v);
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; e++) m = mag(v[e]) > m ? mag(v[e]) : m;
#pragma unroll
    for (int o = 8; o; o >>= 1) {
        const uint32_t b = __shfl_xor(m, o);
        m = b > m ? b : m;
    }
    if (r >= a.rows) return;
    const Scale s = scale_of(m, most_of<Q>());
    if ((threadIdx.x & 15) == 0) a.scales[kb * a.lds + r] = s.s;
    // (up to the next 16 columns: zeros, as v holds there)
    if (c < (a.cols + 15) / 16 * 16) {
        u2 q;
        q[0] = pack4<Q>(v[0] * s.inv, v[1] * s.inv, v[2] * s.inv, v[3] * s.inv);
        q[1] = pack4<Q>(v[4] * s.inv, v[5] * s.inv, v[6] * s.inv, v[7] * s.inv);
        *(u2 *)(a.q + r * a.ldq + c) = q;
    }
}

// A 128 x 128 tile of x by a workgroup of 256 threads: thread (g, l) =
// (tid / 16, tid % 16) holds rows g, g + 16, .. and columns 8 l .. 8 l + 7.
// TR: x is read as its transpose, whose rows are x's columns; the tile turns
// in LDS (rows of 128 + 4 bytes).  SQ: one scale for the tile.
template <typename T, int Q, bool TR, bool SQ>
__global__ __launch_bounds__(256) void quantize_tile(QuantArgs a, int64_t ctiles) {
    constexpr int ROW = 132;
    __shared__ __attribute__((aligned(16))) union {
        uint32_t amax[16][128];
        uint8_t q[128 * ROW];
    } l;
    __shared__ float inv[128];
    const int64_t r0 = blockIdx.x / ctiles * 128, c0 = blockIdx.x % ctiles * 128;
    const int g = threadIdx.x >> 4, lane = threadIdx.x & 15;
    float v[8][8];
    uint32_t m[8] = {};
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const int64_t r = r0 + g + i * 16;
        if (r < a.rows) load_row<T, 8>((const T *)a.x + r * a.ldx, c0 + lane * 8, a.cols, v[i]);
        else
#pragma unroll
            for (int e = 0; e < 8; e++) v[i][e] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < 8; i++)
#pragma unroll
        for (int e = 0; e < 8; e++) m[e] = mag(v[i][e]) > m[e] ? mag(v[i][e]) : m[e];
#pragma unroll
    for (int e = 0; e < 8; e++) l.amax[g][lane * 8 + e] = m[e];
    __syncthreads();
    if (threadIdx.x < 128) {
        uint32_t t = 0;
        for (int i = 0; i < 16; i++) {
            const uint32_t b = l.amax[i][threadIdx.x];
            t = b > t ? b : t;
        }
        if constexpr (SQ) {
#pragma unroll
            for (int o = 32; o; o >>= 1) {
                const uint32_t b = __shfl_xor(t, o);
                t = b > t ? b : t;
            }
            if ((threadIdx.x & 63) == 0) inv[threadIdx.x >> 6] = __builtin_bit_cast(float, t);
        } else {
            const Scale s = scale_of(t, most_of<Q>());
            inv[threadIdx.x] = s.inv;
            if (c0 + threadIdx.x < a.cols)
                a.scales[r0 / 128 * a.lds + c0 + threadIdx.x] = s.s;
        }
    }
    __syncthreads();
    float f[8];
    if constexpr (SQ) {
        const uint32_t t0 = __builtin_bit_cast(uint32_t, inv[0]);
        const uint32_t t1 = __builtin_bit_cast(uint32_t, inv[1]);
        const Scale s = scale_of(t0 > t1 ? t0 : t1, most_of<Q>());
        if (threadIdx.x == 0)
            a.scales[TR ? r0 / 128 * a.lds + c0 / 128 : c0 / 128 * a.lds + r0 / 128] = s.s;
#pragma unroll
        for (int e = 0; e < 8; e++) f[e] = s.inv;
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) f[e] = inv[lane * 8 + e];
    }
    if constexpr (!TR) {
        const int64_t c = c0 + lane * 8, end = (a.cols + 15) / 16 * 16;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int64_t r = r0 + g + i * 16;
            if (r < a.rows && c < end) {
                u2 q;
                q[0] = pack4<Q>(v[i][0] * f[0], v[i][1] * f[1], v[i][2] * f[2], v[i][3] * f[3]);
                q[1] = pack4<Q>(v[i][4] * f[4], v[i][5] * f[5], v[i][6] * f[6], v[i][7] * f[7]);
                *(u2 *)(a.q + r * a.ldq + c) = q;
            }
        }
        return;
    }
    // (amax read out: the last barrier)
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const uint32_t lo = pack4<Q>(v[i][0] * f[0], v[i][1] * f[1], v[i][2] * f[2], v[i][3] * f[3]);
        const uint32_t hi = pack4<Q>(v[i][4] * f[4], v[i][5] * f[5], v[i][6] * f[6], v[i][7] * f[7]);
#pragma unroll
        for (int e = 0; e < 4; e++) {
            l.q[(lane * 8 + e) * ROW + g + i * 16] = (uint8_t)(lo >> (8 * e));
            l.q[(lane * 8 + 4 + e) * ROW + g + i * 16] = (uint8_t)(hi >> (8 * e));
        }
    }
    __syncthreads();
    // rows of the transpose: 8 threads of 16 bytes each
    const int64_t end = (a.rows + 15) / 16 * 16;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int row = i * 32 + (threadIdx.x >> 3), at = (threadIdx.x & 7) * 16;
        if (c0 + row < a.cols && r0 + at < end) {
            u4 q;
            for (int e = 0; e < 4; e++) q[e] = *(const uint32_t *)(l.q + row * ROW + at + e * 4);
            *(u4 *)(a.q + (c0 + row) * a.ldq + r0 + at) = q;
        }
    }
}

hipError_t launch_quantize(const QuantArgs &a, hipStream_t st) {
    if (a.rows == 0 || a.cols == 0) return hipSuccess;
    return by_type(a.type, [&](auto tag) {
        typedef typename decltype(tag)::type T;
        const int64_t kb = (a.cols + 127) / 128, rb = (a.rows + 127) / 128;
        auto go = [&](auto qc) {
            constexpr int Q = decltype(qc)::value;
            if (!a.transpose && a.block_rows == 1) {
                const int64_t rt = (a.rows + 15) / 16;
                return start(quantize_rows<T, Q>, dim3((unsigned)(rt * kb)), 256, st, a, rt);
            }
            const dim3 grid((unsigned)(rb * kb));
            if (!a.transpose) return start(quantize_tile<T, Q, false, true>, grid, 256, st, a, kb);
            if (a.block_rows == 1)
                return start(quantize_tile<T, Q, true, false>, grid, 256, st, a, kb);
            return start(quantize_tile<T, Q, true, true>, grid, 256, st, a, kb);
        };
        return a.qtype == E4M3 ? go(std::integral_constant<int, E4M3>())
                               : go(std::integral_constant<int, E5M2>());
    });
}

}  // namespace ops
}  // namespace ctc
