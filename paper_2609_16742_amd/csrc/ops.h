// Internal launcher interface of the operators around a protected
// classifier: group norm, the 8-bit quantiser and product, the scores of
// given tokens.  Not part of the C ABI.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace ctc {
namespace ops {

// Element types, with the values of ctc_dtype.
enum Type { F32 = 0, F16 = 1, BF16 = 2, E4M3 = 3, E5M2 = 4 };
enum Act { ACT_NONE = 0, ACT_RELU = 1, ACT_SILU = 2 };

inline int type_bytes(int t) { return t == F32 ? 4 : t <= BF16 ? 2 : 1; }

struct NormArgs {
    int type;
    int64_t n, hw;
    int c, groups, carry, act;
    float eps;
    const void *x, *residual, *dy;
    const float *gamma, *beta;   // [c] or null (1 and 0)
    void *y, *dx, *dresidual;
    float *mean, *rstd;          // [n][groups]; read by the backward pass
    float *dgamma, *dbeta;       // [c] or null
    float *ws;
};
// Bytes of a.ws a launch needs for a's type and sizes.
size_t norm_workspace(const NormArgs &a, bool backward);
hipError_t launch_norm_forward(const NormArgs &a, hipStream_t st);
hipError_t launch_norm_backward(const NormArgs &a, hipStream_t st);

struct QuantArgs {
    int type, qtype;
    int64_t rows, cols, ldx;     // of x
    int transpose, block_rows;
    const void *x;
    uint8_t *q;
    int64_t ldq;
    float *scales;
    int64_t lds;
};
hipError_t launch_quantize(const QuantArgs &a, hipStream_t st);

struct ProductArgs {
    int atype, btype, ytype, act;
    int64_t m, n, k;
    const uint8_t *a, *b;
    int64_t lda, ldb, ldy;
    const float *sa, *sb;        // [ceil(k/128)][ldsa], [..][ldsb]
    int64_t ldsa, ldsb;
    int a_block, b_block;        // rows of one scale: 1 or 128
    const float *bias;           // [n] or null
    void *y;
    float *ws;                   // partial sums [splits][m][n]
};
// Bytes of a.ws a product needs (partial sums of a split k).
size_t product_workspace(const ProductArgs &a);
hipError_t launch_product(const ProductArgs &a, hipStream_t st);

struct ScoreArgs {
    int type;
    int64_t rows, ld, ldd;
    int vocab, top_k;
    const void *x;
    const int32_t *target;       // [rows] or null
    float *lse, *logprob, *entropy;
    int32_t *rank, *ids;         // [rows], [rows][top_k]
    float *tops;                 // [rows][top_k]
    const float *g_lse, *g_logprob, *g_entropy;
    void *dx;
    void *ws;
};
constexpr int SCORES_MAX_K = 32;
size_t scores_workspace(const ScoreArgs &a);
hipError_t launch_scores(const ScoreArgs &a, hipStream_t st);
hipError_t launch_scores_backward(const ScoreArgs &a, hipStream_t st);

}  // namespace ops
}  // namespace ctc
