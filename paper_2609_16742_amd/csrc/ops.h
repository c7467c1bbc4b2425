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

struct AttnArgs {
    int type, b, tq, tk, hq, hkv, d, causal;
    float scale;
    const void *q, *k, *v, *dout;
    void *o;                     // read by the backward pass
    float *lse;                  // [b][hq][tq], as o
    // strides in elements: sequence, token, head
    int64_t qs[3], ks[3], vs[3], os[3], dos[3], dqs[3], dks[3], dvs[3];
    const int32_t *qlen, *klen;  // [b] or null
    void *dq, *dk, *dv;
    float *ws;
    int keys_last;               // dk or dv is k or v: dq in a launch before
    // set by the launchers
    int group, gshift, waves, tiles, splits, per, row_tiles, key_tiles, q_chunks, v_chunks, row_splits, q_splits;
    uint32_t gmul;
    float *part, *part_lse, *part_q, *stats, *bounds;
};
constexpr int ATTN_MAX_D = 128;
size_t attention_workspace(const AttnArgs &a, bool backward);
hipError_t launch_attention(const AttnArgs &a, hipStream_t st);
hipError_t launch_attention_backward(const AttnArgs &a, hipStream_t st);

struct HeadSide {                // queries or keys
    const void *x, *dy;
    void *y, *dx;
    const float *weight;         // [d] or null
    float *dweight;              // [d] or null
    int heads;                   // 0: none
    int64_t xs[3], ys[3], dys[3], dxs[3];        // sequence, token, head
};
struct HeadArgs {
    int type, ytype;             // of x and dx, of y and dy
    int b, t, d, norm, interleaved, n_axes, turned, per_image;
    int axes[4];                 // pairs turned by each; their sum is `turned`
    float eps;
    HeadSide side[2];
    const int32_t *positions;    // [b or 1][t][n_axes]
    const float *frequencies;    // [turned]
    float *ws;
    // set by the launcher
    int lanes, tokens;
};
bool head_norm_ok(const HeadArgs &a);            // its heads fit a wave
size_t head_norm_workspace(const HeadArgs &a);   // of the backward pass
hipError_t launch_head_norm(const HeadArgs &a, bool backward, hipStream_t st);

// Tensors of one launch, in chunks: those of tensor i are first[i] ..
// first[i + 1] - 1.
constexpr int CLIP_TENSORS = 96;
struct ClipTable {
    const void *x[CLIP_TENSORS];
    void *y[CLIP_TENSORS];
    int64_t size[CLIP_TENSORS];
    uint32_t first[CLIP_TENSORS + 1];
    uint8_t type[CLIP_TENSORS];
    int n;
};
int64_t clip_chunks_of(int64_t size);
int clip_parts(const ClipTable &t);              // partial sums of a launch
hipError_t launch_clip_squares(const ClipTable &t, double *part, hipStream_t st);
hipError_t launch_clip_scale(const ClipTable &t, const double *part, int parts, double max_norm,
                             float *norm, hipStream_t st);

}  // namespace ops
}  // namespace ctc
