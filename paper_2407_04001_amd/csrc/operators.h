// Arguments of the layer operators, between the checks of operators.cpp (host)
// and the launches in the .hip file of each.
#pragma once

#include <cstdint>

#include "pase_operators.h"

namespace pase {

struct NormForward {
    int dtype, param_dtype;
    int64_t rows;
    int width;
    const void *x, *residual, *gain, *bias;
    void *y, *z;
    int64_t ldx, ldr, ldy, ldz;
    float *mean, *rstd;
    float eps;
};

struct NormBackward {
    int dtype, param_dtype;
    int64_t rows;
    int width;
    const void *dy, *z, *dz, *gain;
    const float *mean, *rstd;
    void *dx, *dgain, *dbias;
    int64_t lddy, ldz, lddz, lddx;
    float *partial;      // [blocks][2][width]: the blocks' sums of dgain and dbias
    int blocks;
};

struct SoftmaxLoss {
    int dtype, targets_64;
    int64_t rows, classes;
    const void *logits, *targets;
    int64_t ldl, ignore;
    const float *dloss;
    int64_t dloss_stride;
    float *loss, *lse;
    void *dlogits;
    int64_t lddl;
    float *low;          // what lse's rounding leaves, or null
};

// c[m][j] = sum over the contraction of a and b; see grouped_matmul.hip for
// what rows, n and k are in each direction.
struct GroupedProduct {
    int dtype, out_dtype, offsets_64;
    int64_t rows;
    int groups, n, k;    // w: groups x n x k
    const void *x, *w, *dy, *offsets;
    void *out;
    int64_t ldx, lddy, ldo;
    float *partial;      // weights gradient: [splits][groups][n][k] when splits > 1
    int splits;
    uint32_t first;      // of this launch, where several share the tiles: see launch_tiles()
};

// An argument [rows, heads, dim]: distances in elements.
struct HeadRows {
    void *p;
    int64_t ld, head_ld;
};

struct RowStats {
    float exponent, delta;   // lse log2 e (infinite where no key is seen) and out . dout, in fp16 lowered (kRaisedGrad in attention.hip)
};

struct Attention {
    int dtype, offsets_64, causal;
    int rows, key_rows, sequences, heads, kv_heads, dim;
    float scale;
    const void *q_offsets, *k_offsets, *k_lengths;
    HeadRows q, k, v, out, dout, dq, dk, dv;
    float *lse;          // [heads][rows]
    RowStats *stats;     // [heads][rows], for the second kernel of the backward pass
    float *partial;      // forward with splits > 1: [splits][rows x heads, up to a multiple of 4], then as many rows of dim, up to a multiple of 4
    int splits, tiles;   // splits: see attention_splits(); tiles: of the queries' (keys') rows, see tiles_of()
    int by_place;        // how tiles of keys are dealt, see Owner in attention.hip
    uint32_t first;
};

struct Rotary {
    int dtype, positions_64, interleaved;
    int64_t rows;
    int heads, dim, half;
    HeadRows x, y;
    const void *positions;
    const double *frequencies;
    float magnitude, sine;   // sine: magnitude, or its negative for the gradient
    int each;                // rows of a workgroup
    int64_t first;
};

struct Dropout {
    int dtype;
    int64_t rows, width, calls;      // calls: of the generator for a row
    const void *x, *residual;
    void *y;
    int64_t ldx, ldr, ldy;
    const uint32_t *seed;
    uint32_t drop;                   // of 2^16
    float scale;
    int64_t first;
};

// 16-byte vectors of a layer norm's row, and the lanes of the team that holds it
inline int norm_vectors(int width, int element) { return (int)(((int64_t)width * element + 15) / 16); }
inline int norm_lanes(int vecs) {
    return vecs <= 16 ? 8 : vecs <= 32 ? 16 : vecs <= 64 ? 32 : vecs <= 256 ? 64 : vecs <= 1024 ? 256 : 1024;
}
// blocks of the layer norm's backward pass (one row of partial sums each)
int norm_backward_blocks(int dtype, int64_t rows, int width);
// parts each group's rows are cut into by the weights' gradient
int grouped_matmul_splits(int64_t rows, int groups, int n, int k);

// shares that each tile's keys are cut into by the forward pass for few queries; 0: the one for many
int attention_splits(int64_t rows, int64_t key_rows, int sequences, int heads, int kv_heads);

constexpr int kMaxShares = 256;    // of a tile's keys, in attention
constexpr int kCus = 256;          // compute units of an MI355X
constexpr int kBig = 256;          // rows and columns of a tile of the grouped products
constexpr int kGradVecs = 1024;   // 16-byte vectors of a row that one workgroup of the loss gradient takes

// Launches: 0 or a hipError_t.
int launch_norm_forward(const NormForward &a, void *stream);
int launch_norm_backward(const NormBackward &a, void *stream);
int launch_softmax_loss(const SoftmaxLoss &a, void *stream);            // loss and lse; dlogits unless null
int launch_softmax_loss_backward(const SoftmaxLoss &a, void *stream);   // dlogits from lse and low
int launch_product_forward(const GroupedProduct &a, void *stream);
int launch_product_rows_grad(const GroupedProduct &a, void *stream);
int launch_product_weights_grad(const GroupedProduct &a, void *stream);
int launch_attention_forward(const Attention &a, void *stream);
int launch_attention_backward(const Attention &a, void *stream);
int launch_rotary(const Rotary &a, void *stream);
int launch_dropout(const Dropout &a, void *stream);
const char *launch_error(int e);

}  // namespace pase
