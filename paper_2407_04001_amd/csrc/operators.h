// Arguments of the layer operators, between the checks of operators.cpp (host)
// and the launches in layer_norm.hip, softmax_loss.hip and grouped_matmul.hip.
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

// 16-byte vectors of a layer norm's row, and the lanes of the team that holds it
inline int norm_vectors(int width, int element) { return (int)(((int64_t)width * element + 15) / 16); }
inline int norm_lanes(int vecs) {
    return vecs <= 16 ? 8 : vecs <= 32 ? 16 : vecs <= 64 ? 32 : vecs <= 256 ? 64 : vecs <= 1024 ? 256 : 1024;
}
// blocks of the layer norm's backward pass (one row of partial sums each)
int norm_backward_blocks(int dtype, int64_t rows, int width);
// parts each group's rows are cut into by the weights' gradient
int grouped_matmul_splits(int64_t rows, int groups, int n, int k);

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
const char *launch_error(int e);

}  // namespace pase
