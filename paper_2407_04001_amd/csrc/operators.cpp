// C entry points of the layer operators: argument checks and workspace sizes.
// Nothing here touches the device; the launches are in the .hip files.
#include "operators.h"

#include <cstdarg>
#include <cstdio>

namespace pase {
namespace {

thread_local char g_error[256] = "";

__attribute__((format(printf, 2, 3))) pase_status refuse(pase_status st, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(g_error, sizeof g_error, fmt, ap);
    va_end(ap);
    return st;
}

pase_status launched(int e) {
    if (e == 0) return PASE_OK;
    return refuse(PASE_ERR_HIP, "launch failed: %s", launch_error(e));
}

constexpr uint64_t kMaxRows = 1ull << 40, kMaxLd = 1ull << 32;
constexpr uint64_t kMaxProductDim = 1u << 20;     // n and k of a grouped product
constexpr uint64_t kMaxProductLd = 1u << 22;      // 256 rows of a tile stay within 2^31 bytes
constexpr uint64_t kMaxClasses = (1ull << 31) - 1024;

int element_bytes(int dtype) { return dtype == PASE_FP32 ? 4 : 2; }

bool known(int dtype) { return dtype == PASE_BF16 || dtype == PASE_FP16 || dtype == PASE_FP32; }

bool aligned(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

#define REQUIRE(cond, ...) \
    do { \
        if (!(cond)) return refuse(PASE_ERR_INVALID_ARGUMENT, __VA_ARGS__); \
    } while (0)

// One matrix argument: there, aligned to its element, with rows that do not overlap.
#define REQUIRE_MATRIX(p, ld, cols, dtype) \
    do { \
        REQUIRE((p) != nullptr, #p " is null"); \
        REQUIRE(aligned(p, element_bytes(dtype)), #p " is not aligned to its element"); \
        REQUIRE((ld) >= (cols), "row stride of " #p " below its row length"); \
        REQUIRE((ld) <= kMaxLd, "row stride of " #p " too large"); \
    } while (0)

pase_status check_norm(int dtype, int param_dtype, uint64_t rows, uint64_t width) {
    REQUIRE(known(dtype), "unknown dtype %d", dtype);
    REQUIRE(param_dtype == dtype || param_dtype == PASE_FP32, "param_dtype is neither dtype nor fp32");
    REQUIRE(width >= 1, "width 0");
    if (width > PASE_NORM_MAX_WIDTH)
        return refuse(PASE_ERR_TOO_LARGE, "width %llu above %d", (unsigned long long)width, PASE_NORM_MAX_WIDTH);
    if (rows > kMaxRows) return refuse(PASE_ERR_TOO_LARGE, "too many rows");
    return PASE_OK;
}

pase_status check_product(int dtype, int out_dtype, uint64_t rows, uint32_t groups, uint64_t n, uint64_t k,
                          const char *out_name) {
    REQUIRE(dtype == PASE_BF16 || dtype == PASE_FP16, "grouped products take bf16 or fp16, not dtype %d", dtype);
    REQUIRE(out_dtype == dtype || out_dtype == PASE_FP32, "%s is neither dtype nor fp32", out_name);
    REQUIRE(groups >= 1, "no groups");
    REQUIRE(n >= 1 && k >= 1, "n or k is 0");
    if (groups > PASE_MAX_GROUPS)
        return refuse(PASE_ERR_TOO_LARGE, "%u groups, above %d", groups, PASE_MAX_GROUPS);
    if (n > kMaxProductDim || k > kMaxProductDim) return refuse(PASE_ERR_TOO_LARGE, "n or k above 2^20");
    if (rows > (1ull << 31) - (1u << 20)) return refuse(PASE_ERR_TOO_LARGE, "too many rows");
    // tiles of the output, at the smallest tile: they are one dimension of a grid
    const uint64_t row_tiles = rows / 16 + groups + 2, w_tiles = ((n + 127) / 128) * ((k + 127) / 128);
    const uint64_t col = (n > k ? n : k) / 16 + 1;
    if (row_tiles > ((1ull << 31) - 1) / col || (uint64_t)groups > ((1ull << 31) - 1) / (w_tiles * 64))
        return refuse(PASE_ERR_TOO_LARGE, "the product has 2^31 tiles or more");
    return PASE_OK;
}

pase_status check_offsets(const void *offsets, int offsets_64) {
    REQUIRE(offsets, "offsets is null");
    REQUIRE(offsets_64 == 0 || offsets_64 == 1, "offsets_64 is neither 0 nor 1");
    REQUIRE(aligned(offsets, offsets_64 ? 8 : 4), "offsets is not aligned to its element");
    return PASE_OK;
}

pase_status check_loss(int dtype, uint64_t rows, uint64_t classes, const void *targets, int targets_64) {
    REQUIRE(known(dtype), "unknown dtype %d", dtype);
    REQUIRE(classes >= 1, "no classes");
    if (classes > kMaxClasses) return refuse(PASE_ERR_TOO_LARGE, "too many classes");
    if (rows > (1ull << 31) - 1) return refuse(PASE_ERR_TOO_LARGE, "too many rows");
    if (rows) {
        REQUIRE(targets, "targets is null");
        REQUIRE(targets_64 == 0 || targets_64 == 1, "targets_64 is neither 0 nor 1");
        REQUIRE(aligned(targets, targets_64 ? 8 : 4), "targets is not aligned to its element");
    }
    return PASE_OK;
}

pase_status check_workspace(const void *workspace, uint64_t have, uint64_t need) {
    if (!need) return PASE_OK;
    REQUIRE(workspace, "workspace is null, %llu bytes are needed", (unsigned long long)need);
    REQUIRE(aligned(workspace, 16), "workspace is not aligned to 16 bytes");
    if (have < need)
        return refuse(PASE_ERR_OUT_OF_MEMORY, "workspace of %llu bytes, %llu are needed", (unsigned long long)have,
                      (unsigned long long)need);
    return PASE_OK;
}

uint64_t norm_bytes(int dtype, uint64_t rows, uint64_t width) {
    return (uint64_t)norm_backward_blocks(dtype, (int64_t)rows, (int)width) * 2 * width * sizeof(float);
}

uint64_t product_bytes(uint64_t rows, uint32_t groups, uint64_t n, uint64_t k) {
    const int splits = grouped_matmul_splits((int64_t)rows, (int)groups, (int)n, (int)k);
    return splits > 1 ? (uint64_t)splits * groups * n * k * sizeof(float) : 0;
}

#define CHECK(call) \
    do { \
        const pase_status st_ = (call); \
        if (st_ != PASE_OK) return st_; \
    } while (0)

pase_status softmax_loss(int dtype, uint64_t rows, uint64_t classes, const void *logits, uint64_t ldl,
                         const void *targets, int targets_64, int64_t ignore_index, const float *dloss,
                         uint64_t dloss_stride, float *loss, float *lse, float *low, void *dlogits, uint64_t lddl,
                         bool grad, void *stream) {
    CHECK(check_loss(dtype, rows, classes, targets, targets_64));
    if (!rows) return PASE_OK;
    REQUIRE_MATRIX(logits, ldl, classes, dtype);
    REQUIRE(loss && lse, "loss or lse is null");
    REQUIRE(aligned(loss, 4) && aligned(lse, 4), "loss or lse is not aligned to its element");
    REQUIRE(!low || aligned(low, 4), "lse_low is not aligned to its element");
    if (grad) {
        REQUIRE_MATRIX(dlogits, lddl, classes, dtype);
        REQUIRE(dloss && aligned(dloss, 4), "dloss is null or not aligned to its element");
        REQUIRE(dloss_stride <= 1, "dloss_stride is neither 0 nor 1");
        REQUIRE(dlogits != logits || ldl == lddl, "dlogits is logits with another row stride");
    }
    SoftmaxLoss a{};
    a.dtype = dtype, a.targets_64 = targets_64;
    a.rows = (int64_t)rows, a.classes = (int64_t)classes;
    a.logits = logits, a.ldl = (int64_t)ldl;
    a.targets = targets, a.ignore = ignore_index;
    a.dloss = dloss, a.dloss_stride = (int64_t)dloss_stride;
    a.loss = loss, a.lse = lse, a.low = low;
    a.dlogits = grad ? dlogits : nullptr, a.lddl = (int64_t)lddl;
    return launched(launch_softmax_loss(a, stream));
}

pase_status softmax_loss_backward(int dtype, uint64_t rows, uint64_t classes, const void *logits, uint64_t ldl,
                                  const void *targets, int targets_64, int64_t ignore_index, const float *lse,
                                  const float *low, const float *dloss, uint64_t dloss_stride, void *dlogits,
                                  uint64_t lddl, void *stream) {
    CHECK(check_loss(dtype, rows, classes, targets, targets_64));
    if (!rows) return PASE_OK;
    REQUIRE_MATRIX(logits, ldl, classes, dtype);
    REQUIRE_MATRIX(dlogits, lddl, classes, dtype);
    REQUIRE(lse && aligned(lse, 4), "lse is null or not aligned to its element");
    REQUIRE(!low || aligned(low, 4), "lse_low is not aligned to its element");
    REQUIRE(dloss && aligned(dloss, 4), "dloss is null or not aligned to its element");
    REQUIRE(dloss_stride <= 1, "dloss_stride is neither 0 nor 1");
    REQUIRE(dlogits != logits || ldl == lddl, "dlogits is logits with another row stride");
    const uint64_t span = (uint64_t)kGradVecs * (16 / element_bytes(dtype));
    if (rows > ((1ull << 31) - 1) / ((classes + span - 1) / span))
        return refuse(PASE_ERR_TOO_LARGE, "the logits have too many elements for one call");
    SoftmaxLoss a{};
    a.dtype = dtype, a.targets_64 = targets_64;
    a.rows = (int64_t)rows, a.classes = (int64_t)classes;
    a.logits = logits, a.ldl = (int64_t)ldl;
    a.targets = targets, a.ignore = ignore_index;
    a.dloss = dloss, a.dloss_stride = (int64_t)dloss_stride;
    a.lse = const_cast<float *>(lse), a.low = const_cast<float *>(low);
    a.dlogits = dlogits, a.lddl = (int64_t)lddl;
    return launched(launch_softmax_loss_backward(a, stream));
}

}  // namespace

int norm_backward_blocks(int dtype, int64_t rows, int width) {
    const int lanes = norm_lanes(norm_vectors(width, element_bytes(dtype)));
    const int64_t teams = lanes < 256 ? 256 / lanes : 1, want = (rows + teams - 1) / teams;
    return (int)(want < 512 ? want : 512);
}

// A part a CU, while parts of an average group keep 512 rows: with fewer tiles than
// CUs the rest would be idle, and a part's sums are written and read once more.
int grouped_matmul_splits(int64_t rows, int groups, int n, int k) {
    const int64_t tiles = (int64_t)groups * ((n + kBig - 1) / kBig) * ((k + kBig - 1) / kBig);
    const int64_t idle = kCus / tiles, deep = rows / groups / 512, most = idle < deep ? idle : deep;
    return (int)(most < 1 ? 1 : most > 32 ? 32 : most);
}

}  // namespace pase

using namespace pase;

extern "C" {

const char *pase_operator_error(void) { return g_error; }

pase_status pase_layer_norm_forward(int dtype, int param_dtype, uint64_t rows, uint64_t width, const void *x,
                                    uint64_t ldx, const void *residual, uint64_t ldr, const void *gain,
                                    const void *bias, float eps, void *y, uint64_t ldy, void *z, uint64_t ldz,
                                    float *mean, float *rstd, void *stream) {
    CHECK(check_norm(dtype, param_dtype, rows, width));
    REQUIRE(eps >= 0, "eps is negative or NaN");
    if (!rows) return PASE_OK;
    REQUIRE_MATRIX(x, ldx, width, dtype);
    REQUIRE_MATRIX(y, ldy, width, dtype);
    if (residual) {
        REQUIRE_MATRIX(residual, ldr, width, dtype);
        REQUIRE(z, "z is null with a residual");
    }
    if (z) REQUIRE_MATRIX(z, ldz, width, dtype);
    REQUIRE(gain && aligned(gain, element_bytes(param_dtype)), "gain is null or not aligned to its element");
    REQUIRE(!bias || aligned(bias, element_bytes(param_dtype)), "bias is not aligned to its element");
    REQUIRE(mean && rstd && aligned(mean, 4) && aligned(rstd, 4), "mean or rstd is null or not aligned");
    NormForward a{};
    a.dtype = dtype, a.param_dtype = param_dtype;
    a.rows = (int64_t)rows, a.width = (int)width;
    a.x = x, a.ldx = (int64_t)ldx;
    a.residual = residual, a.ldr = (int64_t)ldr;
    a.gain = gain, a.bias = bias, a.eps = eps;
    a.y = y, a.ldy = (int64_t)ldy;
    a.z = z, a.ldz = (int64_t)ldz;
    a.mean = mean, a.rstd = rstd;
    return launched(launch_norm_forward(a, stream));
}

pase_status pase_layer_norm_workspace(int dtype, uint64_t rows, uint64_t width, uint64_t *bytes) {
    REQUIRE(bytes, "bytes is null");
    CHECK(check_norm(dtype, dtype, rows, width));
    *bytes = norm_bytes(dtype, rows, width);
    return PASE_OK;
}

pase_status pase_layer_norm_backward(int dtype, int param_dtype, uint64_t rows, uint64_t width, const void *dy,
                                     uint64_t lddy, const void *z, uint64_t ldz, const void *dz, uint64_t lddz,
                                     const void *gain, const float *mean, const float *rstd, void *dx,
                                     uint64_t lddx, void *dgain, void *dbias, void *workspace,
                                     uint64_t workspace_bytes, void *stream) {
    CHECK(check_norm(dtype, param_dtype, rows, width));
    REQUIRE(!dgain || aligned(dgain, element_bytes(param_dtype)), "dgain is not aligned to its element");
    REQUIRE(!dbias || aligned(dbias, element_bytes(param_dtype)), "dbias is not aligned to its element");
    if (rows) {
        REQUIRE_MATRIX(dy, lddy, width, dtype);
        REQUIRE_MATRIX(z, ldz, width, dtype);
        if (dz) REQUIRE_MATRIX(dz, lddz, width, dtype);
        REQUIRE_MATRIX(dx, lddx, width, dtype);
        REQUIRE(dx != dy || lddx == lddy, "dx is dy with another row stride");
        REQUIRE(!dz || dx != dz || lddx == lddz, "dx is dz with another row stride");
        REQUIRE(gain && aligned(gain, element_bytes(param_dtype)), "gain is null or not aligned to its element");
        REQUIRE(mean && rstd && aligned(mean, 4) && aligned(rstd, 4), "mean or rstd is null or not aligned");
        CHECK(check_workspace(workspace, workspace_bytes, norm_bytes(dtype, rows, width)));
    }
    NormBackward a{};
    a.dtype = dtype, a.param_dtype = param_dtype;
    a.rows = (int64_t)rows, a.width = (int)width;
    a.dy = dy, a.lddy = (int64_t)lddy;
    a.z = z, a.ldz = (int64_t)ldz;
    a.dz = dz, a.lddz = (int64_t)lddz;
    a.gain = gain, a.mean = mean, a.rstd = rstd;
    a.dx = dx, a.lddx = (int64_t)lddx;
    a.dgain = dgain, a.dbias = dbias;
    a.partial = static_cast<float *>(workspace);
    a.blocks = norm_backward_blocks(dtype, a.rows, a.width);
    return launched(launch_norm_backward(a, stream));
}

pase_status pase_grouped_matmul_forward(int dtype, int out_dtype, uint64_t rows, uint32_t groups, uint64_t n,
                                        uint64_t k, const void *x, uint64_t ldx, const void *w,
                                        const void *offsets, int offsets_64, void *y, uint64_t ldy, void *stream) {
    CHECK(check_product(dtype, out_dtype, rows, groups, n, k, "out_dtype"));
    if (!rows) return PASE_OK;
    REQUIRE_MATRIX(x, ldx, k, dtype);
    REQUIRE_MATRIX(w, k, k, dtype);
    REQUIRE_MATRIX(y, ldy, n, out_dtype);
    REQUIRE(ldx <= kMaxProductLd && ldy <= kMaxProductLd, "row stride above 2^22");
    CHECK(check_offsets(offsets, offsets_64));
    GroupedProduct a{};
    a.dtype = dtype, a.out_dtype = out_dtype, a.offsets_64 = offsets_64;
    a.rows = (int64_t)rows, a.groups = (int)groups, a.n = (int)n, a.k = (int)k;
    a.x = x, a.ldx = (int64_t)ldx;
    a.w = w, a.offsets = offsets;
    a.out = y, a.ldo = (int64_t)ldy;
    return launched(launch_product_forward(a, stream));
}

pase_status pase_grouped_matmul_workspace(int dtype, int grad_dtype, uint64_t rows, uint32_t groups, uint64_t n,
                                          uint64_t k, uint64_t *bytes) {
    REQUIRE(bytes, "bytes is null");
    CHECK(check_product(dtype, grad_dtype, rows, groups, n, k, "grad_dtype"));
    *bytes = product_bytes(rows, groups, n, k);
    return PASE_OK;
}

pase_status pase_grouped_matmul_backward(int dtype, int grad_dtype, uint64_t rows, uint32_t groups, uint64_t n,
                                         uint64_t k, const void *dy, uint64_t lddy, const void *x, uint64_t ldx,
                                         const void *w, const void *offsets, int offsets_64, void *dx,
                                         uint64_t lddx, void *dw, void *workspace, uint64_t workspace_bytes,
                                         void *stream) {
    CHECK(check_product(dtype, grad_dtype, rows, groups, n, k, "grad_dtype"));
    if (rows) {
        REQUIRE_MATRIX(dy, lddy, n, dtype);
        REQUIRE(lddy <= kMaxProductLd, "row stride above 2^22");
        if (dx) {
            REQUIRE_MATRIX(dx, lddx, k, dtype);
            REQUIRE_MATRIX(w, k, k, dtype);
            REQUIRE(lddx <= kMaxProductLd, "row stride above 2^22");
        }
        if (dw) {
            REQUIRE_MATRIX(x, ldx, k, dtype);
            REQUIRE(ldx <= kMaxProductLd, "row stride above 2^22");
        }
    }
    if (dw) {
        REQUIRE_MATRIX(dw, k, k, grad_dtype);
        CHECK(check_workspace(workspace, workspace_bytes, product_bytes(rows, groups, n, k)));
    }
    CHECK(check_offsets(offsets, offsets_64));
    GroupedProduct a{};
    a.dtype = dtype, a.out_dtype = dtype, a.offsets_64 = offsets_64;
    a.rows = (int64_t)rows, a.groups = (int)groups, a.n = (int)n, a.k = (int)k;
    a.x = x, a.ldx = (int64_t)ldx;
    a.dy = dy, a.lddy = (int64_t)lddy;
    a.w = w, a.offsets = offsets;
    if (dx && rows) {
        a.out = dx, a.ldo = (int64_t)lddx;
        CHECK(launched(launch_product_rows_grad(a, stream)));
    }
    if (dw) {
        a.out_dtype = grad_dtype;
        a.out = dw, a.ldo = (int64_t)k;
        a.splits = grouped_matmul_splits(a.rows, a.groups, a.n, a.k);
        a.partial = a.splits > 1 ? static_cast<float *>(workspace) : nullptr;
        CHECK(launched(launch_product_weights_grad(a, stream)));
    }
    return PASE_OK;
}

pase_status pase_softmax_loss_forward(int dtype, uint64_t rows, uint64_t classes, const void *logits, uint64_t ldl,
                                      const void *targets, int targets_64, int64_t ignore_index, float *loss,
                                      float *lse, void *stream) {
    return softmax_loss(dtype, rows, classes, logits, ldl, targets, targets_64, ignore_index, nullptr, 0, loss, lse,
                        nullptr, nullptr, 0, false, stream);
}

pase_status pase_softmax_loss_forward_parts(int dtype, uint64_t rows, uint64_t classes, const void *logits,
                                            uint64_t ldl, const void *targets, int targets_64, int64_t ignore_index,
                                            float *loss, float *lse, float *lse_low, void *stream) {
    if (rows) REQUIRE(lse_low, "lse_low is null");
    return softmax_loss(dtype, rows, classes, logits, ldl, targets, targets_64, ignore_index, nullptr, 0, loss, lse,
                        lse_low, nullptr, 0, false, stream);
}

pase_status pase_softmax_loss_grad(int dtype, uint64_t rows, uint64_t classes, const void *logits, uint64_t ldl,
                                   const void *targets, int targets_64, int64_t ignore_index, const float *dloss,
                                   uint64_t dloss_stride, float *loss, float *lse, void *dlogits, uint64_t lddl,
                                   void *stream) {
    return softmax_loss(dtype, rows, classes, logits, ldl, targets, targets_64, ignore_index, dloss, dloss_stride,
                        loss, lse, nullptr, dlogits, lddl, true, stream);
}

pase_status pase_softmax_loss_backward(int dtype, uint64_t rows, uint64_t classes, const void *logits, uint64_t ldl,
                                       const void *targets, int targets_64, int64_t ignore_index, const float *lse,
                                       const float *dloss, uint64_t dloss_stride, void *dlogits, uint64_t lddl,
                                       void *stream) {
    return softmax_loss_backward(dtype, rows, classes, logits, ldl, targets, targets_64, ignore_index, lse, nullptr,
                                 dloss, dloss_stride, dlogits, lddl, stream);
}

pase_status pase_softmax_loss_backward_parts(int dtype, uint64_t rows, uint64_t classes, const void *logits,
                                             uint64_t ldl, const void *targets, int targets_64, int64_t ignore_index,
                                             const float *lse, const float *lse_low, const float *dloss,
                                             uint64_t dloss_stride, void *dlogits, uint64_t lddl, void *stream) {
    if (rows) REQUIRE(lse_low, "lse_low is null");
    return softmax_loss_backward(dtype, rows, classes, logits, ldl, targets, targets_64, ignore_index, lse, lse_low,
                                 dloss, dloss_stride, dlogits, lddl, stream);
}

}  // extern "C"
