// Softmax loss of rows of logits, its gradient, and both in one pass
// (pase_operators.h).
//
// With m the row's maximum, lse = m + ln sum exp(l - m): no exponent is
// positive, so nothing overflows.  The loss is (m - l[target]) + ln sum and the
// gradient's exponents are (l - m) - ln sum: lse itself, rounded to fp32, would put
// half a unit of m's last place into each, more than a small loss where all logits
// of a row are large.  A row that fits is held in one workgroup's
// registers as it was read, so that the maximum, the sum and the gradient take
// one pass over HBM; a longer one is read again, its maximum and sum formed
// together on the first pass (a sum of terms exp(l - m) grows by the factor
// exp(m - m') when the maximum moves to m').
// Bound by HBM: the logits read once, the gradient written once.
#include "operators.h"
#include "vectors.h"

namespace pase {
namespace {

template <typename T> __device__ __forceinline__ T masked() {
    return (T)(-__builtin_inff());
}

__device__ __forceinline__ int64_t target_of(const SoftmaxLoss &a, int64_t row) {
    return a.targets_64 ? static_cast<const int64_t *>(a.targets)[row]
                        : (int64_t) static_cast<const int32_t *>(a.targets)[row];
}

// A row's log-sum-exp as two numbers whose sum it is: its maximum and the log of its
// sum, or lse and what the rounding of lse left.  Both -inf (or -inf and 0): every class is
// masked, as the sum is 0 then alone (otherwise the maximum's own term is 1 or NaN).
struct Lse {
    float high, low;
    __device__ __forceinline__ bool empty() const { return high + low == -__builtin_inff(); }
};

template <typename T>
__device__ __forceinline__ float row_loss(const T *logits, int64_t classes, int64_t target, Lse lse) {
    if (target < 0 || target >= classes) return __builtin_nanf("");
    return lse.empty() ? __builtin_inff() : (lse.high - (float)logits[target]) + lse.low;
}

// lse, its remainder where asked for (exact: high + low = lse + remainder), and the loss of a row.
template <typename T>
__device__ __forceinline__ void put_row(const SoftmaxLoss &a, int64_t row, const T *logits, int64_t target, Lse lse) {
    const float sum = lse.high + lse.low, of_low = sum - lse.high;
    a.lse[row] = sum;
    if (a.low) a.low[row] = lse.empty() ? 0.0f : (lse.high - (sum - of_low)) + (lse.low - of_low);
    a.loss[row] = row_loss(logits, a.classes, target, lse);
}

// What a row's gradient needs: (exp(l - lse) - [target]) * scale, where scale is 0 for
// a row with every class masked and NaN for a target out of range.
struct RowGrad {
    Lse lse;
    float scale;
};

__device__ __forceinline__ RowGrad row_grad(const SoftmaxLoss &a, int64_t row, int64_t target, Lse lse) {
    const float g = a.dloss[row * a.dloss_stride];
    const bool known = target >= 0 && target < a.classes, empty = lse.empty();
    // every class masked: any finite lse makes exp(-inf - lse) = 0, and the scale takes the target's -1 away
    return {{empty ? 0.0f : lse.high, empty ? 0.0f : lse.low}, !known ? __builtin_nanf("") : empty ? 0.0f : g};
}

template <typename T> __device__ __forceinline__ T grad_of(T logit, bool target, const RowGrad &g) {
    const float p = __expf(((float)logit - g.lse.high) - g.lse.low);
    return (T)((target ? p - 1.0f : p) * g.scale);
}

// Gradient of one vector.  KEEP: the target's own place keeps its logit.
template <typename T, bool KEEP = false>
__device__ __forceinline__ void grad_pack(T *out, int64_t at, int64_t n, const Pack<T> &l, int64_t target, const RowGrad &g) {
    if (n <= 0) return;
    Pack<T> o;
    const int64_t hit = target - at;
#pragma unroll
    for (int j = 0; j < kVec<T>; j++) o.e[j] = KEEP && j == hit ? l.e[j] : grad_of(l.e[j], j == hit, g);
    store_pack(out + at, n, o);
}

template <typename T> __device__ __forceinline__ void zero_row(T *out, int64_t classes, int threads) {
    Pack<T> zero;
    zero.v = 0;
    for (int64_t at = (int64_t)threadIdx.x * kVec<T>; at < classes; at += (int64_t)threads * kVec<T>)
        store_pack(out + at, classes - at, zero);
}

// One row a workgroup of WAVES waves, NV vectors a lane.  Bound by HBM: 16384 x 32768 in
// bf16, loss and gradient, 380-400 us for 2.15 GB (5.4-5.7 TB/s).  Sixteen waves with sixteen
// vectors a lane (rows of 131072 in bf16) would leave one workgroup on a CU, which loads,
// sums and stores by turns: 1608 us against 501 for k_loss_long.
template <typename T, int NV, int WAVES, bool GRAD>
__global__ __launch_bounds__(WAVES * 64) void k_loss_row(SoftmaxLoss a) {
    constexpr int V = kVec<T>, THREADS = WAVES * 64;
    __shared__ float lds[2 * WAVES];
    const int64_t row = blockIdx.x;
    const T *logits = static_cast<const T *>(a.logits) + row * a.ldl;
    T *out = static_cast<T *>(a.dlogits) + row * a.lddl;
    const int64_t target = target_of(a, row);
    if (target == a.ignore) {
        if (threadIdx.x == 0) {
            a.loss[row] = 0, a.lse[row] = 0;
            if (a.low) a.low[row] = 0;
        }
        if (GRAD) zero_row(out, a.classes, THREADS);
        return;
    }
    Pack<T> l[NV];
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int64_t at = (int64_t)(threadIdx.x + i * THREADS) * V;
        l[i] = load_pack(logits + at, a.classes - at, masked<T>());
    }
    float top = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
        for (int j = 0; j < V; j++) top = fmaxf(top, (float)l[i].e[j]);
    top = group_max<WAVES>(top, lds);
    const float from = top == -__builtin_inff() ? 0.0f : top;
    float s[1] = {0};
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
        for (int j = 0; j < V; j++) s[0] += __expf((float)l[i].e[j] - from);
    group_sum<WAVES>(s, lds + WAVES);
    const Lse lse = {top, logf(s[0])};
    if (threadIdx.x == 0) put_row(a, row, logits, target, lse);
    if (GRAD) {
        // in place, the target's logit is read above before its own lane writes it
        __syncthreads();
        const RowGrad g = row_grad(a, row, target, lse);
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int64_t at = (int64_t)(threadIdx.x + i * THREADS) * V;
            grad_pack(out, at, a.classes - at, l[i], target, g);
        }
    }
}

// A longer row: read by kAhead vectors a lane in flight, and for the gradient again,
// one by one (that pass also writes; with 8 in flight 1280 x 65536 in fp32 took 210 us
// against 161).  4096 x 131072 in bf16: loss 188 us (1.07 GB, 5.7 TB/s), loss and
// gradient 501 us; 1 x 131072 loss 9 us.
// Or, where workgroups that share the row make its gradient (SPLIT): leaves the maximum in
// lse and the log of the sum in loss for them.
constexpr int kAhead = 8;

template <typename T, bool GRAD, bool SPLIT = false> __global__ __launch_bounds__(1024) void k_loss_long(SoftmaxLoss a) {
    constexpr int V = kVec<T>, WAVES = 16, THREADS = 1024;
    __shared__ float lds[2 * WAVES];
    const int64_t row = blockIdx.x;
    const T *logits = static_cast<const T *>(a.logits) + row * a.ldl;
    T *out = static_cast<T *>(a.dlogits) + row * a.lddl;
    const int64_t target = target_of(a, row);
    if (target == a.ignore) {
        if (threadIdx.x == 0) {
            a.loss[row] = 0, a.lse[row] = 0;
            if (a.low) a.low[row] = 0;
        }
        if (GRAD) zero_row(out, a.classes, THREADS);
        return;
    }
    const int64_t first = (int64_t)threadIdx.x * V, stride = (int64_t)THREADS * V;
    float top = -__builtin_inff(), from = 0.0f, sum = 0.0f;
    for (int64_t at = first; at < a.classes; at += kAhead * stride) {
        Pack<T> l[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; i++)
            l[i] = load_pack(logits + at + i * stride, a.classes - at - i * stride, masked<T>());
        float t = top;
#pragma unroll
        for (int i = 0; i < kAhead; i++)
#pragma unroll
            for (int j = 0; j < V; j++) t = fmaxf(t, (float)l[i].e[j]);
        if (t > top) {
            sum *= __expf(top - t);   // top is -inf only while the sum is 0 or NaN
            top = from = t;
        }
#pragma unroll
        for (int i = 0; i < kAhead; i++)
#pragma unroll
            for (int j = 0; j < V; j++) sum += __expf((float)l[i].e[j] - from);
    }
    const float all = group_max<WAVES>(top, lds);
    float s[1] = {top == -__builtin_inff() ? sum : sum * __expf(top - all)};
    group_sum<WAVES>(s, lds + WAVES);
    const Lse lse = {all, logf(s[0])};
    if (threadIdx.x == 0) {
        if (SPLIT)
            a.lse[row] = lse.high, a.loss[row] = lse.low;
        else
            put_row(a, row, logits, target, lse);
    }
    if (GRAD) {
        __syncthreads();
        const RowGrad g = row_grad(a, row, target, lse);
        for (int64_t at = first; at < a.classes; at += stride)
            grad_pack(out, at, a.classes - at, load_pack(logits + at, a.classes - at, masked<T>()), target, g);
    }
}

// Gradient from the lse, from it and its remainder, or from what k_loss_long left of a row
// (kSplit; the target's place keeps its logit for k_loss_ends): 256 threads take 4 vectors
// each of one row.
enum From { kLse, kParts, kSplit };

template <typename T, From F> __global__ __launch_bounds__(256) void k_loss_grad(SoftmaxLoss a, int chunks) {
    constexpr int V = kVec<T>;
    const int64_t row = blockIdx.x / chunks, at0 = (int64_t)(blockIdx.x % chunks) * kGradVecs * V + threadIdx.x * V;
    const T *logits = static_cast<const T *>(a.logits) + row * a.ldl;
    T *out = static_cast<T *>(a.dlogits) + row * a.lddl;
    if (at0 >= a.classes) return;   // before the row's values are waited for: most waves, where rows are short
    const int64_t target = target_of(a, row);
    const bool ignored = target == a.ignore;
    const RowGrad g = row_grad(a, row, target, {a.lse[row], F == kSplit ? a.loss[row] : F == kParts ? a.low[row] : 0.0f});
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int64_t at = at0 + (int64_t)i * 256 * V, n = a.classes - at;
        if (n <= 0) return;
        if (ignored) {
            Pack<T> zero;
            zero.v = 0;
            store_pack(out + at, n, zero);
        } else {
            grad_pack<T, F == kSplit>(out, at, n, load_pack(logits + at, n, masked<T>()), target, g);
        }
    }
}

// The end of a gradient that workgroups shared: the rows' loss and lse, and the gradient
// of their targets, whose logits the others could not read once it is written.
template <typename T> __global__ __launch_bounds__(256) void k_loss_ends(SoftmaxLoss a) {
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row >= a.rows) return;
    const int64_t target = target_of(a, row);
    if (target == a.ignore) return;
    T *out = static_cast<T *>(a.dlogits) + row * a.lddl;
    const Lse lse = {a.lse[row], a.loss[row]};
    put_row(a, row, out, target, lse);
    if (target >= 0 && target < a.classes) out[target] = grad_of(out[target], true, row_grad(a, row, target, lse));
}

// Launches a kernel of `blocks` workgroups a row, on as many rows at a time as one launch holds.
template <typename T, typename K, typename... Args>
int on_rows(K *kernel, int64_t blocks, int threads, void *stream, const SoftmaxLoss &a, Args... args) {
    const int64_t most = most_blocks(threads) / blocks;
    for (int64_t row = 0; row < a.rows; row += most) {
        SoftmaxLoss part = a;
        part.rows = a.rows - row < most ? a.rows - row : most;
        part.logits = static_cast<const T *>(a.logits) + row * a.ldl;
        part.targets = static_cast<const char *>(a.targets) + row * (a.targets_64 ? 8 : 4);
        if (a.dloss) part.dloss = a.dloss + row * a.dloss_stride;
        if (a.loss) part.loss = a.loss + row;
        part.lse = a.lse + row;
        if (a.low) part.low = a.low + row;
        if (a.dlogits) part.dlogits = static_cast<T *>(a.dlogits) + row * a.lddl;
        if (const int e = launch(kernel, part.rows * blocks, threads, stream, part, args...)) return e;
    }
    return 0;
}

template <typename T, From F> int grad_from(const SoftmaxLoss &a, void *stream) {
    const int chunks = (int)((a.classes + kGradVecs * kVec<T> - 1) / (kGradVecs * kVec<T>));
    return on_rows<T>(k_loss_grad<T, F>, chunks, 256, stream, a, chunks);
}

template <typename T, bool GRAD> int loss_rows(const SoftmaxLoss &a, void *stream) {
    const int64_t vecs = (a.classes + kVec<T> - 1) / kVec<T>;
    if (vecs <= 256) return on_rows<T>(k_loss_row<T, 4, 1, GRAD>, 1, 64, stream, a);
    if (vecs <= 1024) return on_rows<T>(k_loss_row<T, 4, 4, GRAD>, 1, 256, stream, a);
    if (vecs <= 4096) return on_rows<T>(k_loss_row<T, 8, 8, GRAD>, 1, 512, stream, a);
    if constexpr (GRAD) {
        // fewer rows than fill the chip: the gradient by workgroups that share rows
        // (1 x 131072 in fp32: 28 us in one kernel, 14 in three)
        if (a.rows < 2 * kCus) {
            if (const int e = launch(k_loss_long<T, false, true>, a.rows, 1024, stream, a)) return e;
            if (const int e = grad_from<T, kSplit>(a, stream)) return e;
            return launch(k_loss_ends<T>, (a.rows + 255) / 256, 256, stream, a);
        }
    }
    return on_rows<T>(k_loss_long<T, GRAD>, 1, 1024, stream, a);
}

template <typename T> int grad_typed(const SoftmaxLoss &a, void *stream) {
    return a.low ? grad_from<T, kParts>(a, stream) : grad_from<T, kLse>(a, stream);
}

template <typename T> int loss_typed(const SoftmaxLoss &a, void *stream) {
    return a.dlogits ? loss_rows<T, true>(a, stream) : loss_rows<T, false>(a, stream);
}

}  // namespace

int launch_softmax_loss(const SoftmaxLoss &a, void *stream) {
    if (a.dtype == PASE_BF16) return loss_typed<__bf16>(a, stream);
    if (a.dtype == PASE_FP16) return loss_typed<_Float16>(a, stream);
    return loss_typed<float>(a, stream);
}

int launch_softmax_loss_backward(const SoftmaxLoss &a, void *stream) {
    if (a.dtype == PASE_BF16) return grad_typed<__bf16>(a, stream);
    if (a.dtype == PASE_FP16) return grad_typed<_Float16>(a, stream);
    return grad_typed<float>(a, stream);
}

}  // namespace pase
