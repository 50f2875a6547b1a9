// Rotary positions (pase_operators.h).
//
// Pair i of a head turns by the angle position * frequencies[i], the gradient by its
// negative.  A workgroup forms the sines and cosines of its rows once, in LDS, for all
// their heads.  Angles of far positions need 64 bits: turns t = position * frequency / (2
// pi) in fp64, of which only the fraction counts, taken to the nearest quarter q with a rest in
// [-1/8, 1/8] turns that 32 bits hold to 2^-28; sine and cosine of the rest then change
// places and signs by q.
// Bound by HBM: x read once, y written once.  16384 rows of 32 heads of 64 in bf16 28 us for 134 MB (4.8 TB/s).
#include <hip/hip_runtime.h>

#include "operators.h"
#include "vectors.h"

namespace pase {
namespace {

constexpr int kAngles = 512;   // of a workgroup, at most

// (cosine, sine) of 2 pi t
__device__ __forceinline__ float2 turn(double t) {
    t -= __builtin_rint(t);
    const double q = __builtin_rint(4 * t);
    const float rest = (float)(4 * t - q) * 0.5f;   // half turns
    const float s = sinpif(rest), c = cospif(rest);
    const int quarter = (int)q & 3;
    const float x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;
    return {quarter == 1 || quarter == 2 ? -x : x, quarter >= 2 ? -y : y};
}

template <typename T> __global__ __launch_bounds__(256) void k_rotary(Rotary a) {
    constexpr int V = kVec<T>;
    __shared__ float2 angle[kAngles];
    const int64_t row0 = (a.first + blockIdx.x) * a.each;
    const int rows = a.rows - row0 < a.each ? (int)(a.rows - row0) : a.each;
    for (int i = threadIdx.x; i < rows * a.half; i += 256) {
        const int r = i / a.half;
        const int64_t position = a.positions_64 ? static_cast<const int64_t *>(a.positions)[row0 + r]
                                                : (int64_t) static_cast<const int32_t *>(a.positions)[row0 + r];
        const float2 v = turn((double)position * a.frequencies[i - r * a.half] * 0.15915494309189533577);   // 1 / (2 pi)
        angle[i] = {v.x * a.magnitude, v.y * a.sine};
    }
    __syncthreads();
    // vectors of a head: of pairs (both ends of V pairs, or V / 2 neighbouring ones), then of the rest
    const int paired = a.interleaved ? (2 * a.half + V - 1) / V : (a.half + V - 1) / V, rest = a.dim - 2 * a.half;
    const int per = paired + (a.x.p == a.y.p ? 0 : (rest + V - 1) / V), row_vectors = a.heads * per;
    for (int i = threadIdx.x; i < rows * row_vectors; i += 256) {
        const int r = i / row_vectors, in = i - r * row_vectors, head = in / per, u = in - head * per;
        const T *x = static_cast<const T *>(a.x.p) + (row0 + r) * a.x.ld + head * a.x.head_ld;
        T *y = static_cast<T *>(a.y.p) + (row0 + r) * a.y.ld + head * a.y.head_ld;
        const float2 *w = angle + r * a.half;
        if (u >= paired) {
            const int at = 2 * a.half + (u - paired) * V;
            store_pack(y + at, a.dim - at, load_pack(x + at, a.dim - at, (T)0.0f));
        } else if (a.interleaved) {
            const int at = u * V, n = 2 * a.half - at;
            Pack<T> p = load_pack(x + at, n, (T)0.0f);
#pragma unroll
            for (int j = 0; j < V; j += 2) {
                const float2 t = w[j < n ? (at + j) / 2 : 0];
                const float b = (float)p.e[j], c = (float)p.e[j + 1];
                p.e[j] = (T)(b * t.x - c * t.y), p.e[j + 1] = (T)(b * t.y + c * t.x);
            }
            store_pack(y + at, n, p);
        } else {
            const int at = u * V, n = a.half - at;
            Pack<T> p = load_pack(x + at, n, (T)0.0f), q = load_pack(x + a.half + at, n, (T)0.0f);
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float2 t = w[j < n ? at + j : 0];
                const float b = (float)p.e[j], c = (float)q.e[j];
                p.e[j] = (T)(b * t.x - c * t.y), q.e[j] = (T)(b * t.y + c * t.x);
            }
            store_pack(y + at, n, p);
            store_pack(y + a.half + at, n, q);
        }
    }
}

template <typename T> int go(Rotary a, void *stream) {
    // as many rows as a thread each has an angle of, while two workgroups a CU are left
    int64_t each = 256 / a.half;
    if (each > a.rows / (2 * kCus)) each = a.rows / (2 * kCus);
    a.each = (int)(each < 1 ? 1 : each);
    const int64_t blocks = (a.rows + a.each - 1) / a.each, most = most_blocks(256);
    for (int64_t at = 0; at < blocks; at += most) {
        a.first = at;
        if (const int e = launch(k_rotary<T>, blocks - at < most ? blocks - at : most, 256, stream, a)) return e;
    }
    return 0;
}

}  // namespace

int launch_rotary(const Rotary &a, void *stream) {
    return a.dtype == PASE_BF16 ? go<__bf16>(a, stream) : a.dtype == PASE_FP16 ? go<_Float16>(a, stream) : go<float>(a, stream);
}

}  // namespace pase
