// Dropout with the residual's addition (pase_operators.h).
//
// Whether an element stays follows from its place and the seed alone, by Philox 4x32-10
// (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, 2011): one
// call gives eight elements 16 bits each, so that no mask is stored and the backward pass
// is the same call on the gradient.  16 bits an element halve the generator's work against
// 32; what they leave of a probability is in the scale.
// Bound by HBM: x and the residual read once, y written once.  16384 x 1024 in bf16 with the residual 16 us
// for 101 MB (6.3 TB/s, partly from the caches).
#include <hip/hip_runtime.h>

#include "operators.h"
#include "vectors.h"

namespace pase {
namespace {

// The four words of one call.
__device__ __forceinline__ uint4 philox(uint64_t counter, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
    uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32);
#pragma unroll
    for (int i = 0; i < 10; i++) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0, c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1, c3 = (uint32_t)a;
        k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
    return {c0, c1, c2, c3};
}

constexpr int kEach = 4;   // calls a thread

template <typename T, bool RESIDUAL> __global__ __launch_bounds__(256) void k_dropout(Dropout a) {
    constexpr int V = kVec<T>, N = 8 / V;
    const uint32_t k0 = a.seed[0], k1 = a.seed[1], c2 = a.seed[2], c3 = a.seed[3];
    // the workgroup's first call, by its row and place; the others follow in 32 bits
    const int64_t begin = (a.first + blockIdx.x) * (256 * kEach), row0 = begin / a.calls;
    const uint32_t at0 = (uint32_t)(begin - row0 * a.calls), calls = (uint32_t)a.calls;
#pragma unroll
    for (int k = 0; k < kEach; k++) {
        const uint32_t in = at0 + k * 256 + threadIdx.x, down = in / calls;
        const int64_t row = row0 + down;
        if (row >= a.rows) return;
        const int64_t col = (int64_t)(in - down * calls) * 8, n = a.width - col;
        const T *x = static_cast<const T *>(a.x) + row * a.ldx + col;
        const T *r = static_cast<const T *>(a.residual) + row * a.ldr + col;
        T *y = static_cast<T *>(a.y) + row * a.ldy + col;
        Pack<T> px[N], pr[N];
#pragma unroll
        for (int i = 0; i < N; i++) {
            px[i] = load_pack(x + i * V, n - i * V, (T)0.0f);
            if (RESIDUAL) pr[i] = load_pack(r + i * V, n - i * V, (T)0.0f);
        }
        const uint4 bits = philox((uint64_t)begin + k * 256 + threadIdx.x, c2, c3, k0, k1);
        const uint32_t word[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
        for (int i = 0; i < N; i++) {
#pragma unroll
            for (int j = 0; j < V; j++) {
                const int e = i * V + j;
                const uint32_t number = e & 1 ? word[e >> 1] >> 16 : word[e >> 1] & 0xffff;
                const float kept = number >= a.drop ? (float)px[i].e[j] * a.scale : 0.0f;
                px[i].e[j] = (T)(RESIDUAL ? kept + (float)pr[i].e[j] : kept);
            }
            if (n > i * V) store_pack(y + i * V, n - i * V, px[i]);
        }
    }
}

template <typename T> int go(Dropout a, void *stream) {
    const int64_t blocks = (a.rows * a.calls + 256 * kEach - 1) / (256 * kEach), most = most_blocks(256);
    for (int64_t at = 0; at < blocks; at += most) {
        a.first = at;
        const int64_t n = blocks - at < most ? blocks - at : most;
        if (const int e = a.residual ? launch(k_dropout<T, true>, n, 256, stream, a) : launch(k_dropout<T, false>, n, 256, stream, a))
            return e;
    }
    return 0;
}

}  // namespace

int launch_dropout(const Dropout &a, void *stream) {
    return a.dtype == PASE_BF16 ? go<__bf16>(a, stream) : a.dtype == PASE_FP16 ? go<_Float16>(a, stream) : go<float>(a, stream);
}

}  // namespace pase
