// Residual add + layer norm, forward and backward (pase_operators.h).
//
// A row is held in registers by one team of lanes (8 to 1024 of them), NV 16-byte
// vectors a lane, so that it is read once although the mean, the sum of squared
// deviations and the output each need all of it.  The variance is summed over
// (z - mean)^2, not z^2 - mean^2, whose difference loses digits where the mean
// is large.  Both passes are bound by HBM: they read and write each operand
// once.  16384 x 1024 in bf16 with a residual: forward 26 us for 134 MB (5.1 TB/s),
// backward 36 us (3.7 TB/s; the sums of dgain and dbias, 2 x 4 MB and a second launch,
// are 5 us of it).  200000 x 64: 16 and 24 us; a wave a row there took 77 and 172.
#include "operators.h"
#include "vectors.h"

namespace pase {
namespace {

constexpr int kThreads = 256;   // of a workgroup, unless one team is larger

template <int LANES> constexpr int kBlock = LANES > kThreads ? LANES : kThreads;
template <int LANES> constexpr int kTeams = kBlock<LANES> / LANES;

// Sums over one team, the same in each of its lanes.  A team of several waves is a
// workgroup; `lds` holds N floats a wave.
template <int LANES, int N> __device__ __forceinline__ void team_sum(float (&v)[N], float *lds) {
    if constexpr (LANES > 64) {
        group_sum<LANES / 64>(v, lds);
    } else {
#pragma unroll
        for (int d = LANES / 2; d; d >>= 1)
#pragma unroll
            for (int i = 0; i < N; i++) v[i] += __shfl_xor(v[i], d, 64);
    }
}

template <typename T, typename P, int NV, int LANES>
__global__ __launch_bounds__(kBlock<LANES>) void k_norm_forward(NormForward a) {
    constexpr int V = kVec<T>, kTeam = LANES, WAVES = LANES > 64 ? LANES / 64 : 1;
    static_assert(LANES <= 64 || kTeams<LANES> == 1, "a team of several waves is a workgroup");
    __shared__ float lds[2 * WAVES];
    const int lane = threadIdx.x % kTeam;
    const int64_t row = (int64_t)blockIdx.x * kTeams<LANES> + threadIdx.x / kTeam;
    if (row >= a.rows) return;   // whole teams
    const T *x = static_cast<const T *>(a.x) + row * a.ldx;
    const T *r = static_cast<const T *>(a.residual) + row * a.ldr;
    const float count = (float)a.width;

    float z[NV][V];
    float s[1] = {0};
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int at = (lane + i * kTeam) * V, n = a.width - at;
        const Pack<T> px = load_pack(x + at, n, (T)0.0f);
#pragma unroll
        for (int j = 0; j < V; j++) z[i][j] = (float)px.e[j];
    }
    if (a.residual) {
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int at = (lane + i * kTeam) * V, n = a.width - at;
            const Pack<T> pr = load_pack(r + at, n, (T)0.0f);
#pragma unroll
            for (int j = 0; j < V; j++) z[i][j] += (float)pr.e[j];
        }
    }
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
        for (int j = 0; j < V; j++) s[0] += z[i][j];
    team_sum<LANES>(s, lds);
    const float mean = s[0] / count;
    float q[1] = {0};
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int n = a.width - (lane + i * kTeam) * V;
#pragma unroll
        for (int j = 0; j < V; j++) {
            const float d = j < n ? z[i][j] - mean : 0.0f;
            q[0] += d * d;
        }
    }
    team_sum<LANES>(q, lds + WAVES);
    const float rstd = 1.0f / sqrtf(q[0] / count + a.eps);
    if (lane == 0) a.mean[row] = mean, a.rstd[row] = rstd;

    T *y = static_cast<T *>(a.y) + row * a.ldy;
    T *zo = static_cast<T *>(a.z) + row * a.ldz;
    const P *gain = static_cast<const P *>(a.gain), *bias = static_cast<const P *>(a.bias);
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int at = (lane + i * kTeam) * V, n = a.width - at;
        if (n <= 0) break;
        Pack<T> py, pz;
        float g[V], b[V];
#pragma unroll
        for (int h = 0; h < V; h += kVec<P>) {
            const Pack<P> pg = load_pack(gain + at + h, n - h, (P)0.0f);
            Pack<P> pb;
            pb.v = 0;
            if (bias) pb = load_pack(bias + at + h, n - h, (P)0.0f);
#pragma unroll
            for (int j = 0; j < kVec<P>; j++) g[h + j] = (float)pg.e[j], b[h + j] = (float)pb.e[j];
        }
#pragma unroll
        for (int j = 0; j < V; j++) {
            py.e[j] = (T)((z[i][j] - mean) * rstd * g[j] + b[j]);
            pz.e[j] = (T)z[i][j];
        }
        store_pack(y + at, n, py);
        if (a.z) store_pack(zo + at, n, pz);
    }
}

// dx row by row, a team taking every (teams in the grid)-th row; its lanes keep
// the sums of dy * h and dy over those rows for their own columns, which the
// workgroup adds up and leaves as one row of `partial`.  512 workgroups: 16384 x 1024
// 30.4 us (operands in cache), with 256 of them 40.5, with 1024 35.2 (more sums to
// write and read).
template <typename T, typename P, int NV, int LANES>
__global__ __launch_bounds__(kBlock<LANES>) void k_norm_backward(NormBackward a) {
    constexpr int V = kVec<T>, kTeam = LANES, TEAMS = kTeams<LANES>, WAVES = LANES > 64 ? LANES / 64 : 1;
    __shared__ float lds[2 * 2 * WAVES];
    __shared__ float join[TEAMS > 1 ? TEAMS : 1][TEAMS > 1 ? V * LANES + 4 : 1];
    const int lane = threadIdx.x % kTeam, team = threadIdx.x / kTeam;
    const P *gain = static_cast<const P *>(a.gain);
    const float inv = 1.0f / (float)a.width;
    float dg[NV][V], db[NV][V];
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
        for (int j = 0; j < V; j++) dg[i][j] = db[i][j] = 0;

    // The next row is on its way while this one is reduced.  Teams of 1024 lanes have 128
    // registers a lane, too few for two rows (57 to 109 of them spilled): 4096 x 8200 in bf16 217 us with the
    // next row against 101 without, 4096 x 16384 in fp32 405 against 250; rows of fp32 to 8192, where nothing
    // spills either way, 4096 x 8192 112 us with and without.
    constexpr bool AHEAD = LANES < 1024;
    Pack<T> ny[NV], nz[NV];
    float next_mean = 0, next_rstd = 0;
    const auto fetch = [&](int64_t row) {
        const T *dy = static_cast<const T *>(a.dy) + row * a.lddy, *z = static_cast<const T *>(a.z) + row * a.ldz;
        next_mean = a.mean[row], next_rstd = a.rstd[row];
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int at = (lane + i * kTeam) * V, n = a.width - at;
            ny[i] = load_pack(dy + at, n, (T)0.0f);
            nz[i] = load_pack(z + at, n, (T)0.0f);
        }
    };
    const int64_t first = (int64_t)blockIdx.x * TEAMS + team, stride = (int64_t)gridDim.x * TEAMS;
    if (AHEAD && first < a.rows) fetch(first);
    int odd = 0;
    for (int64_t row = first; row < a.rows; row += stride, odd ^= 1) {
        if (!AHEAD) fetch(row);
        const float mean = next_mean, rstd = next_rstd;
        Pack<T> py[NV], pz[NV];
#pragma unroll
        for (int i = 0; i < NV; i++) py[i] = ny[i], pz[i] = nz[i];
        if (AHEAD && row + stride < a.rows) fetch(row + stride);
        float g[NV][V];
        float s[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int at = (lane + i * kTeam) * V, n = a.width - at;
#pragma unroll
            for (int h = 0; h < V; h += kVec<P>) {
                const Pack<P> pg = load_pack(gain + at + h, n - h, (P)0.0f);
#pragma unroll
                for (int j = 0; j < kVec<P>; j++) g[i][h + j] = (float)pg.e[j];
            }
            // Past the row's end dy and the gain are 0, and z the mean: a 0 there would make h = -mean * rstd, which
            // may be past fp32's range, and 0 * h NaN.  (A select for every element took the registers of a second
            // row: 4096 x 4096 in bf16 67 us against 42.)
            if (n < V)
#pragma unroll
                for (int j = 0; j < V; j++)
                    if (j >= n) pz[i].e[j] = (T)mean;
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float d = (float)py[i].e[j], h = ((float)pz[i].e[j] - mean) * rstd;
                const float dh = d * g[i][j];
                db[i][j] += d;
                dg[i][j] += d * h;
                s[0] += dh;
                s[1] += dh * h;
            }
        }
        team_sum<LANES>(s, lds + odd * 2 * WAVES);
        const float m0 = s[0] * inv, m1 = s[1] * inv;
        const T *dz = static_cast<const T *>(a.dz) + row * a.lddz;
        T *dx = static_cast<T *>(a.dx) + row * a.lddx;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int at = (lane + i * kTeam) * V, n = a.width - at;
            if (n <= 0) break;
            Pack<T> pd, po;
            pd.v = 0;
            if (a.dz) pd = load_pack(dz + at, n, (T)0.0f);
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float h = ((float)pz[i].e[j] - mean) * rstd, dh = (float)py[i].e[j] * g[i][j];
                float d = (dh - m0 - h * m1) * rstd;
                if (a.dz) d += (float)pd.e[j];
                po.e[j] = (T)d;
            }
            store_pack(dx + at, n, po);
        }
    }
    float *out = a.partial + (int64_t)blockIdx.x * 2 * a.width;
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int at = (lane + i * kTeam) * V;
        if (TEAMS == 1) {
#pragma unroll
            for (int h = 0; h < V; h += 4) {
                Pack<float> g, b;
#pragma unroll
                for (int j = 0; j < 4; j++) g.e[j] = dg[i][h + j], b.e[j] = db[i][h + j];
                store_pack(out + at + h, a.width - at - h, g);
                store_pack(out + a.width + at + h, a.width - at - h, b);
            }
        } else {   // the teams' LANES V columns of this i, one team after the other
#pragma unroll
            for (int which = 0; which < 2; which++) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < V; j++) join[team][j * LANES + lane] = which ? db[i][j] : dg[i][j];
                __syncthreads();
                for (int c = threadIdx.x; c < V * LANES; c += kBlock<LANES>) {
                    const int col = i * LANES * V + c, slot = (c % V) * LANES + c / V;
                    float s = 0;
#pragma unroll
                    for (int t = 0; t < TEAMS; t++) s += join[t][slot];
                    if (col < a.width) out[which * a.width + col] = s;
                }
            }
        }
    }
}

// dgain and dbias: the column sums of `partial`, 64 columns a workgroup, its 16
// waves each taking every 16th row.
template <typename P> __global__ __launch_bounds__(1024) void k_norm_sums(NormBackward a) {
    __shared__ float join[16][65];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane, cols = 2 * (int64_t)a.width;
    float s = 0;
    if (col < cols)
#pragma unroll 8
        for (int b = wave; b < a.blocks; b += 16) s += a.partial[b * cols + col];
    join[wave][lane] = s;
    __syncthreads();
    if (wave || col >= cols) return;
    s = 0;
#pragma unroll
    for (int w = 0; w < 16; w++) s += join[w][lane];
    P *out = static_cast<P *>(col < a.width ? a.dgain : a.dbias);
    if (out) out[col < a.width ? col : col - a.width] = (P)s;
}

// Teams by row length: the fewest lanes that hold the row in up to four vectors each
// (two in teams below a wave, which keeps the rows of a wave's loads close).
template <typename T, typename P, typename F> int by_width(int width, F &&f) {
    const int vecs = norm_vectors(width, sizeof(T));
    switch (norm_lanes(vecs)) {
    case 8: return vecs <= 8 ? f.template operator()<T, P, 1, 8>() : f.template operator()<T, P, 2, 8>();
    case 16: return f.template operator()<T, P, 2, 16>();
    case 32: return f.template operator()<T, P, 2, 32>();
    case 64: return vecs <= 128 ? f.template operator()<T, P, 2, 64>() : f.template operator()<T, P, 4, 64>();
    case 256: return f.template operator()<T, P, 4, 256>();
    default:
        if (vecs <= 2048) return f.template operator()<T, P, 2, 1024>();
        if constexpr (sizeof(T) == 4) return f.template operator()<T, P, 4, 1024>();
        return (int)hipErrorInvalidValue;   // wider than PASE_NORM_MAX_WIDTH: refused before
    }
}

template <typename F> int by_type(int dtype, int param_dtype, int width, F &&f) {
    if (dtype == PASE_FP32) return by_width<float, float>(width, f);
    if (dtype == PASE_BF16)
        return param_dtype == PASE_FP32 ? by_width<__bf16, float>(width, f) : by_width<__bf16, __bf16>(width, f);
    return param_dtype == PASE_FP32 ? by_width<_Float16, float>(width, f) : by_width<_Float16, _Float16>(width, f);
}

struct Forward {
    const NormForward &a;
    void *stream;
    template <typename T, typename P, int NV, int LANES> int operator()() {
        constexpr int TEAMS = kTeams<LANES>, THREADS = kBlock<LANES>;
        const int64_t most = most_blocks(THREADS) * TEAMS;
        for (int64_t row = 0; row < a.rows; row += most) {
            NormForward part = a;
            part.rows = a.rows - row < most ? a.rows - row : most;
            part.x = static_cast<const T *>(a.x) + row * a.ldx;
            if (a.residual) part.residual = static_cast<const T *>(a.residual) + row * a.ldr;
            part.y = static_cast<T *>(a.y) + row * a.ldy;
            if (a.z) part.z = static_cast<T *>(a.z) + row * a.ldz;
            part.mean = a.mean + row, part.rstd = a.rstd + row;
            if (const int e = launch(k_norm_forward<T, P, NV, LANES>, (part.rows + TEAMS - 1) / TEAMS, THREADS, stream, part)) return e;
        }
        return 0;
    }
};

struct Backward {
    const NormBackward &a;
    void *stream;
    template <typename T, typename P, int NV, int LANES> int operator()() {
        if (a.blocks)
            if (const int e = launch(k_norm_backward<T, P, NV, LANES>, a.blocks, kBlock<LANES>, stream, a)) return e;
        if (!a.dgain && !a.dbias) return 0;
        return launch(k_norm_sums<P>, (2 * (int64_t)a.width + 63) / 64, 1024, stream, a);
    }
};

}  // namespace

int launch_norm_forward(const NormForward &a, void *stream) {
    return by_type(a.dtype, a.param_dtype, a.width, Forward{a, stream});
}

int launch_norm_backward(const NormBackward &a, void *stream) {
    return by_type(a.dtype, a.param_dtype, a.width, Backward{a, stream});
}

const char *launch_error(int e) { return hipGetErrorString((hipError_t)e); }

}  // namespace pase
