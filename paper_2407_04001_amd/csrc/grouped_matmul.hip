// Matrix products grouped by ragged row ranges, and their gradients
// (pase_operators.h).
//
// Three directions of one product c[m][j] = sum_i A(m, i) B(j, i):
//
//   direction   m            j       i            A            B
//   kForward    rows of e    n       k            x[m][i]      w[e][j][i]
//   kRowsGrad   rows of e    k       n            dy[m][i]     w[e][i][j]
//   kWeights    n            k       rows of e    dy[i][m]     x[i][j]
//
// An operand whose rows run along i in memory ("along") is staged in LDS as
// rows of 64 i, one whose rows run along m or j ("across") as 64 rows of i; the
// matrix instruction wants eight consecutive i a lane, which is a 16-byte LDS
// read of the first and two transposing reads of the second.
#include "operators.h"
#include "vectors.h"

namespace pase {
namespace {

enum Direction { kForward, kRowsGrad, kWeights };

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <typename T> struct Mfma;
template <> struct Mfma<__bf16> {
    typedef __bf16 Frag __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x4 go(Frag a, Frag b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Mfma<_Float16> {
    typedef _Float16 Frag __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x4 go(Frag a, Frag b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};

__device__ __forceinline__ int64_t offset_at(const GroupedProduct &a, int e) {
    int64_t o = a.offsets_64 ? static_cast<const int64_t *>(a.offsets)[e]
                             : (int64_t) static_cast<const int32_t *>(a.offsets)[e];
    return o < 0 ? 0 : o > a.rows ? a.rows : o;
}

// Rows of virtual group v: 0 is the rows before offsets[0], 1 .. groups the
// groups, groups + 1 the rows from offsets[groups] on.
__device__ __forceinline__ void group_rows(const GroupedProduct &a, int v, int64_t &lo, int64_t &hi) {
    lo = v == 0 ? 0 : offset_at(a, v - 1);
    hi = v == a.groups + 1 ? a.rows : offset_at(a, v);
    if (hi < lo) hi = lo;
}

struct Tile {
    int group;         // -1: rows of no group
    int64_t row, end;  // first row, end of its group's rows
    int col;           // column tile
    bool none;
};

// The tile of this workgroup among the row tiles (BM rows; every virtual group
// begins a new one) x `cols` column tiles.  How many row tiles there are is
// known on the device only: the grid is an upper bound, and what is left over
// returns.  Workgroups go round the 8 XCDs by their number, so the tiles are
// dealt such that each XCD has one contiguous run of them, and within a run
// kBand row tiles go through all column tiles together: their A rows stay in
// that XCD's L2 while B passes once per band.
constexpr int kXcds = 8, kBand = 8;

template <int BM> __device__ Tile find_tile(const GroupedProduct &a, int cols) {
    const int lane = threadIdx.x & 63;
    int64_t total = 0;
    for (int v0 = 0; v0 < a.groups + 2; v0 += 64) {
        const int v = v0 + lane;
        int64_t lo = 0, hi = 0;
        if (v < a.groups + 2) group_rows(a, v, lo, hi);
        int t = (int)((hi - lo + BM - 1) / BM);
#pragma unroll
        for (int d = 32; d; d >>= 1) t += __shfl_xor(t, d, 64);
        total += t;
    }
    total = __builtin_amdgcn_readfirstlane((int)total);
    const int64_t tiles = total * cols, per = (tiles + kXcds - 1) / kXcds;
    const int64_t i = blockIdx.x / kXcds, at = (int64_t)(blockIdx.x % kXcds) * per + i;
    Tile out;
    out.none = i >= per || at >= tiles;
    if (out.none) return out;
    const int64_t band = at / (kBand * (int64_t)cols), in = at - band * kBand * cols;
    const int high = (int)(total - band * kBand < kBand ? total - band * kBand : kBand);
    int64_t rest = band * kBand + in % high;
    out.col = (int)(in / high);
    for (int v0 = 0; v0 < a.groups + 2; v0 += 64) {
        const int v = v0 + lane;
        int64_t lo = 0, hi = 0;
        if (v < a.groups + 2) group_rows(a, v, lo, hi);
        const int t = (int)((hi - lo + BM - 1) / BM);
        int upto = t;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d, 64);
            if (lane >= d) upto += o;
        }
        const uint64_t found = __ballot(rest < upto);
        if (found) {
            const int src = __builtin_ctzll(found);
            const int before = __shfl(upto, src, 64) - __shfl(t, src, 64);
            out.row = __shfl(lo, src, 64) + (rest - before) * BM;
            out.end = __shfl(hi, src, 64);
            out.group = v0 + src - 1;
            if (out.group == a.groups) out.group = -1;
            break;
        }
        rest -= __shfl(upto, 63, 64);
    }
    out.group = __builtin_amdgcn_readfirstlane(out.group);
    return out;
}

// LDS places, in 16-byte chunks.  "Along": row r, chunk c (8 i) of a row of 8
// chunks; "across": i row, chunk c (8 columns) of a row of R / 8.  The chunk is
// permuted by a function of the row so that the 16 lanes that read together
// reach different banks.  On the j side a lane's 16 MFMA rows are j = 16 q + 4 t + r
// (q = lane / 4 % 4, r = lane % 4, t the fragment), so that the four fragments
// of a lane end as 16 consecutive columns of c, stored together.
__device__ __forceinline__ int along_m(int r, int c) { return r * 8 + (c ^ ((r >> 1) & 7)); }
__device__ __forceinline__ int along_j(int r, int c) { return r * 8 + (c ^ (((r >> 1) & 1) | ((r >> 3) & 6))); }
template <int R> __device__ __forceinline__ int across_m(int i, int c) {
    return i * (R / 8) + (c ^ (2 * ((i & 3) | ((i >> 1) & 4))));
}
template <int R> __device__ __forceinline__ int across_j(int i, int c) {
    return i * (R / 8) + (c ^ ((i & 1) | ((i & 2) << 2)));
}

// ---------------------------------------------------------------- any alignment
// 128 x 128 tiles, 64 of i at a time; four waves, 64 x 64 each.  Operands go
// through registers, where what lies past an edge becomes 0.
constexpr int kTile = 128, kDepth = 64;

template <typename T, bool ACROSS>
__device__ __forceinline__ void fetch(Pack<T> (&r)[4], const T *base, int64_t ld, int64_t rows, int64_t depth, int64_t i0) {
#pragma unroll
    for (int s = 0; s < 4; s++) {
        const int p = threadIdx.x + s * 256;
        if (ACROSS) {   // 64 rows of i, 16 chunks of m or j
            const int i = p >> 4, c = p & 15;
            r[s] = load_pack(base + (i0 + i) * ld + c * 8, i0 + i < depth ? rows - c * 8 : 0, (T)0.0f);
        } else {        // 128 rows of m or j, 8 chunks of i
            const int row = p >> 3, c = p & 7;
            r[s] = load_pack(base + row * ld + i0 + c * 8, row < rows ? depth - i0 - c * 8 : 0, (T)0.0f);
        }
    }
}

template <typename T, bool ACROSS, bool J> __device__ __forceinline__ void put(Pack<T> *lds, const Pack<T> (&r)[4]) {
#pragma unroll
    for (int s = 0; s < 4; s++) {
        const int p = threadIdx.x + s * 256;
        const int at = ACROSS ? (J ? across_j<kTile>(p >> 4, p & 15) : across_m<kTile>(p >> 4, p & 15))
                              : (J ? along_j(p >> 3, p & 7) : along_m(p >> 3, p & 7));
        lds[at] = r[s];
    }
}

// Fragment t of the wave's 64 rows from `first` on, i = 32 h .. 32 h + 31.
template <typename T, bool ACROSS, bool J, int R>
__device__ __forceinline__ typename Mfma<T>::Frag frag(const Pack<T> *lds, int first, int t, int h) {
    typedef typename Mfma<T>::Frag Frag;
    const int lane = threadIdx.x & 63, l = lane & 15, q = lane >> 4;
    if (!ACROSS) {
        const int r = first + (J ? (l >> 2) * 16 + t * 4 + (l & 3) : t * 16 + l);
        const int c = h * 4 + q;
        return *reinterpret_cast<const Frag *>(lds + (J ? along_j(r, c) : along_m(r, c)));
    }
    // 4 rows of i x 16 columns a transposing read: a lane gives 4 columns of one row, and gets one column's 4 rows
    const int col = first + (J ? (l & 3) * 16 + t * 4 : t * 16 + (l & 3) * 4);
    union {
        Frag f;
        s16x4 half[2];
    } u;
#pragma unroll
    for (int s = 0; s < 2; s++) {
        const int i = h * 32 + q * 8 + s * 4 + (l >> 2);
        const int at = J ? across_j<R>(i, col >> 3) : across_m<R>(i, col >> 3);
        const char *p = reinterpret_cast<const char *>(lds + at) + (col & 4) * 2;
        u.half[s] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4 *)reinterpret_cast<uintptr_t>(p));
    }
    return u.f;
}

// A lane's 16 consecutive columns of one row of c.
template <typename T, typename O> __device__ __forceinline__ void store16(O *p, int64_t n, const f32x4 (&v)[4]) {
    constexpr int V = kVec<O>;
#pragma unroll
    for (int s = 0; s < 16; s += V) {
        Pack<O> o;
#pragma unroll
        for (int j = 0; j < V; j++) o.e[j] = (O)v[(s + j) >> 2][(s + j) & 3];
        if (n > s) store_pack(p + s, n - s, o);
    }
}

template <typename T, typename O, Direction D> __global__ __launch_bounds__(256) void k_product(GroupedProduct a) {
    constexpr bool A_ACROSS = D == kWeights, B_ACROSS = D != kForward;
    __shared__ Pack<T> lds[2][2][kTile * 8];
    const T *x = static_cast<const T *>(a.x), *w = static_cast<const T *>(a.w), *dy = static_cast<const T *>(a.dy);
    const T *A, *B;
    int64_t lda, ldb, m_rows, j_rows, depth;
    O *c = static_cast<O *>(a.out);
    if (D == kWeights) {
        const int nt = (a.n + kTile - 1) / kTile, kt = (a.k + kTile - 1) / kTile;
        const int e = blockIdx.x / (nt * kt), t = blockIdx.x % (nt * kt), m0 = t / kt * kTile, j0 = t % kt * kTile;
        int64_t lo, hi;
        group_rows(a, e + 1, lo, hi);
        A = dy + lo * a.lddy + m0, lda = a.lddy, m_rows = a.n - m0;
        B = x + lo * a.ldx + j0, ldb = a.ldx, j_rows = a.k - j0;
        depth = hi - lo;
        c += ((int64_t)e * a.n + m0) * a.k + j0;
    } else {
        const int cols = D == kForward ? a.n : a.k;
        const Tile t = find_tile<kTile>(a, (cols + kTile - 1) / kTile);
        if (t.none) return;
        const int j0 = t.col * kTile;
        const int64_t e = t.group < 0 ? 0 : t.group;
        m_rows = t.end - t.row, j_rows = cols - j0;
        if (D == kForward) {
            A = x + t.row * a.ldx, lda = a.ldx;
            B = w + (e * a.n + j0) * a.k, ldb = a.k;
            depth = a.k;
        } else {
            A = dy + t.row * a.lddy, lda = a.lddy;
            B = w + e * a.n * a.k + j0, ldb = a.k;
            depth = a.n;
        }
        if (t.group < 0) depth = 0;
        c += t.row * a.ldo + j0;
    }
    const int wave = threadIdx.x >> 6, wm = (wave >> 1) * 64, wj = (wave & 1) * 64;
    f32x4 acc[4][4] = {};
    Pack<T> ra[4], rb[4];
    if (depth > 0) {
        fetch<T, A_ACROSS>(ra, A, lda, m_rows, depth, 0);
        fetch<T, B_ACROSS>(rb, B, ldb, j_rows, depth, 0);
        put<T, A_ACROSS, false>(lds[0][0], ra);
        put<T, B_ACROSS, true>(lds[0][1], rb);
    }
    int at = 0;
    for (int64_t i0 = 0; i0 < depth; i0 += kDepth, at ^= 1) {
        __syncthreads();
        const bool more = i0 + kDepth < depth;
        if (more) {
            fetch<T, A_ACROSS>(ra, A, lda, m_rows, depth, i0 + kDepth);
            fetch<T, B_ACROSS>(rb, B, ldb, j_rows, depth, i0 + kDepth);
        }
#pragma unroll
        for (int h = 0; h < 2; h++) {
            typename Mfma<T>::Frag fa[4], fb[4];
#pragma unroll
            for (int t = 0; t < 4; t++) {
                fa[t] = frag<T, A_ACROSS, false, kTile>(lds[at][0], wm, t, h);
                fb[t] = frag<T, B_ACROSS, true, kTile>(lds[at][1], wj, t, h);
            }
#pragma unroll
            for (int m = 0; m < 4; m++)
#pragma unroll
                for (int j = 0; j < 4; j++) acc[m][j] = Mfma<T>::go(fb[j], fa[m], acc[m][j]);
        }
        if (more) {
            put<T, A_ACROSS, false>(lds[at ^ 1][0], ra);
            put<T, B_ACROSS, true>(lds[at ^ 1][1], rb);
        }
    }
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int m = 0; m < 4; m++) {
        const int row = wm + m * 16 + (lane & 15), col = wj + (lane >> 4) * 16;
        if (row < m_rows && col < j_rows) store16<T, O>(c + row * a.ldo + col, j_rows - col, acc[m]);
    }
}

template <typename T, typename O, Direction D> int go(const GroupedProduct &a, void *stream) {
    int64_t blocks;
    if (D == kWeights) {
        blocks = (int64_t)a.groups * ((a.n + kTile - 1) / kTile) * ((a.k + kTile - 1) / kTile);
    } else {
        const int cols = D == kForward ? a.n : a.k;
        const int64_t tiles = (a.rows / kTile + a.groups + 2) * ((cols + kTile - 1) / kTile);
        blocks = (tiles + kXcds - 1) / kXcds * kXcds;
    }
    return launch(k_product<T, O, D>, blocks, 256, stream, a);
}

template <Direction D> int by_type(const GroupedProduct &a, void *stream) {
    if (a.dtype == PASE_BF16)
        return a.out_dtype == PASE_FP32 ? go<__bf16, float, D>(a, stream) : go<__bf16, __bf16, D>(a, stream);
    return a.out_dtype == PASE_FP32 ? go<_Float16, float, D>(a, stream) : go<_Float16, _Float16, D>(a, stream);
}

}  // namespace

int launch_product_forward(const GroupedProduct &a, void *stream) { return by_type<kForward>(a, stream); }
int launch_product_rows_grad(const GroupedProduct &a, void *stream) { return by_type<kRowsGrad>(a, stream); }
int launch_product_weights_grad(const GroupedProduct &a, void *stream) { return by_type<kWeights>(a, stream); }

}  // namespace pase
