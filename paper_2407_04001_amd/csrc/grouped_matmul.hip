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
#include "lds.h"
#include "operators.h"
#include "vectors.h"

namespace pase {
namespace {

enum Direction { kForward, kRowsGrad, kWeights };

typedef float f32x4 __attribute__((ext_vector_type(4)));

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

// 64 virtual groups from `first` on, one a lane: virtual group 0 is the rows before
// offsets[0], 1 .. groups the groups, groups + 1 the rows from offsets[groups] on.
// `before` is where the one before `first` ends.  Offsets are kept within 0 .. rows
// and not below any earlier one, so that every row has one virtual group whatever
// they hold.
struct Ranges {
    int lo, hi;
    int tiles, upto;   // of BM rows: this group's, and those up to and with it

    __device__ __forceinline__ Ranges(const GroupedProduct &a, int first, int before, int bm) {
        const int lane = threadIdx.x & 63, v = first + lane;
        int64_t o = a.rows;
        if (v <= a.groups)
            o = a.offsets_64 ? static_cast<const int64_t *>(a.offsets)[v]
                             : (int64_t) static_cast<const int32_t *>(a.offsets)[v];
        o = o > a.rows ? a.rows : o;
        hi = o < before ? before : (int)o;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(hi, d, 64);
            if (lane >= d && o > hi) hi = o;
        }
        lo = __shfl_up(hi, 1, 64);
        if (lane == 0) lo = before;
        upto = tiles = (int)(((uint32_t)(hi - lo) + bm - 1) / bm);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d, 64);
            if (lane >= d) upto += o;
        }
    }
    __device__ __forceinline__ int end() const { return __builtin_amdgcn_readlane(hi, 63); }
    __device__ __forceinline__ int all() const { return __builtin_amdgcn_readlane(upto, 63); }
};

struct Tile {
    int group;         // -1: rows of no group
    int row, end;      // first row, end of its group's rows
    int col;           // column tile
    bool none;
};

// The tiles of BM rows (every virtual group begins a new one) x `cols` columns of
// tiles, dealt to the workgroups.  How many row tiles there are is known on the
// device only: the grid is an upper bound, or as many workgroups as run at once,
// each taking every (grid)-th.  Workgroups go round the 8 XCDs by their number,
// so each XCD gets one contiguous run of the tiles, and within a run kBand row
// tiles go through all column tiles together: their A rows stay in that XCD's L2
// while B passes once per band.
constexpr int kXcds = 8, kBand = 8;

template <int BM> struct Deal {
    uint32_t cols, total, per;   // row tiles; tiles of an XCD's run

    __device__ __forceinline__ Deal(const GroupedProduct &a, int cols_) {
        cols = cols_, total = 0;
        int before = 0;
        for (int v = 0; v < a.groups + 2; v += 64) {
            const Ranges r(a, v, before, BM);
            total += r.all();
            before = r.end();
        }
        per = (total * cols + kXcds - 1) / kXcds;
    }

    // The i-th tile of this workgroup's run.
    __device__ __forceinline__ Tile get(const GroupedProduct &a, uint32_t i) const {
        Tile out;
        const uint32_t at = blockIdx.x % kXcds * per + i;
        out.none = i >= per || at >= total * cols;
        if (out.none) return out;
        const uint32_t band = at / (kBand * cols), in = at - band * kBand * cols;
        const uint32_t high = total - band * kBand < kBand ? total - band * kBand : kBand;
        // (quotients are formed in vector registers)
        out.col = __builtin_amdgcn_readfirstlane(in / high);
        int rest = __builtin_amdgcn_readfirstlane(band * kBand + in % high);
        int before = 0;
        for (int v = 0;; v += 64) {
            const Ranges r(a, v, before, BM);
            const uint64_t found = __ballot(rest < r.upto);
            if (found) {
                const int src = __builtin_ctzll(found), first = __builtin_amdgcn_readlane(r.upto - r.tiles, src);
                out.row = __builtin_amdgcn_readlane(r.lo, src) + (rest - first) * BM;
                out.end = __builtin_amdgcn_readlane(r.hi, src);
                out.group = v + src - 1 == a.groups ? -1 : v + src - 1;
                return out;
            }
            rest -= r.all();
            before = r.end();
        }
    }
};

// Rows of group e.
__device__ __forceinline__ void group_rows(const GroupedProduct &a, int e, int &lo, int &hi) {
    int before = 0;
    for (int v = 0;; v += 64) {
        const Ranges r(a, v, before, 1 << 30);
        if (e + 1 < v + 64) {
            lo = __builtin_amdgcn_readlane(r.lo, e + 1 - v), hi = __builtin_amdgcn_readlane(r.hi, e + 1 - v);
            return;
        }
        before = r.end();
    }
}

// The group with the `rank`-th most rows (ties to the lower one): the weights' gradient
// begins with the longest groups, so that the workgroups that start last have the
// least to do.  More groups than lanes keep their own order; their lengths even out.
__device__ __forceinline__ int longest(const GroupedProduct &a, int rank) {
    if (a.groups == 1 || a.groups > 62) return rank;
    const Ranges r(a, 0, 0, 1 << 30);
    const int lane = threadIdx.x & 63;
    const int mine = lane >= 1 && lane <= a.groups ? r.hi - r.lo : -1;
    int above = 0;
    for (int l = 1; l <= a.groups; l++) {
        const int other = __builtin_amdgcn_readlane(mine, l);
        above += other > mine || (other == mine && l < lane);
    }
    return __builtin_ctzll(__ballot(mine >= 0 && above == rank)) - 1;
}

// LDS places, in 16-byte chunks.  "Along": row r, chunk c (8 i) of a row of 8
// chunks; "across": i row, chunk c (8 columns) of a row of R / 8.  The chunk is
// permuted by a function of the row so that the 16 lanes that read together
// reach different banks.  On the j side fragment t's MFMA rows are j = 32 (t / 2) +
// 8 q + 4 (t % 2) + r (q = lane / 4 % 4, r = lane % 4), so that two fragments of a lane
// end as 8 consecutive columns of c, and four lanes' stores as 64 adjacent bytes.
__device__ __forceinline__ int along_m(int r, int c) { return r * 8 + (c ^ ((r >> 1) & 7)); }
__device__ __forceinline__ int along_j(int r, int c) { return r * 8 + (c ^ (((r >> 1) & 1) | ((r >> 2) & 6))); }
template <int R> __device__ __forceinline__ int across_m(int i, int c) {
    return i * (R / 8) + (c ^ (2 * ((i & 3) | ((i >> 1) & 4))));
}
template <int R> __device__ __forceinline__ int across_j(int i, int c) { return i * (R / 8) + (c ^ ((i & 3) << 2)); }

// What one workgroup computes at a time: m_rows x j_rows of c (at most a tile of
// them) from `depth` of the contraction.
template <typename T, typename O> struct Part {
    const T *a, *b;
    O *c;
    int lda, ldb, m_rows, j_rows, depth;

    // One tile of the forward product or the rows' gradient.
    template <Direction D, int BM, int BN> __device__ __forceinline__ void rows(const GroupedProduct &g, const Tile &t) {
        const T *x = static_cast<const T *>(g.x), *w = static_cast<const T *>(g.w), *dy = static_cast<const T *>(g.dy);
        const int j0 = t.col * BN;
        const int64_t e = t.group < 0 ? 0 : t.group;
        m_rows = t.end - t.row, j_rows = (D == kForward ? g.n : g.k) - j0;
        if (D == kForward) {
            a = x + t.row * g.ldx, lda = (int)g.ldx;
            b = w + (e * g.n + j0) * g.k, ldb = g.k;
            depth = g.k;
        } else {
            a = dy + t.row * g.lddy, lda = (int)g.lddy;
            b = w + e * g.n * g.k + j0, ldb = g.k;
            depth = g.n;
        }
        if (t.group < 0) depth = 0;
        c = static_cast<O *>(g.out) + t.row * g.ldo + j0;
    }

    // This workgroup's tile of the weights' gradient: of one group, or of one of the
    // a.splits equal runs of 64-row steps that the group's rows are cut into (each
    // run's sums are a matrix of their own).
    template <int BM, int BN> __device__ __forceinline__ void weights(const GroupedProduct &g) {
        const uint32_t nt = (g.n + BM - 1) / BM, kt = (g.k + BN - 1) / BN, tiles = nt * kt;
        const uint32_t block = g.first + blockIdx.x, item = __builtin_amdgcn_readfirstlane(block / tiles);
        // workgroups go round the XCDs: an XCD gets neighbouring tiles of a group
        uint32_t t = block - item * tiles;
        if (tiles % kXcds == 0) t = t % kXcds * (tiles / kXcds) + t / kXcds;
        const int m0 = __builtin_amdgcn_readfirstlane(t / kt * BM), j0 = __builtin_amdgcn_readfirstlane(t % kt * BN);
        const int part = __builtin_amdgcn_readfirstlane(item / g.groups), e = longest(g, item - part * g.groups);
        int lo, hi;
        group_rows(g, e, lo, hi);
        if (g.splits > 1) {
            const uint32_t steps = (hi - lo + 63) >> 6;
            const int from = __builtin_amdgcn_readfirstlane((uint64_t)steps * part / g.splits) * 64;
            const int to = __builtin_amdgcn_readfirstlane((uint64_t)steps * (part + 1) / g.splits) * 64;
            hi = lo + to < hi ? lo + to : hi;
            lo += from;
        }
        a = static_cast<const T *>(g.dy) + lo * g.lddy + m0, lda = (int)g.lddy, m_rows = g.n - m0;
        b = static_cast<const T *>(g.x) + lo * g.ldx + j0, ldb = (int)g.ldx, j_rows = g.k - j0;
        depth = hi - lo;
        c = static_cast<O *>(g.out) + (((int64_t)part * g.groups + e) * g.n + m0) * g.k + j0;
    }
};

// ---------------------------------------------------------------- any alignment
// Where a row may begin at an odd element.  128 x 128 tiles, 64 of i at a time; four waves, 64 x 64 each.  Operands go
// through registers, where what lies past an edge becomes 0.  Bound by the latency of
// those loads, one step ahead: 16384 x 1023 -> 4095 in 8 ragged groups 317 us (433
// TFLOP/s), 487 with one workgroup a CU and every load tested against the edges.
constexpr int kTile = 128, kDepth = 64;

template <typename T, bool ACROSS>
__device__ __forceinline__ void fetch(Pack<T> (&r)[4], const T *base, int64_t ld, int64_t rows, int64_t depth, int64_t i0) {
    if (rows >= kTile && i0 + kDepth <= depth) {   // nothing past an edge: four loads in flight, no tests between
#pragma unroll
        for (int s = 0; s < 4; s++) {
            const int p = threadIdx.x + s * 256;
            const T *from = ACROSS ? base + (i0 + (p >> 4)) * ld + (p & 15) * 8 : base + (p >> 3) * ld + i0 + (p & 7) * 8;
            r[s].v = reinterpret_cast<const Unaligned16<T> *>(from)->v;
        }
        return;
    }
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
        const int r = first + (J ? (t >> 1) * 32 + (l >> 2) * 8 + (t & 1) * 4 + (l & 3) : t * 16 + l);
        const int c = h * 4 + q;
        return *reinterpret_cast<const Frag *>(lds + (J ? along_j(r, c) : along_m(r, c)));
    }
    // 4 rows of i x 16 columns a transposing read: a lane gives 4 columns of one row, and gets one column's 4 rows
    const int col = first + (J ? (t >> 1) * 32 + (l & 3) * 8 + (t & 1) * 4 : t * 16 + (l & 3) * 4);
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

// A lane's columns of one row of c, of the n that exist from p on: 8 and, 32 on, 8
// (PAIRED fragments), or four times 4, 16 apart.
template <bool PAIRED, typename O> __device__ __forceinline__ void store_row(O *p, int n, const f32x4 (&v)[4]) {
    constexpr int V = kVec<O>;
#pragma unroll
    for (int s = 0; s < 16; s += V) {
        const int at = PAIRED ? (s & 7) + (s >> 3) * 32 : s * 4;
        Pack<O> o;
#pragma unroll
        for (int j = 0; j < V; j++) o.e[j] = (O)v[(s + j) >> 2][(s + j) & 3];
        if (n > at) store_pack(p + at, n - at, o);
    }
}

template <typename T, typename O, Direction D> __global__ __launch_bounds__(256, 2) void k_product(GroupedProduct a) {
    constexpr bool A_ACROSS = D == kWeights, B_ACROSS = D != kForward;
    __shared__ Pack<T> lds[2][2][kTile * 8];
    Part<T, O> p;
    if (D == kWeights) {
        p.template weights<kTile, kTile>(a);
    } else {
        const Tile t = Deal<kTile>(a, ((D == kForward ? a.n : a.k) + kTile - 1) / kTile).get(a, a.first + blockIdx.x / kXcds);
        if (t.none) return;
        p.template rows<D, kTile, kTile>(a, t);
    }
    const T *A = p.a, *B = p.b;
    const int64_t lda = p.lda, ldb = p.ldb, m_rows = p.m_rows, j_rows = p.j_rows, depth = p.depth;
    O *c = p.c;
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
        const int row = wm + m * 16 + (lane & 15), col = wj + (lane >> 4) * 8;
        if (row < m_rows && col < j_rows) store_row<true>(c + row * a.ldo + col, (int)(j_rows - col), acc[m]);
    }
}

// ---------------------------------------------------------------- 4-byte aligned rows
// 256 x 256 tiles, 64 of i at a time, eight waves of 128 x 64.  The operands go
// from HBM to LDS without passing registers (buffer loads to LDS, 16 bytes a
// lane): the buffer's range ends at the operand's last element, so what a tile
// overhangs reads as 0.  Only what lies past i = depth in a row along i is
// inside that range; the fragments of the last step are masked there.
// 16384 x 4096 x 4096 in bf16 402-412 us (1.34 PFLOP/s; the library's own 1.3-1.68 on
// like shapes): the matrix units are busy for 60 % of the cycles at the 1.96 GHz the
// card holds.  Without its loads the loop takes 360 us, without its LDS reads 377,
// without both 303: it is bound by neither alone.  Tried and slower: 128 x 256 tiles,
// two workgroups a CU (522); stages of 32 i, four deep (455-482); two groups of waves
// a barrier apart, one reading while the other multiplies (446).
// 16384 x 1024 -> 4096 in 8 even groups 123 us (1.12 PFLOP/s), in ragged ones 142-163:
// the last round of tiles is then nearly empty, and bound by latency (halving its
// tiles changed nothing).
constexpr int kStage = 2 * kBig * 8 * 16;   // bytes of one step's two operands in LDS

// One operand's loads: 4 of 16 bytes a lane and step, each 64 rows (along) or 16 i
// (across) on from the one before.
template <typename T, bool ACROSS, bool J> struct Feed {
    const char *base;     // of the step to load next
    int left;             // i from that step on
    int ld;               // bytes
    int rows, at[4];      // rows (along) or columns (across) that exist; the lane's byte offsets
    u32x4 range;          // buffer descriptor of the step being loaded; empty past the last
    uint32_t dst;

    __device__ __forceinline__ explicit Feed(int ld_elems) {
        ld = ld_elems * 2;
        const int q = threadIdx.x;   // LDS chunk the lane's first load fills; the permutation is its own inverse
        if (ACROSS)
            at[0] = (q >> 5) * ld + ((J ? across_j<kBig>(q >> 5, q & 31) : across_m<kBig>(q >> 5, q & 31)) & 31) * 16;
        else
            at[0] = (q >> 3) * ld + ((J ? along_j(q >> 3, q & 7) : along_m(q >> 3, q & 7)) & 7) * 16;
#pragma unroll
        for (int s = 1; s < 4; s++) at[s] = at[0] + s * (ACROSS ? 16 : 64) * ld;
    }

    __device__ __forceinline__ void turn_to(const T *p, int have, int depth) {
        base = reinterpret_cast<const char *>(p), left = depth;
        rows = have < kBig ? have : kBig;
    }

    __device__ __forceinline__ void next(const char *lds) {
        // below 2^31, as 256 rows are; checked by words of 4 bytes, so the last element's own word has to be inside
        uint32_t bytes = ACROSS ? ((left < 64 ? left : 64) - 1) * ld + rows * 2 : (rows - 1) * ld + left * 2;
        bytes = left > 0 ? (bytes + 3) & ~3u : 0;
        const uint64_t at0 = reinterpret_cast<uint64_t>(base);
        range = u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)at0),
                      (uint32_t)__builtin_amdgcn_readfirstlane((int)(at0 >> 32) & 0xffff),
                      (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000};
        dst = lds_address(lds) + (__builtin_amdgcn_readfirstlane(threadIdx.x) >> 6) * 1024;
        base += ACROSS ? 64 * (int64_t)ld : 128;
        left -= 64;
    }

    __device__ __forceinline__ void issue(int s) { load_to_lds(range, at[s], dst + s * 8192); }

    __device__ __forceinline__ void load(const char *lds) {
        next(lds);
#pragma unroll
        for (int s = 0; s < 4; s++) issue(s);
    }
};

// The same fragments as frag(), by byte address: `at` is `base` plus the address
// of the operand's stage.  One address register an operand, from which each
// fragment's place follows by an exclusive or and a constant.
template <typename T, bool ACROSS, bool J> struct Reader {
    typedef typename Mfma<T>::Frag Frag;
    uint32_t base;

    __device__ __forceinline__ explicit Reader(int first) {
        const int lane = threadIdx.x & 63, l = lane & 15, q = lane >> 4;
        if (ACROSS) {
            const int i = q * 8 + (l >> 2), col = first + (J ? (l & 3) * 8 : (l & 3) * 4);
            base = (J ? across_j<kBig>(i, col >> 3) : across_m<kBig>(i, col >> 3)) * 16 + (col & 4) * 2;
        } else {
            const int r = first + (J ? (l >> 2) * 8 + (l & 3) : l);
            base = (J ? along_j(r, q) : along_m(r, q)) * 16;
        }
    }

    static __device__ __forceinline__ void read(Frag &to, uint32_t at, int t, int h) {
        if (!ACROSS) {
            to = *(__attribute__((address_space(3))) const Frag *)(uintptr_t)((at ^ (h * 64)) + (J ? (t >> 1) * 4096 + (t & 1) * 512 : t * 2048));
            return;
        }
        union {
            Frag f;
            s16x4 half[2];
        } u;
        const uint32_t col = J ? (at ^ ((t >> 1) * 64)) + (t & 1) * 8 : at ^ (t * 32);
#pragma unroll
        for (int s = 0; s < 2; s++)
            u.half[s] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4 *)(uintptr_t)(col + (h * 32 + s * 4) * (kBig * 2)));
        to = u.f;
    }
};

template <typename F> __device__ __forceinline__ void mask_frag(F &f, int left) {
    union {
        F f;
        uint32_t d[4];
    } u;
    u.f = f;
#pragma unroll
    for (int j = 0; j < 4; j++) u.d[j] = left >= 2 * j + 2 ? u.d[j] : left == 2 * j + 1 ? u.d[j] & 0xffff : 0;
    f = u.f;
}

template <typename T, typename O, Direction D> __global__ __launch_bounds__(512) void k_product_big(GroupedProduct a) {
    constexpr bool A_ACROSS = D == kWeights, B_ACROSS = D != kForward;
    // A lane's 16 bytes of c are one fragment's 4 columns in fp32 and two fragments' 8
    // in 16 bits: the j side's rows are in order in the first case, paired in the second.
    constexpr bool PAIRED = sizeof(O) == 2;
    typedef typename Mfma<T>::Frag Frag;
    __shared__ __attribute__((aligned(1024))) char lds[2][kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = (wave >> 2) * 128, wj = (wave & 3) * 64;
    // A step is four groups of 16 products: i halves h, and for each the wave's upper
    // and lower rows of A.  Each group's fragments are read while the group before
    // it multiplies.  By the middle of a step all of it has been read and the next
    // step has arrived, so one barrier a step is enough: after it the step after next
    // is loaded into this step's half of LDS.
    Frag f[3][4], g[2][4];
    f32x4 acc[8][4];
    const Reader<T, A_ACROSS, false> ra(wm);
    const Reader<T, B_ACROSS, PAIRED> rb(wj);
    const uint32_t stage0 = lds_address(lds[0]);
    // four products, and what is issued behind them
    const auto multiply = [&](const Frag &fm, const Frag(&gj)[4], int m) {
#pragma unroll
        for (int j = 0; j < 4; j++) acc[m][j] = Mfma<T>::go(gj[j], fm, acc[m][j]);
    };
    const auto mask = [&](Frag(&of)[4], int left, int h) {
#pragma unroll
        for (int m = 0; m < 4; m++) mask_frag(of[m], left - h * 32 - ((threadIdx.x & 63) >> 4) * 8);
    };

    Part<T, O> p;
    const Deal<kBig> deal(a, D == kWeights ? 1 : ((D == kForward ? a.n : a.k) + kBig - 1) / kBig);
    uint32_t turn = blockIdx.x / kXcds;
    if (D == kWeights) {
        p.template weights<kBig, kBig>(a);
    } else {
        const Tile t = deal.get(a, turn);
        if (t.none) return;
        p.template rows<D, kBig, kBig>(a, t);
    }
    Feed<T, A_ACROSS, false> fa(p.lda);
    Feed<T, B_ACROSS, PAIRED> fb(p.ldb);
    // the first two steps of a tile; the second may be past its end
    const auto feed = [&]() {
        if (p.depth <= 0) return;
        fa.turn_to(p.a, p.m_rows, p.depth);
        fb.turn_to(p.b, p.j_rows, p.depth);
#pragma unroll
        for (int u = 0; u < 2; u++) {
            fa.load(lds[u]);
            fb.load(lds[u] + kStage / 2);
        }
    };
    feed();
    for (;;) {
        Tile after;
        after.none = true;
        if (D != kWeights) after = deal.get(a, turn += gridDim.x / kXcds);
#pragma unroll
        for (int m = 0; m < 8; m++)
#pragma unroll
            for (int j = 0; j < 4; j++) acc[m][j] = 0.0f;
        if (p.depth > 0) {
            const int steps = (p.depth + 63) >> 6;
            wait_loads<8>();   // this tile's second step may be on its way
            barrier();
            // this step's and the next step's places, each operand's; the compiler would
            // keep every fragment's address of both in registers, more than there are
            uint32_t at_a = stage0 + ra.base, at_b = stage0 + kStage / 2 + rb.base;
            uint32_t other_a = at_a + kStage, other_b = at_b + kStage;
#pragma unroll
            for (int m = 0; m < 4; m++) rb.read(g[0][m], at_b, m, 0), ra.read(f[0][m], at_a, m, 0);
            for (int t = 0; t + 1 < steps; t++) {
                char *cur = lds[t & 1];
                asm volatile("" : "+v"(at_a), "+v"(at_b), "+v"(other_a), "+v"(other_b));
#pragma unroll
                for (int m = 0; m < 4; m++) {
                    multiply(f[0][m], g[0], m);
                    __builtin_amdgcn_sched_barrier(0);
                    ra.read(f[1][m], at_a, 4 + m, 0);
                    ra.read(f[2][m], at_a, m, 1);
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int m = 0; m < 4; m++) {
                    multiply(f[1][m], g[0], 4 + m);
                    __builtin_amdgcn_sched_barrier(0);
                    if (m < 2) {
#pragma unroll
                        for (int k = 2 * m; k < 2 * m + 2; k++) rb.read(g[1][k], at_b, k, 1), ra.read(f[0][k], at_a, 4 + k, 1);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                fa.next(cur);
                fb.next(cur + kStage / 2);
                wait_loads<0>();   // all are the next step's
                barrier();
#pragma unroll
                for (int m = 0; m < 4; m++) {
                    multiply(f[2][m], g[1], m);
                    __builtin_amdgcn_sched_barrier(0);
                    fa.issue(m);
                    rb.read(g[0][m], other_b, m, 0);
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int m = 0; m < 4; m++) {
                    multiply(f[0][m], g[1], 4 + m);
                    __builtin_amdgcn_sched_barrier(0);
                    ra.read(f[0][m], other_a, m, 0);
                    fb.issue(m);
                    __builtin_amdgcn_sched_barrier(0);
                }
                const uint32_t ta = at_a, tb = at_b;
                at_a = other_a, at_b = other_b, other_a = ta, other_b = tb;
            }
            const int left = p.depth - (steps - 1) * 64;
#pragma unroll
            for (int h = 0; h < 2; h++) {
#pragma unroll
                for (int m = 0; m < 4; m++) {
                    if (h) rb.read(g[0][m], at_b, m, 1), ra.read(f[0][m], at_a, m, 1);
                    ra.read(f[1][m], at_a, 4 + m, h);
                }
                if (D != kWeights) {   // along i, what lies past the end is not 0; across, it is
                    mask(f[0], left, h);
                    mask(f[1], left, h);
                    if (!B_ACROSS) mask(g[0], left, h);
                }
#pragma unroll
                for (int m = 0; m < 8; m++) multiply(f[m >> 2][m & 3], g[0], m);
            }
        }
        // the last loads, past the end, filled LDS with 0; nobody reads LDS any more
        wait_loads<0>();
        barrier();
        O *c = p.c;
        const int m_rows = p.m_rows, j_rows = p.j_rows;
        if (!after.none) {   // the next tile's loads go before this one's stores; finding the tile after it waits for both
            p.template rows<D, kBig, kBig>(a, after);
            feed();
        }
        const int row = wm + (lane & 15), col = wj + (lane >> 4) * kVec<O>;
        c += row * a.ldo + col;
        if (m_rows >= kBig && j_rows >= kBig) {
#pragma unroll
            for (int m = 0; m < 8; m++) store_row<PAIRED>(c + m * 16 * a.ldo, 64, acc[m]);
        } else {
#pragma unroll
            for (int m = 0; m < 8; m++)
                if (row + m * 16 < m_rows && col < j_rows) store_row<PAIRED>(c + m * 16 * a.ldo, j_rows - col, acc[m]);
        }
        if (after.none) return;
    }
}

// ---------------------------------------------------------------- few rows
// Forward with few rows a group: what counts is reading each weight once.  A
// workgroup takes 16 MT rows and 32 columns; its four waves take every fourth 32 of
// the contraction, straight from HBM to the matrix unit (a lane's 16 bytes are its
// part of a fragment), and add up through LDS.  Bound by HBM and latency: 64 rows in 8
// groups of 1024 x 4096 (67 MB) 16-18 us, 3.7-4.2 TB/s.
template <typename T, typename O, int MT> __global__ __launch_bounds__(256) void k_product_thin(GroupedProduct a) {
    typedef typename Mfma<T>::Frag Frag;
    union Piece {
        Pack<T> p;
        Frag f;
    };
    constexpr int JT = 2, BM = 16 * MT, BN = 16 * JT;
    __shared__ f32x4 join[3][MT * JT][64];
    const Tile tile = Deal<BM>(a, (a.n + BN - 1) / BN).get(a, a.first + blockIdx.x / kXcds);
    if (tile.none) return;
    Part<T, O> p;
    p.template rows<kForward, BM, BN>(a, tile);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, q = lane >> 4;
    f32x4 acc[MT][JT] = {};
    // rows past the end read the last one again; they are not stored
    const T *pa[MT], *pb[JT];
#pragma unroll
    for (int m = 0; m < MT; m++) {
        const int r = m * 16 + l;
        pa[m] = p.a + (int64_t)(r < p.m_rows ? r : p.m_rows - 1) * p.lda;
    }
#pragma unroll
    for (int j = 0; j < JT; j++) {   // MFMA row 4 h + r of fragment j is column 8 h + 4 j + r, as in frag()
        const int r = (l >> 2) * 8 + j * 4 + (l & 3);
        pb[j] = p.b + (int64_t)(r < p.j_rows ? r : p.j_rows - 1) * p.ldb;
    }
    // (Holding the next pieces in registers as well was no faster: 12-24 rows a group
    // 20.7-26.2 us against 18.7-22.7, 8 groups of 1024 x 4096.)
    const auto step = [&](int i, int n) {   // n: how many of this lane's 8 exist; the rest are 0
        Piece fa[MT], fb[JT];
#pragma unroll
        for (int j = 0; j < JT; j++) fb[j].p = load_pack(pb[j] + i, n, (T)0.0f);
#pragma unroll
        for (int m = 0; m < MT; m++) fa[m].p = load_pack(pa[m] + i, n, (T)0.0f);
#pragma unroll
        for (int m = 0; m < MT; m++)
#pragma unroll
            for (int j = 0; j < JT; j++) acc[m][j] = Mfma<T>::go(fb[j].f, fa[m].f, acc[m][j]);
    };
    const int whole = p.depth & ~127, tail = whole + wave * 32;
    for (int i = wave * 32; i < whole; i += 128) step(i + q * 8, 8);
    if (tail < p.depth) step(tail + q * 8, p.depth - tail - q * 8);
    if (wave)
#pragma unroll
        for (int t = 0; t < MT * JT; t++) join[wave - 1][t][lane] = acc[t / JT][t % JT];
    __syncthreads();
    if (wave) return;
    const int col = q * 8;
    constexpr int V = kVec<O>;
#pragma unroll
    for (int m = 0; m < MT; m++) {
#pragma unroll
        for (int j = 0; j < JT; j++)
#pragma unroll
            for (int w = 0; w < 3; w++) acc[m][j] += join[w][m * JT + j][lane];
        const int r = m * 16 + l;
        if (r >= p.m_rows) continue;
        O *c = p.c + r * a.ldo + col;
#pragma unroll
        for (int s = 0; s < 8; s += V) {
            Pack<O> o;
#pragma unroll
            for (int j = 0; j < V; j++) o.e[j] = (O)acc[m][(s + j) >> 2][(s + j) & 3];
            if (p.j_rows > col + s) store_pack(c + s, p.j_rows - col - s, o);
        }
    }
}

// The rows' gradient with few rows a group: as above with 64 columns a workgroup, but
// w's rows run across, so each wave passes its 32 x 64 of w through LDS of its own
// (no barriers) for the transposing reads.  The next 32 are loaded meanwhile.  The
// same 64 rows: 27 us (32 turns of a load's latency), 16 us with n and k exchanged.
template <typename T, int MT> __global__ __launch_bounds__(256) void k_rows_grad_thin(GroupedProduct a) {
    typedef typename Mfma<T>::Frag Frag;
    union Piece {
        Pack<T> p;
        Frag f;
    };
    constexpr int JT = 4, BM = 16 * MT, BN = 16 * JT, kRow = BN * 2 + 16;   // LDS bytes of a row: 16 more, for the banks
    __shared__ __attribute__((aligned(16))) char lds[4 * 32 * kRow > 3 * MT * JT * 1024 ? 4 * 32 * kRow : 3 * MT * JT * 1024];
    const Tile tile = Deal<BM>(a, (a.k + BN - 1) / BN).get(a, a.first + blockIdx.x / kXcds);
    if (tile.none) return;
    Part<T, T> p;
    p.template rows<kRowsGrad, BM, BN>(a, tile);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, q = lane >> 4;
    char *mine = lds + wave * 32 * kRow;
    f32x4 acc[MT][JT] = {};
    const T *pa[MT];
#pragma unroll
    for (int m = 0; m < MT; m++) {
        const int r = m * 16 + l;
        pa[m] = p.a + (int64_t)(r < p.m_rows ? r : p.m_rows - 1) * p.lda;
    }
    Pack<T> w[4];
    Piece fa[MT];
    const auto fetch = [&](int i) {   // i .. i + 31 of the contraction; past its end 0
#pragma unroll
        for (int s = 0; s < 4; s++) {
            const int r = s * 8 + (lane >> 3), c = (lane & 7) * 8;
            w[s] = load_pack(p.b + (int64_t)(i + r) * p.ldb + c, i + r < p.depth ? p.j_rows - c : 0, (T)0.0f);
        }
#pragma unroll
        for (int m = 0; m < MT; m++) fa[m].p = load_pack(pa[m] + i + q * 8, p.depth - i - q * 8, (T)0.0f);
    };
    int i = wave * 32;
    if (i < p.depth) fetch(i);
    while (i < p.depth) {
        Piece f[MT];
#pragma unroll
        for (int m = 0; m < MT; m++) f[m] = fa[m];
#pragma unroll
        for (int s = 0; s < 4; s++)
            reinterpret_cast<Pack<T> *>(mine + (s * 8 + (lane >> 3)) * kRow)[lane & 7] = w[s];
        i += 128;
        if (i < p.depth) fetch(i);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < JT; j++) {
            union {
                Frag f;
                s16x4 half[2];
            } u;
#pragma unroll
            for (int s = 0; s < 2; s++)   // columns as in frag(): two fragments end as 8 consecutive ones
                u.half[s] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(
                    mine + (q * 8 + s * 4 + (l >> 2)) * kRow + ((j >> 1) * 32 + (l & 3) * 8 + (j & 1) * 4) * 2));
#pragma unroll
            for (int m = 0; m < MT; m++) acc[m][j] = Mfma<T>::go(u.f, f[m].f, acc[m][j]);
        }
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    f32x4 *join = reinterpret_cast<f32x4 *>(lds);
    if (wave)
#pragma unroll
        for (int t = 0; t < MT * JT; t++) join[((wave - 1) * MT * JT + t) * 64 + lane] = acc[t / JT][t % JT];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int m = 0; m < MT; m++) {
#pragma unroll
        for (int j = 0; j < JT; j++)
#pragma unroll
            for (int o = 0; o < 3; o++) acc[m][j] += join[(o * MT * JT + m * JT + j) * 64 + lane];
        const int r = m * 16 + l;
        if (r < p.m_rows) store_row<true>(p.c + r * a.ldo + q * 8, p.j_rows - q * 8, acc[m]);
    }
}

template <Direction D> bool feeds_big(const GroupedProduct &a) {
    const auto even = [](const void *p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 4 == 0 && ld % 2 == 0; };
    if (D == kForward) return even(a.x, a.ldx) && even(a.w, a.k);
    if (D == kRowsGrad) return even(a.dy, a.lddy) && even(a.w, a.k);
    return even(a.dy, a.lddy) && even(a.x, a.ldx);
}

template <int BM, int BN, Direction D> int64_t blocks_for(const GroupedProduct &a) {
    if (D == kWeights) return (int64_t)a.splits * a.groups * ((a.n + BM - 1) / BM) * ((a.k + BN - 1) / BN);
    const int cols = D == kForward ? a.n : a.k;
    const int64_t tiles = (a.rows / BM + a.groups + 2) * ((cols + BN - 1) / BN);
    return (tiles + kXcds - 1) / kXcds * kXcds;
}

// Launches a kernel that takes one tile a workgroup, on as many of the `blocks` tiles at a
// time as one launch holds.  a.first is where the launch begins: a tile of the weights'
// gradient, or a tile of each XCD's run.
template <Direction D, typename K> int launch_tiles(K *kernel, int64_t blocks, int threads, void *stream, GroupedProduct a) {
    const int64_t most = most_blocks(threads) / kXcds * kXcds;
    for (int64_t at = 0; at < blocks; at += most) {
        a.first = (uint32_t)(D == kWeights ? at : at / kXcds);
        if (const int e = launch(kernel, blocks - at < most ? blocks - at : most, threads, stream, a)) return e;
    }
    return 0;
}

// The sum of a.splits matrices of `count` elements, in order.
template <typename O> __global__ __launch_bounds__(256) void k_join(GroupedProduct a, int64_t count) {
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    const int64_t n = count - at;
    if (n <= 0) return;
    f32x4 sum = 0.0f;
    for (int p = 0; p < a.splits; p++) {
        const Pack<float> v = load_pack(a.partial + p * count + at, n, 0.0f);
#pragma unroll
        for (int j = 0; j < 4; j++) sum[j] += v.e[j];
    }
    O *out = static_cast<O *>(a.out) + at;
#pragma unroll
    for (int j = 0; j < 4; j++)
        if (j < n) out[j] = (O)sum[j];
}

// Whether the kernels for few rows a group are the faster ones, by what bounds each
// (microseconds; measured with 8 and 64 groups of 1024 x 4096, 4096 x 1024 and 1024 x
// 1024).  They read the weights of the groups that have rows, once for every 64 of
// these, at 3.6-4.6 (forward) and 5 TB/s (gradient, and 4 ns for each of its
// contraction): 12, 48 and 200 rows a group of 8 x 1024 x 4096 forward 18, 32 and 79,
// gradient 27, 32 and 43.  Big tiles take a time for each 64 of the contraction,
// whatever rows are in them, and use no more CUs than there are tiles: the same
// forward 24, 26 and 31 (128 tiles of 16 steps), gradient 73, 74 and 78 (32 tiles of 64
// steps).  Where rows are not 4-byte aligned a tile takes 2.2 times as long (16384 x
// 1023 -> 4095 in 8 groups 317 us), and these kernels read at 1.0 and 2.7 TB/s (176 rows
// a group of 32 x 1023 x 1365: 325 and 122 us).  Left out: the bytes of big tiles (1024
// groups of 256 x 64 -> 256 take 87 us, of which this counts 15) and uneven groups, whose
// average stands for all.
template <Direction D> bool few_rows(const GroupedProduct &a, bool big) {
    const double some = (double)a.rows / a.groups, live = a.groups * (1 - __builtin_exp(-some));
    const double reads = 2.0 * live * a.n * a.k * (some < 16 ? 1 : 0.75 + some / 64);
    const double rate = D == kForward ? (!big ? 1.0e6 : some < 16 ? 4.6e6 : 3.6e6) : big ? 5.0e6 : 2.7e6;
    const double thin = 4 + reads / rate + (D == kForward ? 0 : 1 + a.n * 0.004);
    const int cols = ((D == kForward ? a.n : a.k) + kBig - 1) / kBig, steps = ((D == kForward ? a.k : a.n) + 63) / 64;
    const double rounds = __builtin_ceil((some / kBig + 0.9) * a.groups * cols / kCus);
    return thin < (7 + rounds * steps * 1.05) * (big ? 1 : 2.2);
}

template <typename T, typename O, Direction D> int go(const GroupedProduct &a, void *stream) {
    const bool big = feeds_big<D>(a);
    if constexpr (D != kWeights) {
        if (few_rows<D>(a, big)) {
            const int64_t some = a.rows / a.groups;
            if constexpr (D == kForward) {
                if (some < 8) return launch_tiles<D>(k_product_thin<T, O, 1>, blocks_for<16, 32, D>(a), 256, stream, a);
                if (some < 16) return launch_tiles<D>(k_product_thin<T, O, 2>, blocks_for<32, 32, D>(a), 256, stream, a);
                return launch_tiles<D>(k_product_thin<T, O, 4>, blocks_for<64, 32, D>(a), 256, stream, a);
            } else {
                if (some < 8) return launch_tiles<D>(k_rows_grad_thin<T, 1>, blocks_for<16, 64, D>(a), 256, stream, a);
                if (some < 16) return launch_tiles<D>(k_rows_grad_thin<T, 2>, blocks_for<32, 64, D>(a), 256, stream, a);
                return launch_tiles<D>(k_rows_grad_thin<T, 4>, blocks_for<64, 64, D>(a), 256, stream, a);
            }
        }
    }
    if (!big) return launch_tiles<D>(k_product<T, O, D>, blocks_for<kTile, kTile, D>(a), 256, stream, a);
    int64_t blocks = blocks_for<kBig, kBig, D>(a);
    if (D != kWeights && blocks > kCus) blocks = kCus;   // one a CU: LDS holds no second
    return launch_tiles<D>(k_product_big<T, O, D>, blocks, 512, stream, a);
}

template <typename T> int weights(const GroupedProduct &a, void *stream) {
    const bool narrow = a.out_dtype != PASE_FP32;
    if (a.splits == 1) return narrow ? go<T, T, kWeights>(a, stream) : go<T, float, kWeights>(a, stream);
    GroupedProduct parts = a;
    parts.out = a.partial;
    if (const int e = go<T, float, kWeights>(parts, stream)) return e;
    const int64_t count = (int64_t)a.groups * a.n * a.k, blocks = (count + 1023) / 1024;
    return narrow ? launch(k_join<T>, blocks, 256, stream, a, count) : launch(k_join<float>, blocks, 256, stream, a, count);
}

template <typename T> int forward(const GroupedProduct &a, void *stream) {
    return a.out_dtype == PASE_FP32 ? go<T, float, kForward>(a, stream) : go<T, T, kForward>(a, stream);
}

}  // namespace

int launch_product_forward(const GroupedProduct &a, void *stream) {
    return a.dtype == PASE_BF16 ? forward<__bf16>(a, stream) : forward<_Float16>(a, stream);
}
int launch_product_rows_grad(const GroupedProduct &a, void *stream) {   // always in the operands' type
    return a.dtype == PASE_BF16 ? go<__bf16, __bf16, kRowsGrad>(a, stream) : go<_Float16, _Float16, kRowsGrad>(a, stream);
}
int launch_product_weights_grad(const GroupedProduct &a, void *stream) {
    return a.dtype == PASE_BF16 ? weights<__bf16>(a, stream) : weights<_Float16>(a, stream);
}

}  // namespace pase
