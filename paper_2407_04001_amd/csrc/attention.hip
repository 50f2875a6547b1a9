// Attention over ragged sequences and its gradients (pase_operators.h).
//
// Scores stand in the matrix instruction's result with the query (forward, dq) or the
// key (dk, dv) along the lanes: s^T = k q^T gives a lane one query and 16 of 32 keys, so
// maxima and sums over keys stay in a lane but for one exchange with lane ^ 32, a
// rescaling of the output is one factor a lane, and the weights are, rounded, the next
// product's operand as they stand: o^T += v^T p^T contracts over keys, in the order that
// the result registers hold them (keys 4 h + {0..3, 8..11} of 16 in half h of the wave),
// which the transposing LDS reads of v follow.  p never leaves the registers.
//
// Exponents are powers of two, p = 2^(c s - c m) with c = scale log2 e, one fused
// multiply-add each.
#include <type_traits>

#include "lds.h"
#include "operators.h"
#include "vectors.h"

namespace pase {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

template <typename T> struct Mfma;
template <> struct Mfma<__bf16> {
    typedef __bf16 Frag __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x16 go(Frag a, Frag b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Mfma<_Float16> {
    typedef _Float16 Frag __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x16 go(Frag a, Frag b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
};

// fp16's least numbers are 2^-24, which weights of many keys come near: before they are rounded they are 2^kRaised
// times their size, which the sum and the output share.  Forward they then reach 2^14 (see Softmax), and those below 2^-20 of
// the reference are off by up to 2^-31 of it instead of 2^-25; backward 2^12, and below 2^-26 by 2^-37.  The rest up to
// 2^16 is for exponents off by their own roundings.  It costs no instruction: the exponent's reference has it.
template <typename T> constexpr int kRaised = 0;
template <typename T> constexpr int kRaisedGrad = 0;
template <> constexpr int kRaised<_Float16> = 6;
template <> constexpr int kRaisedGrad<_Float16> = 12;

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Keeps a uniform branch a branch, where the compiler would make it selects on every path.
__device__ __forceinline__ void stay_apart() { asm volatile(""); }

// The lane's partner with the same query (or key): the other half of the wave.
__device__ __forceinline__ float other_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float other_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// ---------------------------------------------------------------- which rows a workgroup has
__device__ __forceinline__ int clamped(const void *p, int wide, int i, int lo, int hi) {
    const int64_t o = wide ? static_cast<const int64_t *>(p)[i] : (int64_t) static_cast<const int32_t *>(p)[i];
    return o < lo ? lo : o > hi ? hi : (int)o;
}

// Range v of sequences + 2: the rows before offsets[0], each sequence's, those from
// offsets[sequences] on.
struct Range {
    int lo, hi;
    __device__ __forceinline__ Range(const void *offsets, int wide, int sequences, int rows, int v) {
        lo = v == 0 ? 0 : clamped(offsets, wide, v - 1, 0, rows);
        hi = v > sequences ? rows : clamped(offsets, wide, v, lo, rows);
    }
};

__device__ __forceinline__ int wave_sum_of(int v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
    return uniform(v);
}

// The `item`-th tile, of `size` of a range's rows x group: its range and its place in it, -1 where there is none.
// Range v owns the tiles from start(v) * group / size + v up to its successor's, as many as it needs or
// one more, late ranges and places first (`late`: forward and dq, where these see the most keys) or early ones
// (dk and dv: the most queries see these); which range a tile is of follows by a search of 128 probes a round.
// a.by_place (early ones, up to 128 ranges, which stand in the lanes): tiles are dealt by the places left behind
// them, whatever the order of their sequences, so that the workgroups that start last have the
// least to do; it takes a few sums over the lanes, 2 us a workgroup.
// Offsets that break their rule give some range: whatever it is, rows stay within it.
struct Owner {
    int v, place;

    __device__ __forceinline__ Owner(const Attention &a, const void *offsets, int rows, int group, int size, int item, bool late) {
        const int lane = threadIdx.x & 63;
        const auto start = [&](int v) { return v == 0 ? 0 : v > a.sequences + 1 ? rows : clamped(offsets, a.offsets_64, v - 1, 0, rows); };
        if (!late && a.by_place) {
            const int s0 = start(lane), s1 = start(lane + 64), next = __shfl(s1, 0, 64);
            int e0 = __shfl_down(s0, 1, 64), e1 = __shfl_down(s1, 1, 64);
            e0 = lane == 63 ? next : e0, e1 = lane == 63 ? rows : e1;
            const int n0 = e0 > s0 ? ((e0 - s0) * group + size - 1) / size : 0, n1 = e1 > s1 ? ((e1 - s1) * group + size - 1) / size : 0;
            // tiles that are `r`-th or further of their range
            const auto count = [&](int r) { return wave_sum_of((n0 >= r ? n0 - r + 1 : 0) + (n1 >= r ? n1 - r + 1 : 0)); };
            v = 0, place = -1;
            if (item >= count(1)) return;
            int r = 1, most = n0 > n1 ? n0 : n1;
#pragma unroll
            for (int d = 32; d; d >>= 1) {
                const int o = __shfl_xor(most, d, 64);
                most = o > most ? o : most;
            }
            most = uniform(most);
            while (r < most) {   // the last r with more than `item` tiles
                const int mid = (r + most + 1) >> 1;
                if (count(mid) > item)
                    r = mid;
                else
                    most = mid - 1;
            }
            // of the ranges that have an r-th tile
            const int rank = item - count(r + 1);
            const uint64_t h0 = __ballot(n0 >= r), h1 = __ballot(n1 >= r);
            const int of0 = __builtin_popcountll(h0);
            const uint64_t has = rank < of0 ? h0 : h1;
            const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(has >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)has, 0));
            const uint64_t mine = __ballot((has >> lane & 1) && before == (rank < of0 ? rank : rank - of0));
            const int from = mine ? __builtin_ctzll(mine) : 0;
            v = uniform(from + (rank < of0 ? 0 : 64));
            place = uniform(__shfl(rank < of0 ? n0 : n1, from, 64)) - r;
            return;
        }
        const int tile = late ? a.tiles - 1 - item : item;
        const auto begin = [&](int v) { return start(v) * group / size + v; };
        // of ranges lo .. lo + n - 1, every step-th; the last round's are all of them
        for (int lo = 0, n = a.sequences + 2;;) {
            const int step = (n + 127) >> 7;
            int probe[2];
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const int at = (lane + 64 * k) * step;
                probe[k] = at < n ? begin(lo + at) : 0x7fffffff;
            }
            const uint64_t before = __ballot(probe[0] <= tile), behind = __ballot(probe[1] <= tile);
            int found = __builtin_popcountll(before) + __builtin_popcountll(behind);   // ranges begin in order
            found = found > 1 ? found - 1 : 0;
            const int value = uniform(__shfl(found < 64 ? probe[0] : probe[1], found & 63, 64));
            lo += found * step;
            if (step == 1) {
                v = uniform(lo), place = tile < value ? -1 : tile - value;
                return;
            }
            n = n - found * step < step ? n - found * step : step;
        }
    }
};

// What a tile of the queries sees, or a tile of the keys is seen by.
struct Sequence {
    int q_lo, q_rows, k_lo, k_rows, keys;   // keys: the first of k_rows that count
    __device__ __forceinline__ Sequence(const Attention &a, int v) {
        const Range q(a.q_offsets, a.offsets_64, a.sequences, a.rows, v), k(a.k_offsets, a.offsets_64, a.sequences, a.key_rows, v);
        q_lo = uniform(q.lo), q_rows = uniform(q.hi - q.lo), k_lo = uniform(k.lo), k_rows = uniform(k.hi - k.lo);
        keys = v < 1 || v > a.sequences ? 0 : k_rows;
        if (a.k_lengths && keys) keys = uniform(clamped(a.k_lengths, a.offsets_64, v - 1, 0, k_rows));
    }
    // How many of the keys query i sees.
    __device__ __forceinline__ int seen(const Attention &a, int i) const {
        if (!a.causal) return keys;
        const int n = i + keys - q_rows + 1;
        return n < 0 ? 0 : n > keys ? keys : n;
    }
};

// ---------------------------------------------------------------- tiles in LDS
// A row of D elements is D / 8 chunks of 16 bytes; chunk c of row r stands at place
// c ^ fold(r) of its row.  Sixteen rows' reads of one chunk, and the four rows x four
// chunks of a transposing read, then reach different banks.
template <int D> __device__ __forceinline__ int fold(int r) {
    if (D == 128) return (r & 3) << 2 | (r >> 2 & 3);
    if (D == 64) return (r >> 1 & 1) << 2 | (r >> 2 & 3);
    return r >> 2 & 3;
}

// Eight elements from `at` on of a row of n, 0 past its end.  The chunk that the end cuts is read whole from
// before it, where the row is that long, and shifted.
template <typename T> __device__ __forceinline__ Pack<T> load_chunk(const T *row, int at, int n) {
    const int have = n - at;
    if (have >= 8 || have <= 0 || n < 8) return load_pack(row + at, have, (T)0.0f);
    union {
        Pack<T> p;
        uint64_t u[2];
    } r;
    r.p = load_pack(row + n - 8, 8, (T)0.0f);
    const int bits = (8 - have) * 16;
    if (bits >= 64) {
        r.u[0] = r.u[1] >> (bits & 63), r.u[1] = 0;
    } else {
        r.u[0] = r.u[0] >> bits | r.u[1] << (64 - bits), r.u[1] >>= bits;
    }
    return r.p;
}

// How tiles are loaded: through registers, or from HBM to LDS without (rows 4-byte aligned, dim even; a buffer's
// range ends with the last row), where a chunk that dim cuts (no multiple of 8) then holds what
// follows the head in memory until trim(), which its loader calls once it has arrived.
enum Load { kThrough, kDirect, kCut };

// Loads ROWS rows of a head, D elements of each (0 past `dim` and past the rows that
// exist), by WAVES waves.
template <typename T, int D, int ROWS, int WAVES, Load LOAD> struct Feed {
    static constexpr bool DIRECT = LOAD != kThrough, CUT = LOAD == kCut;
    static constexpr int kChunks = D / 8, N = ROWS * kChunks / (64 * WAVES);
    static_assert(N >= 1 && ROWS * kChunks == N * 64 * WAVES, "whole loads");
    // A wave's load takes a kilobyte, kPeriod of which are 16 rows, after which the fold repeats: of a
    // wave's loads those 16 rows apart share one place.
    static constexpr int kPeriod = kChunks / 4, kPlaces = !DIRECT || WAVES >= kPeriod ? 1 : kPeriod / WAVES;
    int at[kPlaces];
    Pack<T> r[DIRECT ? 1 : N];
    int64_t ld;
    int dim, wave;

    __device__ __forceinline__ Feed(int64_t ld_, int dim_) : ld(ld_), dim(dim_) {
        wave = uniform(threadIdx.x >> 6) % WAVES;
        if (DIRECT)
#pragma unroll
            for (int n = 0; n < kPlaces; n++) {
                const int q = chunk(n), row = q / kChunks, c = q % kChunks ^ fold<D>(row);
                at[n] = c * 8 < dim ? row * (int)ld * 2 + c * 16 : 0x7fffff00;   // past every range
            }
    }
    __device__ __forceinline__ int block(int n) const {
        return kPlaces == 1 ? n * WAVES + wave : n / kPlaces * kPeriod + wave * kPlaces + n % kPlaces;
    }
    __device__ __forceinline__ int chunk(int n) const { return block(n) * 64 + (threadIdx.x & 63); }

    __device__ __forceinline__ void load(const T *p, int rows, const char *lds) {
        if (DIRECT) {
            rows = rows > ROWS ? ROWS : rows;
            const u32x4 range = buffer_of(p, rows > 0 ? ((rows - 1) * (int)ld + dim) * 2 : 0);
            const uint32_t dst = lds_address(lds);
#pragma unroll
            for (int n = 0; n < N; n++) {
                const uint32_t rows_on = kPlaces == 1 ? n * (64 * WAVES / kChunks) : n / kPlaces * 16;
                load_to_lds(range, (int)((uint32_t)at[n % kPlaces] + rows_on * 2 * (uint32_t)ld), dst + block(n) * 1024);
            }
        } else {
#pragma unroll
            for (int n = 0; n < N; n++) {
                const int q = chunk(n), row = q / kChunks, c = q % kChunks ^ fold<D>(row);
                r[n] = load_pack(p + row * ld + c * 8, row < rows ? dim - c * 8 : 0, (T)0.0f);
            }
        }
    }
    __device__ __forceinline__ void trim(char *lds) const {
        if (LOAD != kCut) return;
#pragma unroll
        for (int n = 0; n < N; n++) {
            const int q = chunk(n), c = q % kChunks ^ fold<D>(q / kChunks);
            if (c == dim / 8)
                for (int e = dim % 8; e < 8; e += 2) *reinterpret_cast<uint32_t *>(lds + q * 16 + e * 2) = 0;
        }
    }
    __device__ __forceinline__ void store(char *lds) {
        if (!DIRECT)
#pragma unroll
            for (int n = 0; n < N; n++) reinterpret_cast<Pack<T> *>(lds)[chunk(n)] = r[n];
    }
};

// The loads of a step of two tiles have arrived, but for the last LEFT of this wave's, and every wave is
// past its reads of the step before.
template <int LEFT, typename F> __device__ __forceinline__ void arrive(const F &a, const F &b, char *lds, int size) {
    if constexpr (F::DIRECT) {
        wait_loads<LEFT>();
        a.trim(lds), b.trim(lds + size);
        if (F::CUT) wait_loads<63>();   // LDS alone
        barrier();
    } else {
        __syncthreads();
    }
}

// Operand reads of a tile (at a multiple of 256 bytes).  Along: row r0 + lane % 32, elements
// 16 s + 8 h of it.  Across: column 32 d + lane % 32, rows 16 g + 4 h + {0..3, 8..11} of the 16.
// A fragment's place follows from the tile's by an exclusive or and a constant; begun anew for
// each tile, so that not all places of all tiles are kept in registers.
template <typename T, int D> struct Reader {
    typedef typename Mfma<T>::Frag Frag;
    uint32_t along, across;   // byte places within a tile

    __device__ __forceinline__ Reader() {
        const int lane = threadIdx.x & 63, h = lane >> 5, l = lane & 15;
        along = ((lane & 31) * (D / 8) + (h ^ fold<D>(lane & 31))) * 16;
        const int row = 4 * h + (l >> 2), c = (lane >> 4 & 1) * 2 + (l >> 1 & 1);
        across = (row * (D / 8) + (c ^ fold<D>(row))) * 16 + (l & 1) * 8;
    }
    static __device__ __forceinline__ uint32_t begin(uint32_t tile, uint32_t place) {
        uint32_t at = tile + place;
        asm volatile("" : "+v"(at));
        return at;
    }
    __device__ __forceinline__ uint32_t rows_of(uint32_t tile) const { return begin(tile, along); }
    __device__ __forceinline__ uint32_t columns_of(uint32_t tile) const { return begin(tile, across); }
    static __device__ __forceinline__ Frag row(uint32_t at, int r0, int s) {
        return *(__attribute__((address_space(3))) const Frag *)(uintptr_t)((at ^ s * 32) + r0 * D * 2);
    }
    static __device__ __forceinline__ Frag column(uint32_t at, int g, int d) {
        union {
            Frag f;
            s16x4 half[2];
        } u;
        u.half[0] = read_across((at ^ d * 64) + g * 16 * D * 2);
        u.half[1] = read_across((at ^ (d * 64 + 32)) + (g * 16 + 8) * D * 2);
        return u.f;
    }
};

// Operand registers of the lane's own row: 16 s + 8 h on, for the D / 16 s; 0 past the n that it has.
template <typename T, int D>
__device__ __forceinline__ void load_row(typename Mfma<T>::Frag (&f)[D / 16], const T *p, int n) {
    const int h = threadIdx.x >> 5 & 1;
    if (n == D) {
#pragma unroll
        for (int s = 0; s < D / 16; s++)
            f[s] = __builtin_bit_cast(typename Mfma<T>::Frag, reinterpret_cast<const Unaligned16<T> *>(p + 16 * s + 8 * h)->v);
        return;
    }
#pragma unroll
    for (int s = 0; s < D / 16; s++) f[s] = __builtin_bit_cast(typename Mfma<T>::Frag, load_chunk(p, 16 * s + 8 * h, n).v);
}

// Eight consecutive registers of a result as an operand.
template <typename T> __device__ __forceinline__ typename Mfma<T>::Frag narrow(const f32x16 &v, int from) {
    typename Mfma<T>::Frag f;
#pragma unroll
    for (int j = 0; j < 8; j++) f[j] = (T)v[from + j];
    return f;
}

// Stores a wave's 32 rows (lane % 32 its row, element 32 d + 8 i + 4 h + j in register 4 i + j
// of v[d]), times `factor`, or 0 where it has `none`, rounded once.  They pass LDS (32 D elements of the wave's own),
// so that whole rows are written 16 bytes a lane.  at(row): where a row goes, or null.
template <typename T, int D, typename F>
__device__ __forceinline__ void store_rows(char *lds, const f32x16 (&v)[D / 32], bool none, float factor, int dim, F at) {
    constexpr int kChunks = D / 8;
    const int lane = threadIdx.x & 63, h = lane >> 5, row = lane & 31;
#pragma unroll
    for (int d = 0; d < D / 32; d++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
            union {
                T e[4];
                uint64_t u;
            } o;
#pragma unroll
            for (int j = 0; j < 4; j++) o.e[j] = none ? (T)0.0f : (T)(v[d][4 * i + j] * factor);
            *reinterpret_cast<uint64_t *>(lds + (row * kChunks + ((d * 4 + i) ^ fold<D>(row))) * 16 + h * 8) = o.u;
        }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int n = 0; n < 32 * kChunks / 64; n++) {
        const int q = n * 64 + lane, r = q / kChunks, c = q % kChunks;
        const Pack<T> o = reinterpret_cast<const Pack<T> *>(lds)[r * kChunks + (c ^ fold<D>(r))];
        T *p = at(r);
        if (p && c * 8 < dim) store_pack(p + c * 8, dim - c * 8, o);
    }
}

template <typename T> __device__ __forceinline__ const T *head_of(const HeadRows &x, int64_t row, int64_t head) {
    return static_cast<const T *>(x.p) + row * x.ld + head * x.head_ld;
}
template <typename T> __device__ __forceinline__ T *out_of(const HeadRows &x, int64_t row, int64_t head) {
    return static_cast<T *>(x.p) + row * x.ld + head * x.head_ld;
}

// The queries of a tile: a range's rows x the heads that share one of keys and values,
// the heads of a row next to each other, so that these heads share the keys' tiles and
// single tokens fill more of a tile.
struct Queries {
    int group, head0, rows, first;   // rows x group there are; the tile's first

    __device__ __forceinline__ bool has(int p) const { return first + p < rows; }
    __device__ __forceinline__ int index(int p) const { return (first + p) / group; }
    __device__ __forceinline__ int head(int p) const { return head0 + (first + p) % group; }
};

// Rows and heads of one share's log-sum-exps in a.partial, which its outputs follow.
__device__ __forceinline__ int64_t part_rows(const Attention &a) { return ((int64_t)a.rows * a.heads + 3) & ~3ll; }

// ---------------------------------------------------------------- forward
// The softmax of one query a lane, so far: the output as the sum of 2^(c (s - m)) v and the
// weights' sum over this lane's half of the keys, both times 2^kRaised.
template <typename T, int D, int KT> struct Softmax {
    typedef typename Mfma<T>::Frag Frag;
    f32x16 o[D / 32] = {};
    float m = -__builtin_inff(), sum = 0;

    // KT more keys: kt and vt are their places (along, across), the lane's query q sees `seen` of
    // them where `some` query of the wave does not see all.  between(): called once the keys are
    // read; before(): before the values are.
    template <typename F, typename G>
    __device__ __forceinline__ void step(uint32_t kt, uint32_t vt, const Frag (&q)[D / 16], int seen, bool some, float c, F between,
                                         G before) {
        f32x16 s[KT / 32];
#pragma unroll
        for (int b = 0; b < KT / 32; b++) {
            s[b] = 0.0f;
#pragma unroll
            for (int d = 0; d < D / 16; d++) s[b] = Mfma<T>::go(Reader<T, D>::row(kt, b * 32, d), q[d], s[b]);
        }
        between();
        if (some) {
            stay_apart();
            seen -= (threadIdx.x >> 5 & 1) * 4;
#pragma unroll
            for (int b = 0; b < KT / 32; b++)
#pragma unroll
                for (int j = 0; j < 16; j++)
                    if (b * 32 + 8 * (j / 4) + j % 4 >= seen) s[b][j] = -__builtin_inff();
        }
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < KT / 32; b++)
#pragma unroll
            for (int j = 0; j < 16; j++) top = fmaxf(top, s[b][j]);
        top = other_max(top);
        // The exponents' reference moves only when it is over 8 too low: weights stay below 2^8,
        // well within either type, and the output is seldom rescaled.
        if (__any((top - m) * c > 8)) {
            const float now = fmaxf(m, top), f = now == m ? 1.0f : __builtin_amdgcn_exp2f((m - now) * c);
            m = now;
            sum *= f;
#pragma unroll
            for (int d = 0; d < D / 32; d++) o[d] *= f;
        }
        const float from = m == -__builtin_inff() ? 0.0f : m * c - kRaised<T>;
        float more = 0;   // a step's sum by itself: small weights, one by one, would vanish behind a large one before them
#pragma unroll
        for (int b = 0; b < KT / 32; b++)
#pragma unroll
            for (int j = 0; j < 16; j++) {
                s[b][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][j], c, -from));
                more += s[b][j];
            }
        sum += more;
        before();
        // weights are rounded to the values' type: by up to 2^-8 (bf16) or 2^-11 of each (see kRaised), either way
#pragma unroll
        for (int g = 0; g < KT / 16; g++) {
            const Frag p = narrow<T>(s[g / 2], g % 2 * 8);
#pragma unroll
            for (int d = 0; d < D / 32; d++) o[d] = Mfma<T>::go(Reader<T, D>::column(vt, g, d), p, o[d]);
        }
    }
    // of both halves' sum: a weight of 2^kRaised or more, or nothing was seen
    __device__ __forceinline__ float lse(float all, float c) const {
        return all == 0 ? -__builtin_inff() : (m * c + (__builtin_amdgcn_logf(all) - kRaised<T>)) * kLn2;
    }
};

// 128 queries a workgroup, 64 keys a step, keys and values two steps deep in LDS: 32 queries
// a wave, whose operand and output stay in registers, at two (128 columns) or four waves a SIMD, so that one
// multiplies while another takes its exponents.  Per score 4 D operations of the matrix
// units and, in a lane, a maximum, a multiply-add, an exponential (a quarter of their rate), an addition and
// half a conversion: at 128 columns both take about as long, at 64 the lanes twice.  Long causal sequences
// (16384 rows in 4, 16 heads of 128 to 4) 324 us, 923 TFLOP/s (an 8192^3 library product 1170-1245); 4 x 4096, 16 heads
// of 64, 861 TFLOP/s without the causal limit.  64 x 256 rows, 16 heads of 64: 46 us for 134 MB, waiting for loads
// 43 % of a wave's time, as a workgroup has four steps only (heads of 63, through registers: 88).  Three steps in LDS (and so three
// workgroups a CU) were slower there, 49.6 us against 44.7.
template <typename T, int D, Load LOAD>
__global__ __launch_bounds__(256, D == 128 ? 2 : LOAD == kDirect ? 4 : 3) void k_forward(Attention a) {
    typedef typename Mfma<T>::Frag Frag;
    constexpr int WAVES = 4, BM = 128, KT = 64, kTile = KT * D * 2;
    __shared__ __attribute__((aligned(1024))) char lds[2][2 * kTile];
    static_assert(2 * 2 * kTile >= BM * D * 2, "the output passes the same LDS");
    const uint32_t item = a.first + blockIdx.x;
    // heads next to each other, so that an XCD's workgroups share as few as may be
    const int kv_head = (int)(item % a.kv_heads);
    const int group = a.heads / a.kv_heads;
    const Owner own(a, a.q_offsets, a.rows, group, BM, (int)(item / a.kv_heads), true);
    if (own.place < 0) return;
    const Sequence sq(a, own.v);
    const Queries qs{group, kv_head * group, sq.q_rows * group, own.place * BM};
    if (!qs.has(0)) return;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), h = lane >> 5, mine = wave * 32 + (lane & 31);
    const bool there = qs.has(mine);
    const int i = qs.index(mine), head = qs.head(mine);
    Frag q[D / 16];
    load_row<T, D>(q, head_of<T>(a.q, there ? sq.q_lo + i : 0, there ? head : 0), a.dim);   // (a lane without a query: any row)

    // keys that the wave's first and last query, and the tile's last, see
    const int last = qs.rows - 1 - qs.first < BM - 1 ? qs.rows - 1 - qs.first : BM - 1;
    const int w_last = wave * 32 + 31 < last ? wave * 32 + 31 : last;
    const bool busy = wave * 32 <= last;
    const int seen = sq.seen(a, i);
    const int all_see = busy ? uniform(sq.seen(a, qs.index(wave * 32))) : 0;
    const int any_sees = busy ? uniform(sq.seen(a, qs.index(w_last))) : 0;
    const int end = uniform(sq.seen(a, qs.index(last)));
    const int tiles = (end + KT - 1) / KT;

    const float c = a.scale * kLog2e;
    Softmax<T, D, KT> softmax;
    Feed<T, D, KT, WAVES, LOAD> fk(a.k.ld, a.dim), fv(a.v.ld, a.dim);
    const Reader<T, D> read;
    const T *k = head_of<T>(a.k, sq.k_lo, kv_head), *v = head_of<T>(a.v, sq.k_lo, kv_head);
    const auto load = [&](int t, char *to) {
        fk.load(k + (int64_t)t * KT * a.k.ld, sq.keys - t * KT, to);
        fv.load(v + (int64_t)t * KT * a.v.ld, sq.keys - t * KT, to + kTile);
    };
    const auto store = [&](char *to) { fk.store(to), fv.store(to + kTile); };
    if (tiles) load(0, lds[0]), store(lds[0]);
    for (int t = 0; t < tiles; t++) {
        const int at = t & 1;
        arrive<0>(fk, fv, lds[at], kTile);
        if (t + 1 < tiles) load(t + 1, lds[at ^ 1]);
        if (t * KT < any_sees) {
            const uint32_t tile = lds_address(lds[at]), kt = read.rows_of(tile), vt = read.columns_of(tile + kTile);
            softmax.step(kt, vt, q, seen - t * KT, (t + 1) * KT > all_see, c, [] {}, [] {});
        }
        if (t + 1 < tiles) store(lds[at ^ 1]);
    }
    const float sum = other_sum(softmax.sum), lse = softmax.lse(sum, c);
    if (there && h == 0) a.lse[(int64_t)head * a.rows + sq.q_lo + i] = lse;
    __syncthreads();
    store_rows<T, D>(lds[0] + wave * 32 * D * 2, softmax.o, sum == 0, 1.0f / sum, a.dim, [&](int r) -> T * {
        const int p = wave * 32 + r;
        return qs.has(p) ? out_of<T>(a.out, sq.q_lo + qs.index(p), qs.head(p)) : nullptr;
    });
}

// Few queries: 32 a workgroup, of one sequence.  Its four waves take every fourth step of 32
// keys each, with no barrier between them, from LDS of their own: the next step's keys are
// loaded where this one's were once they are read, values likewise, so that a wave always
// has loads on their way and LDS holds two workgroups (two steps deep and one workgroup a
// CU: 80 us against 62 for 64 tokens over 131072 keys, 4 heads of 128).  The waves' outputs are
// joined at the end; where tiles are still too few, a.splits workgroups share a tile's keys
// and leave their outputs and log-sum-exps for k_join.
// Bound by HBM: those 64 tokens 58 us for 269 MB (4.6 TB/s), and 4 us for the join; one token
// over 131072 keys, 2 heads, 30 us for 134 MB and 6.
template <typename T, int D, Load LOAD> __global__ __launch_bounds__(256, 2) void k_forward_few(Attention a) {
    constexpr bool DIRECT = LOAD != kThrough;
    typedef typename Mfma<T>::Frag Frag;
    constexpr int WAVES = 4, BM = 32, KT = 32, kTile = KT * D * 2;
    constexpr int kSums = (BM + 1) * D * 4, kOut = kSums + BM * 8;   // a wave's output; its references and sums
    constexpr int kLds = ((2 * kTile > kOut ? 2 * kTile : kOut) + 255) & ~255;
    __shared__ __attribute__((aligned(1024))) char lds[WAVES][kLds];
    const uint32_t block = a.first + blockIdx.x, item = block / a.splits;
    const int part = (int)(block - item * a.splits);
    const int kv_head = (int)(item % a.kv_heads), group = a.heads / a.kv_heads;
    const Owner own(a, a.q_offsets, a.rows, group, BM, (int)(item / a.kv_heads), true);
    if (own.place < 0) return;
    const Sequence sq(a, own.v);
    const Queries qs{group, kv_head * group, sq.q_rows * group, own.place * BM};
    if (!qs.has(0)) return;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), h = lane >> 5, mine = lane & 31;
    const bool there = qs.has(mine);
    const int i = qs.index(mine), head = qs.head(mine);
    const int last = qs.rows - 1 - qs.first < BM - 1 ? qs.rows - 1 - qs.first : BM - 1;
    const int seen = sq.seen(a, i), all_see = uniform(sq.seen(a, qs.index(0)));
    const int64_t tiles = (uniform(sq.seen(a, qs.index(last))) + KT - 1) / KT;
    const int t0 = (int)(tiles * part / a.splits) + wave, t1 = (int)(tiles * (part + 1) / a.splits);

    const float c = a.scale * kLog2e;
    Feed<T, D, KT, 1, LOAD> fk(a.k.ld, a.dim), fv(a.v.ld, a.dim);
    const T *k = head_of<T>(a.k, sq.k_lo, kv_head), *v = head_of<T>(a.v, sq.k_lo, kv_head);
    char *const kt = lds[wave], *const vt = kt + kTile;
    const auto load_keys = [&](int t) {
        if (t < t1) fk.load(k + (int64_t)t * KT * a.k.ld, sq.keys - t * KT, kt), fk.store(kt);
    };
    const auto load_values = [&](int t) {
        if (t < t1) fv.load(v + (int64_t)t * KT * a.v.ld, sq.keys - t * KT, vt), fv.store(vt);
    };
    // this wave's loads up to the last N, and its LDS reads and writes, are done
    const auto done = [](auto n) {
        if (DIRECT)
            wait_loads<decltype(n)::value>();
        else
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_sched_barrier(0);
    };
    using None = std::integral_constant<int, 0>;
    using Other = std::integral_constant<int, decltype(fk)::N>;
    using All = std::integral_constant<int, 63>;   // LDS alone
    load_keys(t0), load_values(t0);
    Frag q[D / 16];
    load_row<T, D>(q, head_of<T>(a.q, there ? sq.q_lo + i : 0, there ? head : 0), a.dim);   // (a lane without a query: any row)
    Softmax<T, D, KT> softmax;
    const Reader<T, D> read;
    for (int t = t0; t < t1; t += WAVES) {
        done(Other{});
        fk.trim(kt);
        softmax.step(
            read.rows_of(lds_address(kt)), read.columns_of(lds_address(vt)), q, seen - t * KT, (t + 1) * KT > all_see, c,
            [&] { done(All{}), load_keys(t + WAVES); },
            [&] {
                if (t + WAVES < t1)
                    done(Other{});
                else
                    done(None{});
            });
        done(All{}), load_values(t + WAVES);
    }
    // A wave's output in quads of columns, a quad's 32 rows adjacent and one place left, so that neither the
    // lanes of a row nor those of a quad meet in a bank.
    const float sum = other_sum(softmax.sum);
    {
        f32x4 *out = reinterpret_cast<f32x4 *>(lds[wave]);
#pragma unroll
        for (int d = 0; d < D / 32; d++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                f32x4 x;
#pragma unroll
                for (int j = 0; j < 4; j++) x[j] = softmax.o[d][4 * e + j];
                out[(d * 8 + e * 2 + h) * (BM + 1) + mine] = x;
            }
        if (h == 0) reinterpret_cast<float2 *>(lds[wave] + kSums)[mine] = {softmax.m, sum};
    }
    __syncthreads();
    const int r = threadIdx.x >> 3;   // eight lanes a row
    if (!qs.has(r)) return;
    float m[WAVES], w[WAVES], all = 0, top = -__builtin_inff();
#pragma unroll
    for (int n = 0; n < WAVES; n++) {
        const float2 of = reinterpret_cast<const float2 *>(lds[n] + kSums)[r];
        m[n] = of.x, w[n] = of.y, top = fmaxf(top, of.x);
    }
#pragma unroll
    for (int n = 0; n < WAVES; n++) {
        const float f = w[n] == 0 ? 0.0f : __builtin_amdgcn_exp2f((m[n] - top) * c);
        all += w[n] * f, w[n] = f;
    }
    const float inverse = 1.0f / all;
    const int64_t row = sq.q_lo + qs.index(r), of = qs.head(r), at = row * a.heads + of;
    if ((threadIdx.x & 7) == 0) {
        const float lse = all == 0 ? -__builtin_inff() : (top * c + (__builtin_amdgcn_logf(all) - kRaised<T>)) * kLn2;
        if (a.splits > 1)
            a.partial[part * part_rows(a) + at] = lse;
        else
            a.lse[of * a.rows + row] = lse;
    }
    if (a.splits > 1 && all == 0) return;   // not read
    const int width = (a.dim + 3) & ~3;
    float *parts = a.partial + a.splits * part_rows(a) + (part * part_rows(a) + at) * width;
    T *out = out_of<T>(a.out, row, of);
#pragma unroll
    for (int n = 0; n < D / 32; n++) {
        const int quad = (threadIdx.x & 7) + n * 8;
        f32x4 x = 0.0f;
#pragma unroll
        for (int k = 0; k < WAVES; k++) {
            const f32x4 y = reinterpret_cast<const f32x4 *>(lds[k])[quad * (BM + 1) + r];
            if (w[k] != 0) x += y * w[k];   // (what a wave that saw nothing left may be NaN)
        }
        x *= inverse;
        if (quad * 4 >= width) break;
        if (a.splits > 1) {
            *reinterpret_cast<f32x4 *>(parts + quad * 4) = x;
        } else {
#pragma unroll
            for (int j = 0; j < 4; j++)
                if (quad * 4 + j < a.dim) out[quad * 4 + j] = all == 0 ? (T)0.0f : (T)x[j];
        }
    }
}

// Joins up to kFewShares shares: eight rows and heads a workgroup, 32 lanes each (1024 rows and heads 4 us, 8 by k_join).
constexpr int kFewShares = 8;

template <typename T> __global__ __launch_bounds__(256) void k_join_few(Attention a) {
    const int64_t at = ((int64_t)a.first + blockIdx.x) * 8 + threadIdx.x / 32, all = part_rows(a);
    const int column = (threadIdx.x & 31) * 4, width = (a.dim + 3) & ~3;
    if (at >= (int64_t)a.rows * a.heads || column >= width) return;
    const float *parts = a.partial + a.splits * all + at * width + column;
    float w[kFewShares], top = -__builtin_inff(), total = 0;
    f32x4 sum = 0.0f;
#pragma unroll
    for (int p = 0; p < kFewShares; p++) {
        w[p] = p < a.splits ? a.partial[p * all + at] : -__builtin_inff();
        top = fmaxf(top, w[p]);
    }
#pragma unroll
    for (int p = 0; p < kFewShares; p++) {
        w[p] = w[p] == -__builtin_inff() ? 0.0f : __expf(w[p] - top);
        total += w[p];
        if (w[p] != 0) sum += w[p] * *reinterpret_cast<const f32x4 *>(parts + p * all * width);   // else it was not written
    }
    const int64_t row = at / a.heads, head = at % a.heads;
    const bool none = total == 0;
    T *out = out_of<T>(a.out, row, head) + column;
#pragma unroll
    for (int j = 0; j < 4; j++)
        if (column + j < a.dim) out[j] = none ? (T)0.0f : (T)(sum[j] / total);
    if (column == 0) a.lse[head * a.rows + row] = none ? -__builtin_inff() : top + logf(total);
}

// Joins the shares of 32 columns of one row and head: weights exp(lse_p - lse).  Eight
// lanes take a share, 32 shares at a time.
template <typename T> __global__ __launch_bounds__(256) void k_join(Attention a) {
    __shared__ float lds[2][4], weight[kMaxShares];
    __shared__ f32x4 sums[4][8];
    const int groups = (a.dim + 31) / 32, width = (a.dim + 3) & ~3;
    const int64_t block = (int64_t)a.first + blockIdx.x, at = block / groups, all = part_rows(a);
    const int column = (int)(block - at * groups) * 32 + (threadIdx.x & 7) * 4;
    const float lse = (int)threadIdx.x < a.splits ? a.partial[threadIdx.x * all + at] : -__builtin_inff();
    const float top = group_max<4>(lse, lds[0]);
    float total[1] = {lse == -__builtin_inff() ? 0.0f : __expf(lse - top)};
    weight[threadIdx.x] = total[0];
    group_sum<4>(total, lds[1]);
    f32x4 sum = 0.0f;
    const float *parts = a.partial + a.splits * all + at * width + column;
#pragma unroll
    for (int n = 0; n < kMaxShares / 32; n++) {
        const int p = n * 32 + threadIdx.x / 8;
        // a share without weight was not written
        if (p < a.splits && column < width && weight[p] != 0) sum += weight[p] * *reinterpret_cast<const f32x4 *>(parts + p * all * width);
    }
#pragma unroll
    for (int d = 8; d < 64; d <<= 1)
#pragma unroll
        for (int j = 0; j < 4; j++) sum[j] += __shfl_xor(sum[j], d, 64);
    if ((threadIdx.x & 63) < 8) sums[threadIdx.x >> 6][threadIdx.x & 7] = sum;
    __syncthreads();
    if (threadIdx.x >= 8) return;
    sum = sums[0][threadIdx.x] + sums[1][threadIdx.x] + sums[2][threadIdx.x] + sums[3][threadIdx.x];
    const int64_t row = at / a.heads, head = at % a.heads;
    const bool none = total[0] == 0;
    T *out = out_of<T>(a.out, row, head) + column;
#pragma unroll
    for (int j = 0; j < 4; j++)
        if (column + j < a.dim) out[j] = none ? (T)0.0f : (T)(sum[j] / total[0]);
    if (column == 0) a.lse[head * a.rows + row] = none ? -__builtin_inff() : top + logf(total[0]);
}

// ---------------------------------------------------------------- backward
// p = exp(s - lse), ds = p (dp - delta) with dp = v . dout and delta = out . dout.  Two
// kernels, each with its own outputs in registers: dq over the keys, which also leaves
// the rows' exponents and deltas, and dk and dv over the queries.  Scores and dp are formed in both (seven
// products where one kernel with atomics would take five): sums have a fixed order.
// p and ds are rounded to the operands' type before their second products: by up to 2^-8
// (bf16) or 2^-11 of each, either way, as the results are once more.  In fp16 p is raised first (kRaisedGrad), as no scale
// of the loss reaches it; ds is not, as one does.

__device__ __forceinline__ float exponent_of(float lse) {   // rows without keys: p = 0
    return lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2e;
}

template <typename T> constexpr float kLower = 1.0f / (1 << kRaisedGrad<T>);

// The sum of a result over teams of `waves` waves: every team but `to` gives its own, in LDS, which `to`
// then adds to its own in the teams' order.  A part is 128 D bytes for each wave.
template <int D> struct Join {
    char *lds;
    int team, wave, waves;

    __device__ __forceinline__ f32x4 &at(int part, int quad) const {
        return *reinterpret_cast<f32x4 *>(lds + ((part * waves * D / 8 + quad * waves + wave) * 64 + (threadIdx.x & 63)) * 16);
    }
    __device__ __forceinline__ void give(const f32x16 (&x)[D / 32], int to) const {
        if (team == to) return;
#pragma unroll
        for (int d = 0; d < D / 32; d++)
#pragma unroll
            for (int e = 0; e < 4; e++)
                at(team - (team > to), d * 4 + e) = f32x4{x[d][4 * e], x[d][4 * e + 1], x[d][4 * e + 2], x[d][4 * e + 3]};
    }
    __device__ __forceinline__ void take(f32x16 (&x)[D / 32], int to, int teams) const {
        if (team != to) return;
#pragma unroll 1
        for (int part = 0; part < teams - 1; part++)
#pragma unroll
            for (int d = 0; d < D / 32; d++)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const f32x4 o = at(part, d * 4 + e);
#pragma unroll
                    for (int j = 0; j < 4; j++) x[d][4 * e + j] += o[j];
                }
    }
};

// Queries along the lanes, as in the forward pass: 128 a workgroup, 64 keys a step.  Long causal sequences (16384
// rows in 4, 16 heads of 128 to 4) 443 us for 448 GFLOP (1 PFLOP/s), the median of 66 passes; 64 x 256 rows, 16 heads of 64 60 us
// for 201 MB, waiting for loads 63 % of a wave's time (three steps in LDS, or four waves a SIMD, changed
// nothing or lost 2 us).
template <typename T, int D, Load LOAD> __global__ __launch_bounds__(256, 2) void k_queries_grad(Attention a) {
    typedef typename Mfma<T>::Frag Frag;
    constexpr int WAVES = 4, BM = 128, KT = D == 128 && LOAD == kThrough ? 32 : 64, kTile = KT * D * 2, kStep = 2 * kTile;
    static_assert(2 * kStep >= BM * D * 2, "the gradient passes the same LDS");
    __shared__ __attribute__((aligned(1024))) char lds[2 * kStep];
    const uint32_t item = a.first + blockIdx.x;
    const int kv_head = (int)(item % a.kv_heads);
    const int group = a.heads / a.kv_heads;
    const Owner own(a, a.q_offsets, a.rows, group, BM, (int)(item / a.kv_heads), true);
    if (own.place < 0) return;
    const Sequence sq(a, own.v);
    const Queries qs{group, kv_head * group, sq.q_rows * group, own.place * BM};
    if (!qs.has(0)) return;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), h = lane >> 5, mine = wave * 32 + (lane & 31);
    const bool there = qs.has(mine);
    const int i = qs.index(mine), head = there ? qs.head(mine) : 0, row = there ? sq.q_lo + i : 0;   // (a lane without a query: any row)
    const int last = qs.rows - 1 - qs.first < BM - 1 ? qs.rows - 1 - qs.first : BM - 1;
    const int w_last = wave * 32 + 31 < last ? wave * 32 + 31 : last;
    const bool busy = wave * 32 <= last;
    const int seen = sq.seen(a, i);
    const int all_see = busy ? uniform(sq.seen(a, qs.index(wave * 32))) : 0;
    const int any_sees = busy ? uniform(sq.seen(a, qs.index(w_last))) : 0;
    const int steps = (uniform(sq.seen(a, qs.index(last))) + KT - 1) / KT;

    const float c = a.scale * kLog2e;
    f32x16 dq[D / 32] = {};
    Feed<T, D, KT, WAVES, LOAD> fk(a.k.ld, a.dim), fv(a.v.ld, a.dim);
    const Reader<T, D> read;
    const T *k = head_of<T>(a.k, sq.k_lo, kv_head), *v = head_of<T>(a.v, sq.k_lo, kv_head);
    const auto step_at = [&](int n) { return lds + (n & 1) * kStep; };
    const auto load = [&](int t) {
        char *to = step_at(t);
        fk.load(k + (int64_t)t * KT * a.k.ld, sq.keys - t * KT, to);
        fv.load(v + (int64_t)t * KT * a.v.ld, sq.keys - t * KT, to + kTile);
    };
    const auto store = [&](int t) { fk.store(step_at(t)), fv.store(step_at(t) + kTile); };
    if (steps) load(0);   // before the rows' own loads are waited for
    Frag q[D / 16], g[D / 16];
    load_row<T, D>(q, head_of<T>(a.q, row, head), a.dim);
    load_row<T, D>(g, head_of<T>(a.dout, row, head), a.dim);
    float delta = 0, lse2 = __builtin_inff();
    {
        Frag out[D / 16];
        load_row<T, D>(out, head_of<T>(a.out, row, head), a.dim);
#pragma unroll
        for (int d = 0; d < D / 16; d++)
#pragma unroll
            for (int j = 0; j < 8; j++) delta += (float)g[d][j] * (float)out[d][j];
        delta = other_sum(delta);
        if (there) {
            const int64_t at = (int64_t)head * a.rows + row;
            lse2 = exponent_of(a.lse[at]);
            if (h == 0) a.stats[at] = {lse2 - kRaisedGrad<T>, delta * kLower<T>};
        }
    }
    if (steps) store(0);
    for (int t = 0; t < steps; t++) {
        arrive<0>(fk, fv, step_at(t), kTile);
        if (t + 1 < steps) load(t + 1);
        if (t * KT < any_sees) {
            const uint32_t tile = lds_address(step_at(t)), kt = read.rows_of(tile), vt = read.rows_of(tile + kTile), kc = read.columns_of(tile);
            const bool whole = (t + 1) * KT <= all_see;
#pragma unroll
            for (int b = 0; b < KT / 32; b++) {
                f32x16 s = 0.0f, dp = 0.0f;
#pragma unroll
                for (int d = 0; d < D / 16; d++) {
                    s = Mfma<T>::go(read.row(kt, b * 32, d), q[d], s);
                    dp = Mfma<T>::go(read.row(vt, b * 32, d), g[d], dp);
                }
#pragma unroll
                for (int j = 0; j < 16; j++) s[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j], c, -lse2)) * (dp[j] - delta);
                if (!whole) {
                    stay_apart();
#pragma unroll
                    for (int j = 0; j < 16; j++)
                        if (8 * (j / 4) + j % 4 >= seen - t * KT - b * 32 - 4 * h) s[j] = 0.0f;
                }
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const Frag ds = narrow<T>(s, e * 8);
#pragma unroll
                    for (int d = 0; d < D / 32; d++) dq[d] = Mfma<T>::go(read.column(kc, b * 2 + e, d), ds, dq[d]);
                }
            }
        }
        if (t + 1 < steps) store(t + 1);
    }
    __syncthreads();
    store_rows<T, D>(lds + wave * 32 * D * 2, dq, lse2 == __builtin_inff(), a.scale, a.dim, [&](int r) -> T * {
        const int p = wave * 32 + r;
        return qs.has(p) ? out_of<T>(a.dq, sq.q_lo + qs.index(p), qs.head(p)) : nullptr;
    });
}

// Keys along the lanes: s = q k^T and dp = dout v^T give a lane one key and 16 of 32
// queries; dv^T += dout^T p and dk^T += q^T ds.  TEAMS teams of waves have the same
// WAVES x 32 keys: the steps through the queries of all heads that share them, QT at a
// time, go round the teams, whose sums are added at the end.
// Loads to LDS: three steps in LDS, two on their way (128 columns: two and one); through registers: one, loaded
// where it is needed.  With 128 columns the accumulators take 128 of a lane's 256 registers at two waves a SIMD; at
// one wave a SIMD and 512 the compiler moved them to and from the second half in every step (2162 us for the whole
// backward pass of 16384 rows in 4 causal sequences, 16 heads of 128 to 4, against 1647).  There 702 us for 598
// GFLOP (852 TFLOP/s), the median of 66 passes; 64 x 256 rows, 16 heads of 64 60 us.
// Through registers nothing is on its way while a step is multiplied: 64 x 256 rows, 16 heads of 63 116 us, 6508 rows
// in 2 sequences, 2 heads of 35, 319 (of 36, in four teams: 71).
template <typename T, int D, int QT, int WAVES, int TEAMS, Load LOAD>
__global__ __launch_bounds__(TEAMS * WAVES * 64, TEAMS > 1 ? 1 : D == 128 ? 2 : 3) void k_keys_grad(Attention a) {
    constexpr bool DIRECT = LOAD != kThrough;
    typedef typename Mfma<T>::Frag Frag;
    constexpr int BM = WAVES * 32, kTile = QT * D * 2, kStats = QT * 8, kStep = 2 * kTile + kStats;
    constexpr int kSteps = !DIRECT ? 1 : D == 128 ? 2 : 3;
    constexpr int kPart = BM * D * 4, kJoin = TEAMS > 2 ? (TEAMS - 1) * kPart : kPart;   // (both gradients pass as many bytes on their way out)
    // The accumulators of 128 columns leave no registers for both operands of a wave's keys:
    // the values stay in LDS.
    constexpr bool kValuesInLds = D == 128;
    constexpr int kValues = kValuesInLds ? BM * D * 2 : 0;
    constexpr int kLds = kValues + TEAMS * kSteps * kStep > kJoin ? kValues + TEAMS * kSteps * kStep : kJoin;
    __shared__ __attribute__((aligned(1024))) char lds[kLds];
    const uint32_t item = a.first + blockIdx.x;
    const int kv_head = (int)(item % a.kv_heads);
    const int group = a.heads / a.kv_heads;
    const Owner own(a, a.k_offsets, a.key_rows, 1, BM, (int)(item / a.kv_heads), false);
    if (own.place < 0) return;
    const Sequence sq(a, own.v);
    const int first = own.place * BM;
    if (first >= sq.k_rows) return;
    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int team = TEAMS == 1 ? 0 : uniform(threadIdx.x >> 6) / WAVES, wave = uniform(threadIdx.x >> 6) % WAVES;
    const int key0 = first + wave * 32, key = key0 + (lane & 31);
    const bool there = key < sq.keys;
    const int64_t row = sq.k_lo + (there ? key : 0);
    Frag k[D / 16], v[kValuesInLds ? 1 : D / 16];
    load_row<T, D>(k, head_of<T>(a.k, row, kv_head), a.dim);   // (a lane without a key: any row)
    f32x16 dk[D / 32] = {}, dv[D / 32] = {};

    const float c = a.scale * kLog2e;
    const int shift = a.causal ? sq.keys - sq.q_rows : 1 << 30;   // query i sees keys up to i + shift
    const int from = first - shift < 0 ? 0 : first - shift;
    const int t0 = from / QT, per = first < sq.keys && from < sq.q_rows ? (sq.q_rows + QT - 1) / QT - t0 : 0;
    const int steps = (per * group + TEAMS - 1) / TEAMS;   // of either team; the second's last one may be empty
    if constexpr (kValuesInLds) {
        if (steps) {
            Feed<T, D, BM, TEAMS * WAVES, LOAD> fv(a.v.ld, a.dim);
            fv.load(head_of<T>(a.v, sq.k_lo + first, kv_head), sq.keys - first, lds);
            fv.store(lds);
            if (LOAD == kCut) {
                wait_loads<0>();
                fv.trim(lds);
            }
        }
    } else {
        load_row<T, D>(v, head_of<T>(a.v, row, kv_head), a.dim);
    }
    Feed<T, D, QT, WAVES, LOAD> fq(a.q.ld, a.dim), fg(a.dout.ld, a.dim);
    const Reader<T, D> read;
    char *const mine = lds + kValues + team * kSteps * kStep;
    const auto step_at = [&](int n) { return mine + (kSteps > 1 ? n % kSteps : 0) * kStep; };
    // the tile and the head of the team's n-th step; past the last, no rows
    const auto load = [&](int n) {
        const int s = TEAMS * n + team, down = s / per, r0 = (t0 + s - down * per) * QT, head = kv_head * group + down;
        const int left = down < group ? sq.q_rows - r0 : 0;
        char *to = step_at(n);
        const int64_t at = left > 0 ? (int64_t)head * a.rows + sq.q_lo + r0 : 0;
        if (DIRECT) {
            const int64_t row = left > 0 ? sq.q_lo + r0 : 0, of = left > 0 ? head : 0;
            fq.load(head_of<T>(a.q, row, of), left, to);
            fg.load(head_of<T>(a.dout, row, of), left, to + kTile);
            // each wave the same: one count of loads for all
            load_words_to_lds(buffer_of(a.stats + at, left > 0 ? (left < QT ? left : QT) * 8 : 0), lane * 4, lds_address(to + 2 * kTile));
            if (QT == 64)
                load_words_to_lds(buffer_of(a.stats + at, left > 0 ? (left < QT ? left : QT) * 8 : 0), lane * 4 + 256, lds_address(to + 2 * kTile + 256));
        } else {
            const int r = threadIdx.x % (WAVES * 64);
            if (r < QT) reinterpret_cast<RowStats *>(to + 2 * kTile)[r] = r < left ? a.stats[at + r] : RowStats{0, 0};
            const int64_t row = left > 0 ? sq.q_lo + r0 : 0, of = left > 0 ? head : 0;
            fq.load(head_of<T>(a.q, row, of), left, to);
            fq.store(to);
            fg.load(head_of<T>(a.dout, row, of), left, to + kTile);
            fg.store(to + kTile);
        }
    };
    if (DIRECT) {
        for (int n = 0; n < kSteps - 1; n++)
            if (n < steps) load(n);
    }
    for (int n = 0; n < steps; n++) {
        if (DIRECT) {
            constexpr int kLoads = 2 * decltype(fq)::N + QT / 32;
            if (kSteps == 3 && n + 1 < steps)
                arrive<kLoads>(fq, fg, step_at(n), kTile);
            else
                arrive<0>(fq, fg, step_at(n), kTile);
            if (n + kSteps - 1 < steps) load(n + kSteps - 1);
        } else {
            __syncthreads();
            load(n);
            __syncthreads();
        }
        const int s = TEAMS * n + team, down = s / per, q0 = (t0 + s - down * per) * QT;
        // a query i of this step sees key j where j <= i + shift; the lane's rows are in the order of its registers
        const int limit = key - shift - q0 - 4 * h;
        if (down < group && q0 + QT - 1 + shift >= key0) {
            const uint32_t qt = lds_address(step_at(n)), gt = qt + kTile, st = gt + kTile;
            const bool whole = q0 + shift >= key0 + 31;
#pragma unroll 1
            for (int b = 0; b < QT / 32; b++) {
                f32x16 s = 0.0f, dp = 0.0f;
                const uint32_t qr = read.rows_of(qt + b * 32 * D * 2);
#pragma unroll
                for (int d = 0; d < D / 16; d++) s = Mfma<T>::go(read.row(qr, 0, d), k[d], s);
                // exponent and delta of rows 8 e + 4 h + {0, 1} and {2, 3}
                const auto stats = [&](int e, int half) {
                    return *(__attribute__((address_space(3))) const f32x4 *)(uintptr_t)(st + (b * 32 + 8 * e + 4 * h + 2 * half) * 8);
                };
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const f32x4 st = stats(e / 2, e % 2);
                    s[2 * e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * e], c, -st[0]));
                    s[2 * e + 1] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * e + 1], c, -st[2]));
                }
                if (!whole) {
                    stay_apart();
#pragma unroll
                    for (int j = 0; j < 16; j++)
                        if (8 * (j / 4) + j % 4 < limit - b * 32) s[j] = 0.0f;
                }
                const Frag p[2] = {narrow<T>(s, 0), narrow<T>(s, 8)};
                const uint32_t gc = read.columns_of(gt + b * 32 * D * 2);
#pragma unroll
                for (int e = 0; e < 2; e++)
#pragma unroll
                    for (int d = 0; d < D / 32; d++) dv[d] = Mfma<T>::go(read.column(gc, e, d), p[e], dv[d]);
                const uint32_t gr = read.rows_of(gt + b * 32 * D * 2), vr = read.rows_of(lds_address(lds) + wave * 32 * D * 2);
#pragma unroll
                for (int d = 0; d < D / 16; d++)
                    dp = Mfma<T>::go(read.row(gr, 0, d), kValuesInLds ? read.row(vr, 0, d) : v[kValuesInLds ? 0 : d], dp);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const f32x4 st = stats(e / 2, e % 2);
                    dp[2 * e] = s[2 * e] * __builtin_fmaf(dp[2 * e], kLower<T>, -st[1]);
                    dp[2 * e + 1] = s[2 * e + 1] * __builtin_fmaf(dp[2 * e + 1], kLower<T>, -st[3]);
                }
                const Frag ds[2] = {narrow<T>(dp, 0), narrow<T>(dp, 8)};
                const uint32_t qc = read.columns_of(qt + b * 32 * D * 2);
#pragma unroll
                for (int e = 0; e < 2; e++)
#pragma unroll
                    for (int d = 0; d < D / 32; d++) dk[d] = Mfma<T>::go(read.column(qc, e, d), ds[e], dk[d]);
            }
        }
    }
    // the first team adds up dv, the second dk; each stores its own
    const Join<D> join{lds, team, wave, WAVES};
    __syncthreads();
    if (TEAMS > 1) {
        join.give(dv, 0);
        __syncthreads();
        join.take(dv, 0, TEAMS);
        __syncthreads();
        join.give(dk, 1);
        __syncthreads();
        join.take(dk, 1, TEAMS);
        __syncthreads();
    }
    // keys of the range that do not count get 0 (their lanes hold another row's result, or anything)
    const int left = sq.k_rows - key0;
    char *out = lds + (team * WAVES + wave) * 32 * D * 2;
    if (team == 0)
        store_rows<T, D>(out, dv, !there, kLower<T>, a.dim, [&](int r) -> T * {
            return r < left ? out_of<T>(a.dv, sq.k_lo + key0 + r, kv_head) : nullptr;
        });
    if (TEAMS == 1) out += WAVES * 32 * D * 2;
    if (team == (TEAMS > 1))
        store_rows<T, D>(out, dk, !there, a.scale, a.dim, [&](int r) -> T * {
            return r < left ? out_of<T>(a.dk, sq.k_lo + key0 + r, kv_head) : nullptr;
        });
}

// ---------------------------------------------------------------- launches
// Tiles of `size` rows that the ranges of `rows` rows can need together.
int64_t tiles_of(int64_t rows, int64_t size, int sequences) { return rows / size + sequences + 2; }

// Launches a kernel that takes one item a workgroup, on as many items at a time as one launch holds.
template <typename K> int launch_items(K *kernel, int64_t items, int threads, void *stream, Attention a) {
    const int64_t most = most_blocks(threads);
    for (int64_t at = 0; at < items; at += most) {
        a.first = (uint32_t)at;
        if (const int e = launch(kernel, items - at < most ? items - at : most, threads, stream, a)) return e;
    }
    return 0;
}

Load load_of(const Attention &a, const HeadRows &x, const HeadRows &y) {
    const auto even = [](const HeadRows &x) {
        return reinterpret_cast<uintptr_t>(x.p) % 4 == 0 && x.ld % 2 == 0 && x.head_ld % 2 == 0;
    };
    return a.dim % 2 || !even(x) || !even(y) ? kThrough : a.dim % 8 ? kCut : kDirect;
}

template <typename T, int D, Load LOAD> int forward(Attention a, void *stream) {
    const int64_t packed = (int64_t)a.rows * (a.heads / a.kv_heads);
    if (a.splits) {
        a.tiles = (int)tiles_of(packed, 32, a.sequences);
        const int64_t items = (int64_t)a.tiles * a.kv_heads * a.splits;
        if (const int e = launch_items(k_forward_few<T, D, LOAD>, items, 256, stream, a)) return e;
        if (a.splits == 1) return 0;
        if (a.splits <= kFewShares) return launch_items(k_join_few<T>, ((int64_t)a.rows * a.heads + 7) / 8, 256, stream, a);
        return launch_items(k_join<T>, (int64_t)a.rows * a.heads * ((a.dim + 31) / 32), 256, stream, a);
    }
    a.tiles = (int)tiles_of(packed, 128, a.sequences);
    return launch_items(k_forward<T, D, LOAD>, (int64_t)a.tiles * a.kv_heads, 256, stream, a);
}

template <typename T, int D> int forward(const Attention &a, void *stream) {
    switch (load_of(a, a.k, a.v)) {
        case kDirect: return forward<T, D, kDirect>(a, stream);
        case kCut: return forward<T, D, kCut>(a, stream);
        default: return forward<T, D, kThrough>(a, stream);
    }
}

template <typename T> int forward(const Attention &a, void *stream) {
    if (a.dim <= 32) return forward<T, 32>(a, stream);
    return a.dim <= 64 ? forward<T, 64>(a, stream) : forward<T, 128>(a, stream);
}

template <typename T, int D, Load LOAD> int queries_grad(Attention a, void *stream) {
    if (!a.rows) return 0;
    a.tiles = (int)tiles_of((int64_t)a.rows * (a.heads / a.kv_heads), 128, a.sequences);
    return launch_items(k_queries_grad<T, D, LOAD>, (int64_t)a.tiles * a.kv_heads, 256, stream, a);
}

// Tiles of 128 keys on one team, or of 64 on four.  Four share a tile's steps: with few tiles and many steps, as
// where long sequences share heads, no CU waits long for the longest tile's (4 causal sequences, 16384
// rows, 16 heads of 128 to 4: 702 us against 1108 on one); with many tiles one team has two workgroups a CU (64 x
// 256 rows, 16 heads of 64: 60 us against 148 on four), and so with few steps, where joining costs as much (59 x 16
// rows, 16 heads of 128, both kernels: 38 us against 57).  Several sequences of sixteen tiles or more are dealt by
// place (the long ones again: 702 us against 746 in their order; forward and dq, whose tiles are
// shorter, gained 1 % there and lost 6 on 4 sequences of 680 rows).  Medians of 66 passes.
template <typename T, int D, Load LOAD> int keys_grad(Attention a, void *stream) {
    if (!a.key_rows) return 0;
    constexpr int QT = D == 32 ? 64 : 32;
    const int64_t some = a.key_rows < a.sequences ? a.key_rows : a.sequences, large = ((int64_t)a.key_rows + 127) / 128;
    const int64_t steps = (int64_t)a.rows / a.sequences * (a.heads / a.kv_heads) / QT;
    if constexpr (LOAD != kThrough) {
        if ((large > some ? large : some) * a.kv_heads < 4 * kCus && steps >= 16) {
            a.tiles = (int)tiles_of(a.key_rows, 64, a.sequences);
            a.by_place = a.sequences > 1 && a.sequences + 2 <= 128 && a.key_rows >= 16 * 64ll * a.sequences;
            return launch_items(k_keys_grad<T, D, QT, 2, 4, LOAD>, (int64_t)a.tiles * a.kv_heads, 512, stream, a);
        }
    }
    a.tiles = (int)tiles_of(a.key_rows, 128, a.sequences);
    return launch_items(k_keys_grad<T, D, QT, 4, 1, LOAD>, (int64_t)a.tiles * a.kv_heads, 256, stream, a);
}

template <typename T, int D> int backward(const Attention &a, void *stream) {
    const Load kv = load_of(a, a.k, a.v), q = load_of(a, a.q, a.dout);
    if (const int e = kv == kDirect ? queries_grad<T, D, kDirect>(a, stream)
                      : kv == kCut  ? queries_grad<T, D, kCut>(a, stream)
                                    : queries_grad<T, D, kThrough>(a, stream))
        return e;
    if (kv == kThrough || q == kThrough) return keys_grad<T, D, kThrough>(a, stream);
    return q == kDirect ? keys_grad<T, D, kDirect>(a, stream) : keys_grad<T, D, kCut>(a, stream);
}

template <typename T> int backward(const Attention &a, void *stream) {
    if (a.dim <= 32) return backward<T, 32>(a, stream);
    return a.dim <= 64 ? backward<T, 64>(a, stream) : backward<T, 128>(a, stream);
}

}  // namespace

int launch_attention_forward(const Attention &a, void *stream) {
    return a.dtype == PASE_BF16 ? forward<__bf16>(a, stream) : forward<_Float16>(a, stream);
}
int launch_attention_backward(const Attention &a, void *stream) {
    return a.dtype == PASE_BF16 ? backward<__bf16>(a, stream) : backward<_Float16>(a, stream);
}

}  // namespace pase
