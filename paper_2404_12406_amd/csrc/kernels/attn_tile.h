// What the attention kernels share: tiles of rows in LDS, their fragments for the matrix
// cores, and which rows of which sequence a block works on.
//
// A fragment is 16 bytes a lane for both types.  A chunk is what one fragment of each
// operand contributes to a sum: 16 elements of bf16 (one 32x32x16 instruction), 8 of fp32
// (four 32x32x2).  Which element is which lane's is the kernels' own choice as long as
// both operands agree.  The sums of a 32x32 tile lie as column l % 32 in lane l, rows
// 8 g + 4 (l / 32) + j in element 4 g + j; taken as the other operand of the next
// product, those elements are the rows 16 c + 4 (l / 32) + {0..3, 8..11} of chunk c in
// bf16 (8 c + 4 (l / 32) + {0..3} in fp32), so col_frag() reads these rows and no value
// moves between lanes.
#pragma once

#include <algorithm>

#include "block_math.h"
#include "lds_dma.h"

namespace ms {
namespace att {

template <typename T> struct Mat;
template <> struct Mat<bf16> {
    typedef bf16x8 Frag;
    static constexpr int V = 8, KC = 16;   // elements of a fragment, of a chunk
    static __device__ __forceinline__ floatx16 mma(Frag a, Frag b, floatx16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Mat<float> {
    typedef floatx4 Frag;
    static constexpr int V = 4, KC = 8;
    static __device__ __forceinline__ floatx16 mma(Frag a, Frag b, floatx16 c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
};

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16_t;
typedef __attribute__((address_space(3))) char lds_char_t;

// How a call of DC padded columns is laid out: rows in LDS have DP of them, a power of two
// (the swizzle's units are eight at a time).
template <int DC> constexpr int kPitch = DC <= 64 ? 64 : DC <= 128 ? 128 : 256;

// Rows of DP elements in LDS, whose 256 bytes of banks are read in one clock.  The low
// bits of a 16-byte unit's number are turned by its row so that what is read together lies
// in different banks: one unit of 16 rows (row_frag), four units of four rows or, in fp32, a
// word of each of 32 columns in two rows (col_frag).  swz() is linear in the row's bits, so
// the part of an address that differs between lanes is worked out once.
template <typename T, int DP>
struct Tile {
    typedef typename Mat<T>::Frag Frag;
    static constexpr int V = Mat<T>::V, U = DP / V, RB = DP * (int)sizeof(T);
    static constexpr int LOW = U < 16 ? 7 : 15;
    static __host__ __device__ __forceinline__ constexpr int swz(int row) {
        return sizeof(T) == 4 ? (row >> 2 & 1) << 3 | (row >> 3 & 1) << 2 | (row & 3)
               : U < 16       ? (row >> 1 & 1) << 2 | (row >> 2 & 3)
                              : (row & 3) << 2 | (row >> 2 & 3);
    }
    static __device__ __forceinline__ int at(int row, int unit) { return row * RB + ((unit ^ swz(row)) << 4); }
    // at(row | row_, unit | unit_) of a tile that begins on 256 bytes: no bits in common, the second ones known
    // when this is compiled.  What differs between lanes is in one register, the rest an XOR.
    static __device__ __forceinline__ const lds_char_t *spot(const char *base, int row, int unit, int byte, int row_, int unit_) {
        const uint32_t p = (uint32_t)(uintptr_t)(const lds_char_t *)base + (uint32_t)(at(row, unit) + byte);
        return (const lds_char_t *)(uintptr_t)((p ^ (uint32_t)(((unit_ ^ swz(row_)) & LOW) << 4)) + (uint32_t)(row_ * RB + ((unit_ & ~LOW) << 4)));
    }

    // Row r0 + l % 32 (r0 a multiple of 32), chunk c of its elements: units 2 c + l / 32.
    static __device__ __forceinline__ Frag row_frag(const char *base, int r0, int c, int lane) {
        return *(const __attribute__((address_space(3))) Frag *)spot(base, lane & 31, lane >> 5, 0, r0, 2 * c);
    }
    // Column 32 t + l % 32, chunk c of the rows from r0 (a multiple of 32) on.
    static __device__ __forceinline__ Frag col_frag(const char *base, int r0, int t, int c, int lane) {
        Frag f;
        if constexpr (sizeof(T) == 2) {
            // ds_read_b64_tr_b16: each 16 lanes address four rows of 16 columns, 8 bytes a
            // lane, and hold a column's four rows afterwards
            const int r = lane & 15, g = lane >> 4, row = 4 * (g >> 1) + (r >> 2), unit = 2 * (g & 1) + ((r & 3) >> 1), byte = (r & 1) << 3;
            v4i16 *v = reinterpret_cast<v4i16 *>(&f);
            v[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t *)spot(base, row, unit, byte, r0 + 16 * c, 4 * t));
            v[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t *)spot(base, row, unit, byte, r0 + 16 * c + 8, 4 * t));
        } else {
            const int m = lane & 31, hh = lane >> 5;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                f[j] = *(const __attribute__((address_space(3))) float *)spot(base, 4 * hh, m >> 2, (m & 3) << 2, r0 + 8 * c + j, 8 * t);
        }
        return f;
    }
};

// Loads of ROWS rows into a tile by NW waves, straight into LDS: each wave's lanes fill
// 1024 bytes in a row.  Rows past the buffer's end and elements past D read as zeros.
template <typename T, int DP, int ROWS, int NW>
struct Loader {
    typedef Tile<T, DP> Ti;
    static constexpr int PER = ROWS * Ti::U / (64 * NW);
    static_assert(PER >= 1 && PER * 64 * NW == ROWS * Ti::U, "whole loads");
    uint32_t off[PER];
    int64_t ts;   // bytes between rows
    __device__ __forceinline__ void init(int64_t row_stride, int D, int w, int lane) {
        ts = row_stride * (int)sizeof(T);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int idx = (i * NW + w) * 64 + lane, row = idx / Ti::U, unit = (idx % Ti::U) ^ Ti::swz(row);
            off[i] = unit * Ti::V < D ? (uint32_t)(row * (int)ts + unit * 16) : 0x80000000u;
        }
    }
    // base: row 0 of the tile; rows: how many there are from there on
    __device__ __forceinline__ void issue(const char *base, int rows, int D, char *lds, int w) const {
        const int n = rows < ROWS ? rows : ROWS;
        const __amdgpu_buffer_rsrc_t r = g2::rsrc(base, n > 0 ? (uint32_t)((n - 1) * (int)ts + D * (int)sizeof(T)) : 0u);
#pragma unroll
        for (int i = 0; i < PER; ++i) g2::dma16<true>(r, lds + (i * NW + w) * 1024, off[i]);
    }
};

// All of a wave's own loads have landed and its reads of LDS are done; then the block's.
__device__ __forceinline__ void tile_sync() {
    __builtin_amdgcn_s_waitcnt(7 << 4);
    g2::block_sync<true>();
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A sequence's rows on the side that blocks divide into tiles, its rows on the other
// side, and the tile.
struct Span {
    int a0, na, b0, nb, tile;
};

// Tiles of ROWS rows over the sequences aoff[0..n]: sequence i's begin at slot
// start / ROWS + i, which leaves each as many slots as it can need without a count of
// tiles having been taken.  Rows before the first and past the last sequence
// are sequences of their own, without partners.  Offsets are held to [0, Ta].
__device__ __forceinline__ Span find_span(const int32_t *aoff, const int32_t *boff, int n, int Ta, int Tb, int slot, int rows) {
    if (!aoff) return Span{0, Ta, 0, Tb, slot};
    auto edge = [&](int i) {   // of n + 2 sequences
        return i <= 0 ? 0 : i > n + 1 ? Ta : min(max(aoff[i - 1], 0), Ta);
    };
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int i0 = 0; i0 <= n + 1; i0 += 64) {
        const int i = i0 + lane;
        before += (int)__popcll(__ballot(i <= n + 1 && edge(i) / rows + i <= slot));
    }
    const int i = uniform(before) - 1;
    const int a0 = uniform(edge(i)), a1 = uniform(max(edge(i + 1), a0));
    Span s{a0, a1 - a0, 0, 0, slot - (a0 / rows + i)};
    if (i >= 1 && i <= n) {
        const int b0 = uniform(min(max(boff[i - 1], 0), Tb));
        s.b0 = b0;
        s.nb = uniform(max(min(max(boff[i], 0), Tb), b0)) - b0;
    }
    return s;
}

// The sum of a wave's values, by moves within the vector registers.
__device__ __forceinline__ int wave_add(int v) {
#define ATT_MOVED(ctrl, rows) __builtin_amdgcn_update_dpp(0, v, ctrl, rows, 0xf, false)
    v += ATT_MOVED(0x111, 0xf);   // from 1, 2, 4 and 8 lanes below, within rows of 16
    v += ATT_MOVED(0x112, 0xf);
    v += ATT_MOVED(0x114, 0xf);
    v += ATT_MOVED(0x118, 0xf);
    v += ATT_MOVED(0x142, 0xa);   // the rows before
    v += ATT_MOVED(0x143, 0xc);
#undef ATT_MOVED
    return __builtin_amdgcn_readlane(v, 63);
}

// The tile that is `rank`-th in work, most first, so that the blocks that take longest
// begin first and none of them is left over at the end.  A causal sequence's tiles have work in steps of one tile's
// rows (from its last one on with last_first, else from its first), others all their keys.
// To 62 sequences, a lane each; beyond, as they come.  Past the last tile: one without rows.
__device__ __forceinline__ Span find_ranked(const int32_t *aoff, const int32_t *boff, int n, int Ta, int Tb, int rank, int rows, bool causal,
                                            bool last_first) {
    const int tiles = (Ta + rows - 1) / rows;
    if (!aoff) return Span{0, Ta, 0, Tb, last_first ? tiles - 1 - rank : rank};
    if (n + 2 > 64) return find_span(aoff, boff, n, Ta, Tb, rank, rows);
    const int i = threadIdx.x & 63;
    auto edge = [&](int i) {   // of n + 2 sequences, as find_span()'s
        return i <= 0 ? 0 : i > n + 1 ? Ta : min(max(aoff[i - 1], 0), Ta);
    };
    Span s{0, 0, 0, 0, 0};
    if (i <= n + 1) {
        s.a0 = edge(i);
        s.na = max(edge(i + 1), s.a0) - s.a0;
        if (i >= 1 && i <= n) {
            s.b0 = min(max(boff[i - 1], 0), Tb);
            s.nb = max(min(max(boff[i], 0), Tb), s.b0) - s.b0;
        }
    }
    const int nt = (s.na + rows - 1) / rows, level = s.nb / rows + tiles + 2;   // of the first tile; above 0 for all
    auto from = [&](int x) {   // tiles of level x and above
        return causal ? min(max(level - x + 1, 0), nt) : level >= x ? nt : 0;
    };
    if (rank >= wave_add(nt)) return Span{0, 0, 0, 0, 0};
    int lo = 0, hi = Tb / rows + tiles + 3;   // all tiles, none
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (wave_add(from(mid)) > rank) lo = mid;
        else hi = mid;
    }
    const int above = from(lo + 1), here = from(lo) - above, k = rank - wave_add(above);   // the k-th of level lo
    int upto = here;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int v = __shfl_up(upto, d);
        if (i >= d) upto += v;
    }
    const uint64_t mine = __ballot(k < upto);
    const int src = uniform((int)__ffsll((unsigned long long)mine) - 1);
    const int j = above + k - (upto - here);   // tiles of this sequence before it
    s.tile = last_first ? nt - 1 - j : j;
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, src); };
    return Span{of(s.a0), of(s.na), of(s.b0), of(s.nb), of(s.tile)};
}

// Which head and which rank a block has: all heads' longest tiles first; heads that lie
// side by side (and share keys) on one XCD, whose L2 they then share, where eight divide them.
__device__ __forceinline__ void find_head(int b, int H, int &head, int &rank) {
    rank = b / H;
    head = b - rank * H;
    if (H % 8 == 0) head = (head & 7) * (H / 8) + (head >> 3);
}

// Slots of find_span().
inline int64_t span_slots(bool packed, int n, int64_t Ta, int rows) {
    return packed ? Ta / rows + n + 2 : (Ta + rows - 1) / rows;
}

// Where there are few blocks they divide their other side: to some 512 of them (1024 in fp32, whose steps take
// longer), as long as two of the `steps` that they have on average are left to each and the partial sums stay
// below 24 MiB.
// (fp32, 1777 rows in 5 sequences, 6 on 2 heads of 72, all gradients: 906 -> 190 us; with 512 blocks 202.  bf16, 4 x 1024
// rows, 8 on 2 heads of 64, forward: 30 us with 1024 blocks, 17 with 304.)
template <typename T>
inline int span_splits(int64_t blocks, int64_t steps, int64_t bytes) {
    const int64_t want = (sizeof(T) == 2 ? 512 : 1024) / std::max<int64_t>(blocks, 1), most = (int64_t(24) << 20) / std::max<int64_t>(bytes, 1);
    return (int)std::max<int64_t>(1, std::min({want, steps / 2, most}));
}

// Up to 768 blocks are one and a half times what the card's 256 CUs hold at once, two each, and the longest end
// alone on a CU that they cannot fill.  Where they have `least` steps or more on average, such blocks have eight waves, which take every
// other step each and meet at the end.  (bf16, 8192 rows of one sequence, 8 heads of 128: forward 178 -> 144 us,
// dv 186 -> 148.  With two to 16 steps the longer start costs more: 64 x 128 rows, 4 heads of 64 forward
// 10 -> 13 us, 8 x 1024 rows 22 -> 24.  With 1152 blocks dv 312 -> 356 us.)
inline bool wide_blocks(int64_t blocks, int64_t steps, int64_t least) { return blocks <= 768 && steps >= least; }

// The sum (maximum) of a lane's value and that of the lane 32 away.
__device__ __forceinline__ floatx2 halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return floatx2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ float both_sum(float v) {
    const floatx2 h = halves(v);
    return h.x + h.y;
}
__device__ __forceinline__ float both_max(float v) {
    const floatx2 h = halves(v);
    return fmaxf(h.x, h.y);
}

// Whether a step has places that some of a wave's rows do not see, known when its loop is
// compiled: the steps without are a loop of their own.  (In one loop the branch around
// wild_product() made copies of all sums, 64 moves a step.)
struct Masked { static constexpr bool value = true; };
struct Full { static constexpr bool value = false; };

template <int N> struct Number { static constexpr int value = N; };

// 2^((s - ref) c).  In bf16 in one operation, on -ref c, whose rounding is a factor of all weights that are
// taken with the same ref; those of another ref, and of other waves or blocks, have another, up to 2^-24 |ref c| ln 2 of
// themselves apart: less than a weight's own 2^-8 to |ref c| of some 2^16.  In fp32 the difference first, which is exact near ref.
template <typename T>
__device__ __forceinline__ float power(float s, float ref, float minus, float c) {
    return __builtin_amdgcn_exp2f(sizeof(T) == 2 ? __builtin_fmaf(s, c, minus) : (s - ref) * c);
}

// A 32x32 tile's sums as fragments: chunk c.
template <typename T>
__device__ __forceinline__ typename Mat<T>::Frag as_frag(const floatx16 &s, int c) {
    typename Mat<T>::Frag f;
#pragma unroll
    for (int j = 0; j < Mat<T>::V; ++j) f[j] = from_f32<T>(s[c * Mat<T>::V + j]);
    return f;
}

__device__ __forceinline__ floatx16 zero16x() {
    floatx16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    return z;
}

// Whether rows r0.. of a tile hold an infinity or NaN.
template <typename T, int DP, int ROWS>
__device__ __forceinline__ bool any_wild(const char *tile, int r0, int lane) {
    typedef Tile<T, DP> Ti;
    // by the largest magnitude, of halves of words in bf16
    u16x2 top = {0, 0};
    uint32_t most = 0;
#pragma unroll 2
    for (int i = 0; i < ROWS * Ti::U / 64; ++i) {
        const u32x4 v = *reinterpret_cast<const u32x4 *>(tile + r0 * Ti::RB + i * 1024 + lane * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 2) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, v[j] & 0x7fff7fffu));
            else most = max(most, v[j] & 0x7fffffffu);
        }
    }
    const bool bad = sizeof(T) == 2 ? top[0] >= 0x7f80u || top[1] >= 0x7f80u : most >= 0x7f800000u;
    return __any(bad);
}

// acc += columns of `tile` times b (N chunks), a row at a time, where rows outside lo..hi, which the
// lane's column does not see, take no part whatever they hold: for tiles with masked places where any_wild().
// (By the rows, not by weights of zero: 0 times an infinity that is seen is NaN, as it is in other tiles.)
template <typename T, int DP, int DC, int N>
__device__ __forceinline__ void wild_product(floatx16 (&acc)[DC / 32], const char *tile, int r0, const typename Mat<T>::Frag (&b)[N], int lo, int hi,
                                             int lane) {
    typedef Mat<T> M;
    typedef Tile<T, DP> Ti;
    constexpr int PER = 4 / (int)sizeof(T);   // elements of a word
    const int n = lane & 31, hh = lane >> 5;
#pragma unroll
    for (int t = 0; t < DC / 32; ++t) {
        __builtin_amdgcn_sched_barrier(0);   // (one tile of columns after the other: together they spill)
#pragma unroll 1
        for (int row = 0; row < N * M::KC; ++row) {
            // whose element is the row's weight: chunk, half of the wave, place in the fragment
            const int c = row / M::KC, in = row % M::KC, half = in >> 2 & 1, e = (in >> 3 << 2) | (in & 3);
            uint32_t word = 0;   // (as they are: converted, all weights would be held over the loop)
#pragma unroll
            for (int k = 0; k < N; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) word = k == c && j == e / PER ? __builtin_bit_cast(u32x4, b[k])[j] : word;
            const float p = __shfl(__uint_as_float(PER == 1 ? word : e & 1 ? word & 0xffff0000u : word << 16), n + 32 * half);
            const bool seen = row >= lo && row <= hi;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int d = 32 * t + 8 * g + 4 * hh;
                const T *v = reinterpret_cast<const T *>(tile + Ti::at(r0 + row, d / M::V)) + d % M::V;
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[t][4 * g + j] = seen ? acc[t][4 * g + j] + p * to_f32(v[j]) : acc[t][4 * g + j];
            }
        }
    }
    __builtin_amdgcn_sched_barrier(0);
}

// acc += columns of `tile` times b.
template <typename T, int DP, int DC, int N>
__device__ __forceinline__ void add_product(floatx16 (&acc)[DC / 32], const char *tile, int r0, const typename Mat<T>::Frag (&b)[N], int lane) {
#pragma unroll
    for (int t = 0; t < DC / 32; ++t)
#pragma unroll
        for (int i = 0; i < N; ++i) acc[t] = Mat<T>::mma(Tile<T, DP>::col_frag(tile, r0, t, i, lane), b[i], acc[t]);
}

// A wave's 32 rows of results, which lie as columns of 32x32 tiles (x scale, or zeros), to
// memory by way of its own part of LDS: whole 16-byte vectors side by side.
template <typename T, int DP, int DC>
__device__ __forceinline__ void store_rows(const floatx16 (&acc)[DC / 32], float scale, bool zero, char *lds, T *out, int64_t ts, int rows, int D,
                                           int lane) {
    typedef Tile<T, DP> Ti;
    const int n = lane & 31, hh = lane >> 5;
#pragma unroll
    for (int t = 0; t < DC / 32; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            T v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = from_f32<T>(zero ? 0.f : acc[t][4 * g + j] * scale);
            const int d = 32 * t + 8 * g + 4 * hh;
            char *to = lds + Ti::at(n, d / Ti::V) + (d % Ti::V) * (int)sizeof(T);
            if constexpr (sizeof(T) == 2) *reinterpret_cast<uint64_t *>(to) = *reinterpret_cast<const uint64_t *>(v);
            else *reinterpret_cast<u32x4 *>(to) = *reinterpret_cast<const u32x4 *>(v);
        }
#pragma unroll
    for (int i = 0; i < 32 * Ti::U / 64; ++i) {
        const int idx = i * 64 + lane, row = idx / Ti::U, unit = idx % Ti::U;
        const u32x4 v = *reinterpret_cast<const u32x4 *>(lds + Ti::at(row, unit));
        if (row < rows && unit * Ti::V < D) *reinterpret_cast<u32x4 *>(out + row * ts + unit * Ti::V) = v;
    }
}

// The same as sums in fp32, [rows][DC].
template <int DC>
__device__ __forceinline__ void store_sums(const floatx16 (&acc)[DC / 32], float *out, int64_t ts, int rows, int lane) {
    const int n = lane & 31, hh = lane >> 5;
    if (n >= rows) return;
#pragma unroll
    for (int t = 0; t < DC / 32; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            floatx4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = acc[t][4 * g + j];
            *reinterpret_cast<floatx4 *>(out + n * ts + 32 * t + 8 * g + 4 * hh) = v;
        }
}

// A wave's 32 rows as the column operand of a product: row l % 32, chunk c; zeros past
// `rows` and D.
template <typename T>
__device__ __forceinline__ typename Mat<T>::Frag load_row(const T *p, int64_t ts, int rows, int D, int c, int lane) {
    const int n = lane & 31, d = (2 * c + (lane >> 5)) * Mat<T>::V;
    typename Mat<T>::Frag v;
#pragma unroll
    for (int j = 0; j < Mat<T>::V; ++j) v[j] = (T)0.f;
    if (n < rows && d < D) v = *reinterpret_cast<const typename Mat<T>::Frag *>(p + n * ts + d);
    return v;
}

// All of them, held in registers; or (HOLD false, where they are too many) read where they are used.
template <typename T, int DC, bool HOLD = true>
struct Rows {
    static constexpr int C = DC / Mat<T>::KC;
    typename Mat<T>::Frag f[HOLD ? C : 1];
    const T *p;
    int64_t ts;
    int rows, D;
    __device__ __forceinline__ void init(const T *p_, int64_t ts_, int rows_, int D_, int lane) {
        p = p_, ts = ts_, rows = rows_, D = D_;
        if constexpr (HOLD)
#pragma unroll
            for (int c = 0; c < C; ++c) f[c] = load_row<T>(p, ts, rows, D, c, lane);
    }
    // They have arrived.  (Where no later wait for all loads is known to the compiler, it would
    // put one in front of their first use, in the loop.)
    __device__ __forceinline__ void settle() {
        if constexpr (HOLD)
#pragma unroll
            for (int c = 0; c < C; ++c) asm volatile("" : "+v"(f[c]));
    }
    __device__ __forceinline__ typename Mat<T>::Frag get(int c, int lane) const {
        if constexpr (HOLD) return f[c];
        else return load_row<T>(p, ts, rows, D, c, lane);
    }
};

}  // namespace att
}  // namespace ms

// F<T, columns>(a, ...) for the columns that heads of a.D elements take.
#define ATT_COLUMNS(F, T, a, ...)                                    \
    ((a).D <= 64    ? F<T, 64>(a __VA_OPT__(, ) __VA_ARGS__)         \
     : (a).D <= 96  ? F<T, 96>(a __VA_OPT__(, ) __VA_ARGS__)         \
     : (a).D <= 128 ? F<T, 128>(a __VA_OPT__(, ) __VA_ARGS__)        \
     : (a).D <= 192 ? F<T, 192>(a __VA_OPT__(, ) __VA_ARGS__)        \
                    : F<T, 256>(a __VA_OPT__(, ) __VA_ARGS__))
