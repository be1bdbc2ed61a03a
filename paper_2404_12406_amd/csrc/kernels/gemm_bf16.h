// Shared by the bf16 GEMM kernels (gemm_bf16.hip, gemm_fused.h): arguments,
// LDS layouts, fragment reads, the tile configuration that gemm_block_body.inc
// is written for, and the host's estimate of a tile's run time.
#pragma once

#include <algorithm>

#include "common.h"
#include "lds_dma.h"
#include "limits.h"
#include "../device.h"

namespace ms {
namespace g2 {

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16_t;

// kDgrad reads the filter from a transposed copy Wt[C][R][S][K] (both
// operands K-contiguous); kDgradN reads W[K][R][S][C] in place as an
// M/N-contiguous operand (no copy, transposing LDS reads).
enum Mode { kFwd = 0, kDgrad = 1, kWgrad = 2, kDgradN = 3 };

constexpr int BK = 64;                   // reduction step (elements)

struct Args {
    const bf16 *a;
    const bf16 *b;
    bf16 *c;              // output (or nullptr when the output is fp32 partials)
    float *part;          // split-K partials: part_stride floats per split (nullptr: splits == 1)
    float *dbpart;        // WGRAD fused bias-gradient partials [splits][M] (nullptr: off)
    float *cspart;        // unit-geometry DGRAD: column sums of dy (the bias gradient),
                          // one partial row per (row tile, summing wave) (nullptr: off)
    int cs_cw;            // columns of dy per block column (a multiple of 8)
    int64_t part_stride;  // FWD/WGRAD: M*N; DGRAD: N*H*W*C (partials indexed by dx pixel)
    const bf16 *bias;     // FWD / DGRAD per-column bias (nullptr: none; DGRAD: the
                          // transposed convolution's forward)
    ConvDims g;
    int M, N, K;          // GEMM extents (DGRAD: bounds over phases)
    int ntm, ntn;
    int ldc;              // bf16 output row stride in elements (0: N); a launch that covers
                          // a column range of a wider output passes the full width
    int k_split, splits;  // reduction range per split (a multiple of BK) and split count
    uint32_t a_bytes, b_bytes;
    // three-dimensional convolutions (D3): T depth taps; the images of the
    // pixel side are m_depth per sample, image o reading A's (WGRAD: B's) tensor,
    // a_depth images per sample, at depth o * d_step + d_off +- tap
    int T, m_depth, a_depth, d_step, d_off;
};

struct Phase {
    int fh, fw, h0, w0, Hp, Wp, Rp, Sp, dh, dw;
};

__device__ __forceinline__ Phase make_phase(const ConvDims &g, int z) {
    Phase f;
    f.fh = z / g.sw;
    f.fw = z % g.sw;
    f.h0 = ((f.fh - g.ph) % g.sh + g.sh) % g.sh;
    f.w0 = ((f.fw - g.pw) % g.sw + g.sw) % g.sw;
    f.Hp = f.h0 < g.H ? (g.H - f.h0 + g.sh - 1) / g.sh : 0;
    f.Wp = f.w0 < g.W ? (g.W - f.w0 + g.sw - 1) / g.sw : 0;
    f.Rp = f.fh < g.R ? (g.R - f.fh + g.sh - 1) / g.sh : 0;
    f.Sp = f.fw < g.S ? (g.S - f.fw + g.sw - 1) / g.sw : 0;
    f.dh = (f.h0 + g.ph - f.fh) / g.sh;
    f.dw = (f.w0 + g.pw - f.fw) / g.sw;
    return f;
}

// 16-byte chunk swizzle of a K-contiguous tile row (128 bytes = 8 chunks).
// 16 consecutive rows reading the same logical chunk land on 16 distinct
// 16-byte bank groups (the LDS serves 256 bytes per clock).
__device__ __forceinline__ int swz_k(int row) { return (row & 7) ^ ((row >> 3) & 1); }

// Slot swizzle of an M/N-contiguous tile k-row ([k][mn], 16-byte slots).
// A transposed read serves 32 lanes at a time: two 16-lane groups that each
// read 4 k-rows x 2 adjacent slots, the second group 2 slots to the right.
// Rows of 16 or more slots start on the same bank, so the XOR must spread
// the 4 rows by 4 slots (the 32 lanes then cover 16 distinct slots = all 64
// banks); rows of 8 slots alternate between the two bank halves and an XOR
// by 2 suffices.  Both keep the slot pair of a group adjacent.
template <int SPR>
__device__ __forceinline__ int swz_m(int krow) {
    if constexpr (SPR >= 16) return (krow & 3) << 2;
    else return (krow & 3) << 1;
}

// MFMA fragment (8 k values of one m/n index) from a [BK k][R mn] tile for
// the 32x32x16 shape: lane l needs column mn0 + l%32 at k-rows
// 16*sub + 8*(l/32) .. +7.  ds_read_b64_tr_b16 works per 16-lane group
// g = l/16: lane 16g + r addresses k-row kb + 4h + r/4 at columns
// cb + 4*(r%4) .. +3 (kb = 16*sub + 8*(g/2), cb = mn0 + 16*(g%2)) and, after
// the in-group transpose, holds column cb + r of k-rows kb + 4h .. kb+4h+3.
template <int R>
__device__ __forceinline__ bf16x8 frag_mn(const char *base, int mn0, int sub, int lane) {
    constexpr int SPR = R / 8;
    const int g = lane >> 4, r = lane & 15;
    const int kb = 16 * sub + 8 * (g >> 1), cb = mn0 + 16 * (g & 1);
    bf16x8 v;
    v4i16 *pv = reinterpret_cast<v4i16 *>(&v);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int krow = kb + 4 * h + (r >> 2);
        const int mn = cb + 4 * (r & 3);
        const int pos = (mn >> 3) ^ swz_m<SPR>(krow);
        const int off = krow * (R * 2) + (pos << 4) + ((mn & 7) << 1);
        pv[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t *)(base + off));
    }
    return v;
}

// Fragment from a row-major [row][BK] tile (128-byte rows, swizzled 16-byte
// chunks): lane l reads row `row` (= tile row + l%32), chunk 2*sub + l/32.
__device__ __forceinline__ bf16x8 frag_kc(const char *base, int row, int sub, int lane) {
    const int chunk = 2 * sub + (lane >> 5);
    const int off = row * (BK * 2) + ((chunk ^ swz_k(row)) << 4);
    return *reinterpret_cast<const bf16x8 *>(base + off);
}

// Column sums of dy for the bias gradient, taken by a unit-geometry input
// gradient (there A = dy: row m holds the K output channels of pixel m).
// Block (tm, tn) adds rows m0 .. m0+BM-1 for columns [tn*cw, tn*cw + cw) of
// K; nwc waves take part, wave w writing partial row tm*nwc + w of part
// ([rows][K] fp32).  Lane t = 64w + l of the nwc*64 owns column vector
// t % cvp (8 channels) of each pass of 8*cvp columns and walks the rows
// t / cvp + i * rgs (rgs = nwc*64 / cvp), NB loads in flight; the lanes of a
// wave that share a column vector meet by shuffles.  Loads go through the
// buffer descriptor of dy with out-of-range rows and columns sent past its
// end, so they read zeros.  The data was read by this block's main loop
// moments earlier.  issue() may be called first (the first batch of the
// first pass, e.g. before an epilogue); run() then starts from it.
template <int NB>
struct DyColumnSums {
    __amdgpu_buffer_rsrc_t ra;
    int M, K, m0, BM, kb, ncv, cvp, cvl, rg, rgs;
    bool on;
    u32x4 v[NB];

    __device__ __forceinline__ DyColumnSums(__amdgpu_buffer_rsrc_t ra_, int M_, int K_, int m0_, int BM_, int tn,
                                            int cw, int w, int nwc, int lane)
        : ra(ra_), M(M_), K(K_), m0(m0_), BM(BM_) {
        kb = tn * cw;
        on = kb < K;   // uniform over the block
        ncv = on ? (min(cw, K - kb) + 7) / 8 : 0;
        cvp = 1;
        while (cvp < ncv && cvp < 64) cvp <<= 1;
        const int t = w * 64 + lane;
        cvl = t % cvp;
        rg = t / cvp;
        rgs = nwc * 64 / cvp;
    }
    __device__ __forceinline__ void issue(int c0, int r0) {
        const int k = kb + (c0 + cvl) * 8;
        const bool kin = c0 + cvl < ncv && k < K;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int r = r0 + i * rgs, m = m0 + r;
            const bool ok = kin && r < BM && m < M;
            const uint32_t off = ok ? ((uint32_t)m * (uint32_t)K + (uint32_t)k) * 2u : kOOB;
            v[i] = __builtin_amdgcn_raw_buffer_load_b128(ra, (int)off, 0, 0);
        }
    }
    __device__ __forceinline__ void add(float (&acc)[8]) const {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                acc[2 * q] += __uint_as_float(v[i][q] << 16);
                acc[2 * q + 1] += __uint_as_float(v[i][q] & 0xffff0000u);
            }
    }
    __device__ __forceinline__ void run(bool issued, int w, int nwc, int tm, int lane, float *__restrict__ part) {
        if (!on) return;
        for (int c0 = 0; c0 < ncv; c0 += cvp) {
            float acc[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] = 0.f;
            for (int r0 = rg; r0 < BM; r0 += NB * rgs) {
                if (!(issued && c0 == 0 && r0 == rg)) issue(c0, r0);
                add(acc);
            }
            for (int sh = cvp; sh < 64; sh <<= 1)
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] += __shfl_xor(acc[e], sh);
            const int k = kb + (c0 + cvl) * 8;
            if (lane < cvp && c0 + cvl < ncv && k < K) {
                float *dst = part + (size_t)(tm * nwc + w) * K + k;
                *reinterpret_cast<floatx4 *>(dst) = floatx4{acc[0], acc[1], acc[2], acc[3]};
                *reinterpret_cast<floatx4 *>(dst + 4) = floatx4{acc[4], acc[5], acc[6], acc[7]};
            }
        }
    }
};

// KG k-groups of WR x WC waves: group g computes the whole block tile from
// the 16-k slices 2g and 2g+1 of every BK step (KG = 2), and the groups add
// their accumulators through LDS at the end.  Each wave then keeps a 64 x 64
// tile (one fragment read per MFMA) with two waves per SIMD.
template <int MODE, int BM, int BN, int WR, int WC, int STAGES, int KG = 1>
struct Cfg {
    static constexpr int NW = WR * WC * KG, NT = NW * 64;
    static constexpr bool A_KC = MODE != kWgrad;
    static constexpr bool B_KC = MODE == kFwd || MODE == kDgrad;   // kDgrad: W transposed to [C][R][S][K]
    static constexpr int A_BYTES = BM * BK * 2, B_BYTES = BN * BK * 2;
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
    static constexpr int LDS_BYTES = STAGES * STAGE_BYTES;
    // forward: the block's bias columns, loaded once into LDS past the stages
    // (one 16-byte load per lane of wave 0)
    static constexpr int BIAS_OFF = LDS_BYTES;
    // 1 KB load instructions per tile, and per wave: where the waves do not
    // divide A's (12 waves, 32 KB), the last waves' spare slots load zeros
    // into a dummy area past everything else, so that every wave issues the
    // same number of loads per stage (the vmcnt waits count them)
    static constexpr int A_INS = A_BYTES / 1024, B_INS = B_BYTES / 1024;
    static constexpr int NIA = (A_INS + NW - 1) / NW;
    static constexpr int NIB = B_INS / NW;
    static constexpr bool A_SPARE = NIA * NW != A_INS;
    static constexpr int DUMMY_OFF = LDS_BYTES + (MODE == kFwd ? 64 * 16 : 0);
    static constexpr int SMEM_BYTES = DUMMY_OFF + (A_SPARE ? 1024 : 0);
    static constexpr int WM = BM / WR, WN = BN / WC;
    static constexpr int TM = WM / 32, TN = WN / 32;   // 32x32 MFMA tiles per wave
    static constexpr int NSUB = BK / 16;               // 16-k slices per step
    static constexpr int EPI_PITCH = WN + 8;           // bf16 elements per staged row
    static constexpr int EPI_ROWS = 32;                // rows staged per pass
    static_assert(NIA >= 1 && NIB >= 1 && A_INS * 1024 == A_BYTES && NIB * NW * 1024 == B_BYTES, "load split");
    static_assert(!A_SPARE || (A_KC && MODE != kWgrad), "spare A load slots: k-contiguous A only");
    static_assert(TM >= 1 && TN >= 1 && WM % 32 == 0 && WN % 32 == 0, "wave tile");
    static_assert(NW * EPI_ROWS * EPI_PITCH * 2 <= LDS_BYTES, "epilogue staging must fit in LDS");
    static_assert(SMEM_BYTES <= 160 * 1024, "LDS");
    static_assert(BN * 2 <= 64 * 16, "bias columns fit the bias area");
    static_assert(KG == 1 || (KG == 2 && STAGES >= 3 && MODE != kWgrad), "k-groups: spread pipeline, no weight gradient");
    // block widths that are not a power of two (192, 288) only with both operands
    // k-contiguous: the transposing reads' slot swizzle needs 2^n slots a row
    static_assert((BN & (BN - 1)) == 0 || (A_KC && B_KC), "a 192- or 288-wide tile reads k-contiguous operands only");
    static_assert(KG == 1 || (WR * WC) * (WM / 32) * (WN / 32) * 16 * 64 * 4 <= LDS_BYTES, "k-group partials fit LDS");
};

// ------------------------------------------------------------------ host
constexpr int kCUs = 256;

struct Tile {
    const char *name;
    int bm, bn;       // block tile
    int wr, wc;       // wave grid (wr * wc waves of (bm/wr) x (bn/wc))
    int stages;       // LDS ring depth (BK = 64 per stage)
    int per_cu;       // blocks resident per CU
    float eff1;       // relative MFMA efficiency with one block on the CU
    float eff;        // ... with per_cu blocks on the CU
    int kg = 1;       // k-groups of wr x wc waves (the block has wr * wc * kg waves)
};

// ---------------------------------------------------------------- planner
// Estimated run time (microseconds) of a GEMM of M x N x K (z independent
// GEMMs of that bound, the stride phases of an input gradient) on tile t
// with the reduction split `splits` ways.  Per BK step a block takes the
// longer of its MFMA time (shared with the blocks resident on its CU) and
// the load latency its LDS ring can hide (STAGES - 1 tiles in flight); a
// wave of blocks also pays a fixed start/drain cost, every output byte is
// written once (fp32 partials when split), and a split adds the reduce pass.
// Constants come from kernel traces of the Linear and conv workloads: a
// 256 x 256 x 64 step of the 8-wave tile takes 1.5 us, a load round trip
// about 1 us.
constexpr double kUnitsPerUs = 2.33e6;   // bm*bn*k per us at relative efficiency 1
constexpr double kLoadUs = 1.0;          // HBM/L2 round trip of a stage's loads
constexpr double kWaveUs = 5.0;          // start + epilogue + drain of one wave of blocks
constexpr double kBytesPerUs = 6.0e6;    // streamed HBM bytes per us
constexpr double kLaunchUs = 3.0;

inline double est_us(const Tile &t, long M, long N, long K, int z, int splits) {
    const long tiles = ((M + t.bm - 1) / t.bm) * ((N + t.bn - 1) / t.bn) * z;
    const long blocks = tiles * splits;
    const long conc = (long)kCUs * t.per_cu;
    const long waves = (blocks + conc - 1) / conc;
    const long resident = std::min<long>(t.per_cu, (blocks + kCUs - 1) / kCUs);
    const long kper = ((K + splits - 1) / splits + BK - 1) / BK * BK;
    const double eff = resident > 1 ? t.eff : t.eff1;
    const double t_mfma = (double)resident * t.bm * t.bn * BK / (kUnitsPerUs * eff);
    const double t_lat = kLoadUs / (t.stages - 1);
    const double step = std::max(t_mfma, t_lat);
    const double out_elems = (double)M * N * z;
    double us = waves * ((double)(kper / BK) * step + kWaveUs) + out_elems * (splits > 1 ? 4.0 * splits : 2.0) / kBytesPerUs;
    if (splits > 1) us += kLaunchUs + out_elems * (4.0 * splits + 2.0) / kBytesPerUs;
    return us;
}

}  // namespace g2
}  // namespace ms
