// For the kernels of the transformer layers: vectors of rows of any width and
// alignment, the joining of softmax statistics, and the activations of the gated
// linear unit with their derivatives.
#pragma once

#include "common.h"
#include "../device.h"

namespace ms {

// A row's 16-byte vector at column c; a last, incomplete one element by element.
template <typename T> struct Loose;   // 16 bytes at the alignment of an element
template <> struct Loose<float> { typedef u32x4 type __attribute__((aligned(4))); };
template <> struct Loose<bf16> { typedef u32x4 type __attribute__((aligned(2))); };

template <typename T>
__device__ __forceinline__ Vec16<T> load_vec(const T *__restrict__ row, int c, int D) {
    constexpr int V = Vec16<T>::N;
    Vec16<T> v;
    if (c + V <= D) {
        v.u = *reinterpret_cast<const typename Loose<T>::type *>(row + c);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v.e[e] = c + e < D ? row[c + e] : (T)0.f;
    }
    return v;
}

template <typename T>
__device__ __forceinline__ void store_vec(T *__restrict__ row, int c, int D, const Vec16<T> &v) {
    constexpr int V = Vec16<T>::N;
    if (c + V <= D) {
        *reinterpret_cast<typename Loose<T>::type *>(row + c) = v.u;
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e < D) row[c + e] = v.e[e];
    }
}

// fp32 rounded to its leading 24 bits (to nearest even; NaN stays one), in the low ones.
__device__ __forceinline__ uint32_t to_f24(float v) {
    const uint32_t u = __float_as_uint(v);
    return v != v ? 0x7fc000u : (u + 0x7fu + ((u >> 8) & 1u)) >> 8;
}

typedef float floatx2 __attribute__((ext_vector_type(2)));

// How many ways to split the steps of a contraction whose rows are known on the
// device only: rounds of blocks over the card, each its share of the steps and some
// five steps' worth of beginning and end, against the partials' traffic.
struct SplitRule {
    int bm, ntn, steps, slots, most;   // tile rows, column tiles, steps, blocks at once, splits at most
    float step_us, row_us;             // a step of one round; a row of partials
    __host__ __device__ __forceinline__ int splits(int rows) const {
        const int tiles = (rows + bm - 1) / bm * ntn;
        int best = 1;
        float us = INFINITY;
        for (int s = 1; s <= most; ++s) {
            const int rounds = (tiles * s + slots - 1) / slots;
            const float t = (float)rounds * ((float)((steps + s - 1) / s) + 5.f) * step_us + (float)s * (float)rows * row_us;
            if (t < us) {
                us = t;
                best = s;
            }
        }
        return best;
    }
};

constexpr float kLog2e = 1.44269504088896341f;

// exp(v - m).  The difference first: with m the larger one it is a finite number
// or minus infinity, whatever the sizes of both (v log2(e) - m log2(e) is not).
__device__ __forceinline__ float exp_below(float v, float m) { return __builtin_amdgcn_exp2f((v - m) * kLog2e); }

// (m, s) stands for s exp(m), m the running maximum: the sum of two.  A maximum of
// minus infinity (nothing yet) comes with s = 0; a NaN stays in s.
__device__ __forceinline__ floatx2 join_lse(floatx2 a, floatx2 b) {
    const float m = fmaxf(a.x, b.x);
    const float sa = a.x == m ? a.y : a.y * exp_below(a.x, m);
    const float sb = b.x == m ? b.y : b.y * exp_below(b.x, m);
    return floatx2{m, sa + sb};
}

// A row's loss from the statistics a of the words other than its target (as join_lse()'s)
// and the target's logit z: d, the logarithm of the odds against the target, is a sum of
// parts with small errors, and neither the loss log(1 + exp(d)) nor what the target's
// probability lacks of 1, 1 / (1 + exp(-d)), is a difference of numbers near 1: both
// keep their leading digits however small they are.  NaN where the row has no
// distribution: no finite logit, an infinite one, or (z NaN) no such word.
struct RowLoss {
    float others;   // log of the sum of the other words' exponentials: -inf where there is none
    float loss;
    float ct;       // the target's entry of dz: minus what its probability lacks of 1
};
__device__ __forceinline__ float target_entry(float d) { return -1.f / (1.f + expf(-d)); }
__device__ __forceinline__ RowLoss row_loss(floatx2 a, float z) {
    const float ls = logf(a.y);
    // (the difference first: it is exact where both are large)
    const float d = z == INFINITY ? NAN : (a.x - z) + ls;
    RowLoss r;
    r.others = d != d ? NAN : a.x + ls;
    r.loss = fmaxf(d, 0.f) + log1pf(expf(-fabsf(d)));
    r.ct = target_entry(d);
    return r;
}

// Columns of one statistic and reference of exponentials that are kept.
constexpr int kProbCols = 64;

// The reference r of the kept exponentials exp(v - r) of values whose largest is
// top: a multiple of 64 ln 2 that leaves that one between 2^-16 and 2^48.  Parts of
// a row nearly always agree on it; where they do not, their factor is a power of
// two, by which the exponentials, rounded to bf16 already, are multiplied without
// another error.  Far from zero, where such multiples are not exact, top itself.
__device__ __forceinline__ float prob_ref(float top) {
    constexpr float kStep = 44.3614195558364998f;
    return fabsf(top) < 1e6f ? kStep * floorf((top + 11.f) * (1.f / kStep)) : top;
}

namespace act {

// FAST: on the hardware's exponential and reciprocal (each within some 2 units
// in 2^-24), for results that are rounded to bf16; else the library's.
template <bool FAST>
__device__ __forceinline__ float exp_(float v) {
    return FAST ? __builtin_amdgcn_exp2f(v * kLog2e) : expf(v);
}
template <bool FAST>
__device__ __forceinline__ float rcp_(float v) {
    return FAST ? __builtin_amdgcn_rcpf(v) : 1.f / v;
}
template <bool FAST>
__device__ __forceinline__ float sigmoid(float z) { return rcp_<FAST>(1.f + exp_<FAST>(-z)); }

// The normal distribution's cumulative probability and density.  FAST: the tail
// from Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26
// (within 1.5e-7), taken on the negative side so that small results do not
// come from a difference.
template <bool FAST>
__device__ __forceinline__ void normal(float z, float &cdf, float &pdf) {
    const float e = exp_<FAST>(-0.5f * z * z);
    pdf = 0.398942280401432678f * e;
    if constexpr (FAST) {
        const float u = fabsf(z) * 0.707106781186547524f;
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f, u, 1.f));
        float p = __builtin_fmaf(1.061405429f, t, -1.453152027f);
        p = __builtin_fmaf(p, t, 1.421413741f);
        p = __builtin_fmaf(p, t, -0.284496736f);
        p = __builtin_fmaf(p, t, 0.254829592f);
        const float tail = 0.5f * p * t * e;
        cdf = z < 0.f ? tail : 1.f - tail;
    } else {
        cdf = 0.5f * erfcf(-z * 0.707106781186547524f);
    }
}

// a = act(z), d = act'(z)
template <bool FAST>
__device__ __forceinline__ void both(int kind, float z, float &a, float &d) {
    switch (kind) {
    case kActSilu: {
        const float s = sigmoid<FAST>(z);
        a = z * s;
        d = __builtin_fmaf(a, 1.f - s, s);
        return;
    }
    case kActGelu: {
        float cdf, pdf;
        normal<FAST>(z, cdf, pdf);
        a = z * cdf;
        d = __builtin_fmaf(z, pdf, cdf);
        return;
    }
    case kActGeluTanh: {   // 0.5 (1 + tanh(p)) = sigmoid(2 p), p = sqrt(2 / pi) (z + 0.044715 z^3)
        const float z2 = z * z;
        const float s = sigmoid<FAST>(1.59576912160573071f * z * __builtin_fmaf(0.044715f, z2, 1.f));
        a = z * s;
        d = __builtin_fmaf(a * (1.f - s), 1.59576912160573071f * __builtin_fmaf(0.134145f, z2, 1.f), s);
        return;
    }
    case kActRelu:
        a = z < 0.f ? 0.f : z;
        d = z > 0.f ? 1.f : 0.f;
        return;
    default: {   // kActSigmoid
        a = sigmoid<FAST>(z);
        d = a * (1.f - a);
        return;
    }
    }
}

template <bool FAST>
__device__ __forceinline__ float value(int kind, float z) {
    float a, d;
    both<FAST>(kind, z, a, d);
    return a;
}

}  // namespace act
}  // namespace ms
