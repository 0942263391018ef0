// Sums over a row's softmax as a lane forms them, under a temperature and with masked logits: shared by the kernels behind
// ulorl_token_topk and ulorl_distill_*.
#ifndef ULORL_ROW_SUMS_HPP
#define ULORL_ROW_SUMS_HPP

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "logits_stream.hpp"

namespace ulorl_detail {

// Logits at or below -9e29 are masked (the filler of short vectors is one of them).  A lane's running maximum starts a little
// above: by so much that the terms of masked logits are 0 against it (the rounding of m scale is 1e23 there).
constexpr float kFloor = -8.99e29f;

// Per-lane statistics of the stream; x = z scale in log2 units, relative to the lane's maximum.
// S + Sc: sum 2^(x - mL), its rounding residuals carried in Sc; T + Tc: sum 2^(x - mL) (x - mL), likewise.
struct Lane {
    float m, mL, S, Sc, T, Tc;
};

// The larger, not-a-number if one is (a row that holds one is refused at its end): one instruction for three values, and none to
// quiet what came out of bit operations, which fmaxf needs.
__device__ __forceinline__ float larger(float x, float y) { return __builtin_elementwise_maximum(x, y); }

// WEIGHTED: T is wanted.  Its terms are added in chains of eight fused steps, and a batch of up to four of these to the running sum with
// a residual: one chain over a row would round the same way again and again where terms are alike (the entropy off by 3e-5 at
// 600 terms a lane, 1e-3 at 30000).
template <int COUNT, bool WEIGHTED = true>
__device__ __forceinline__ void absorb_scaled(const float* f, float cm, float scale, Lane& a)
{
    const float mn = larger(a.m, cm);
    const float mLn = mn * scale;
    const float d = a.mL - mLn;
    const float sc = fast_exp2(d);
    const float T = WEIGHTED ? sc * fmaf(d, a.S, a.T) : 0.0f, Tc = WEIGHTED ? sc * fmaf(d, a.Sc, a.Tc) : 0.0f;
    const float S = sc * a.S, Sc = sc * a.Sc;
    // the terms as a tree over neighbours: a sum of eight is done before the next eight terms are formed
    float e[COUNT / 8 > 0 ? COUNT / 8 : 1];
    float weighted = 0.0f;
#pragma unroll
    for (int c = 0; c < COUNT; c += 8) {
        constexpr int W = COUNT < 8 ? COUNT : 8;
        float p[W], chain = 0.0f;
#pragma unroll
        for (int k = 0; k < W; ++k) {
            const float x = fmaf(f[c + k], scale, -mLn);
            p[k] = fast_exp2(x);
            if constexpr (WEIGHTED) chain = k == 0 ? p[k] * x : fmaf(p[k], x, chain);
        }
        if constexpr (WEIGHTED) weighted = c == 0 ? chain : weighted + chain;
#pragma unroll
        for (int w = W / 2; w >= 1; w >>= 1)
#pragma unroll
            for (int k = 0; k < w; ++k) p[k] += p[k + w];
        e[c / 8] = p[0];
    }
#pragma unroll
    for (int w = COUNT / 16; w >= 1; w >>= 1)
#pragma unroll
        for (int k = 0; k < w; ++k) e[k] += e[k + w];
    const float t = S + e[0];                   // TwoSum: the residual of a small term against a sum near 1 is kept
    const float bv = t - S;
    a.Sc = Sc + ((S - (t - bv)) + (e[0] - bv));
    a.S = t;
    if constexpr (WEIGHTED) {
        // The running sum is the larger addend, so this is its residual; where it is not (at the beginning, after a new maximum) the sum
        // at least doubles, and what is missed is a rounding of it once.
        a.T = T + weighted;
        a.Tc = Tc + (weighted - (a.T - T));
    }
    a.m = mn;
    a.mL = mLn;
}

template <int CTRL>
__device__ __forceinline__ float from_lane(float x)
{
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140, kRotate8 = 0x128;      // 7 - lane in each 8, 15 - lane in each 16
__device__ __forceinline__ float wave_max(float x)
{
    x = larger(x, from_lane<kXor1>(x));
    x = larger(x, from_lane<kXor2>(x));
    x = larger(x, from_lane<kMirror8>(x));
    x = larger(x, from_lane<kMirror16>(x));
    const int i = __float_as_int(x);
    return larger(larger(__int_as_float(__builtin_amdgcn_readlane(i, 0)), __int_as_float(__builtin_amdgcn_readlane(i, 16))),
                  larger(__int_as_float(__builtin_amdgcn_readlane(i, 32)), __int_as_float(__builtin_amdgcn_readlane(i, 48))));
}

// The stride to check and to use: a lone row has none, whatever its caller's tensor says (a column taken as a row says 1).
inline int64_t row_stride_of(int64_t N, int64_t V, int64_t row_stride)
{
    return N == 1 && V > 0 && V <= 0x7fffffffLL ? (V + 7) / 8 * 8 : row_stride;
}

// Vectors that hold a row.  V + kPerVec - 1 would pass 32 bits at the largest V.
template <class Tr>
constexpr int vectors_of(int32_t V)
{
    return (V - 1) / Tr::kPerVec + 1;
}

// A vector of a row; behind the row's end, and where V ends inside a vector, the filler.
template <class Tr>
__device__ __forceinline__ u32x4 load_vector(const typename Tr::elem* rowp, int32_t V, int i)
{
    constexpr int E = Tr::kPerVec;
    const int nvec = V / E;
    if (i < nvec) return load_stream(reinterpret_cast<const u32x4*>(rowp) + i);
    u32x4 v = Tr::filler();
    if (i == nvec) {
        for (int e = 0; e < V - nvec * E; ++e) {
            if constexpr (E == 8) {
                const uint32_t b = rowp[i * E + e];
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    if (w == (e >> 1)) v[w] = (e & 1) ? (v[w] & 0xffffu) | (b << 16) : (v[w] & 0xffff0000u) | b;
            } else {
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    if (w == e) v[w] = __float_as_uint(rowp[i * E + e]);
            }
        }
    }
    return v;
}

// e^x and ln x in 64 bits, to a few units of the last place, in a third of the instructions of the library's functions: they are
// most of what finishing a row costs.  x = (n + f) ln 2 with |f| <= 1/2, and the Taylor series of 2^f up to f^12 (the next term is below
// 2e-16).  exp64: not-a-number stays, below e^-1100 is 0.
__device__ __forceinline__ double exp64(double x)
{
    x = x < -1100.0 ? -1100.0 : x;
    // x log2(e) in two parts: the rounding of one product would be |x| units of the last place
    const double hi = x * 1.4426950408889634, n = rint(hi);
    const double f = fma(x, 1.4426950408889634, -n) + x * 2.0355273740931033e-17;
    double p = 2.5678435993488196e-11;
    p = fma(p, f, 4.44553827187081e-10);
    p = fma(p, f, 7.054911620801121e-09);
    p = fma(p, f, 1.0178086009239696e-07);
    p = fma(p, f, 1.3215486790144305e-06);
    p = fma(p, f, 1.5252733804059838e-05);
    p = fma(p, f, 0.00015403530393381606);
    p = fma(p, f, 0.0013333558146428441);
    p = fma(p, f, 0.009618129107628477);
    p = fma(p, f, 0.055504108664821576);
    p = fma(p, f, 0.2402265069591007);
    p = fma(p, f, 0.6931471805599453);
    p = fma(p, f, 1.0);
    return ldexp(p, (int)n);
}
// A step of second order from the 32-bit logarithm: its error (1e-6 where the logarithm is 12) cubed.  For x within the range of 32 bits.
__device__ __forceinline__ double log64(double x)
{
    const double l = (double)__builtin_amdgcn_logf((float)x) * 0.69314718055994530942;
    const double r = fma(x, exp64(-l), -1.0);       // ln(1 + r) is missing
    return l + fma(-0.5 * r, r, r);
}

}  // namespace ulorl_detail

#endif
