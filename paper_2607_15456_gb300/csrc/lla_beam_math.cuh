// lla_beam_math.cuh -- the logarithm of a sum and the power of the length penalty (lla_beam.cu), in few fp64 operations: one
// takes about 100 cycles, and these are on the way of every call.  They compile for the host too, where their
// bounds are tested.
#pragma once

#include <math.h>
#include <stdint.h>
#include <string.h>

#include <cmath>

namespace lla {
namespace {

template <typename To, typename From>
__host__ __device__ __forceinline__ To bits_of(From x) {
    static_assert(sizeof(To) == sizeof(From), "the same bits");
    To y;
    memcpy(&y, &x, sizeof(y));
    return y;
}

// For a number in the i-th of 32 parts of [1, 2): a float r near its reciprocal, and -log r.
struct LogTable {
    float r[32];
    double minus_log[32];
};
inline const LogTable &log_table() {
    static const LogTable t = [] {
        LogTable x;
        for (int i = 0; i < 32; ++i) {
            x.r[i] = static_cast<float>(1.0 / (1.0 + (i + 0.5) / 32));
            x.minus_log[i] = -std::log(static_cast<double>(x.r[i]));
        }
        return x;
    }();
    return t;
}

// log (hi + lo) of a normal positive hi, |lo| <= 2^-11 hi (of another: some number), off by less than 4e-9.  (lo is the sum of the
// rounding errors of at most 4096 tiles, each half a step of hi at most.)  By a table, as in P. T. P. Tang, "Table-driven
// implementation of the logarithm function" (1990): with hi + lo = 2^e m (1 + lo / hi), and that m r (1 + lo / hi) = 1 + u, |u| <= 1/62,
// it is e log 2 - log r + log (1 + u), the last a short series in fp32.
__host__ __device__ __forceinline__ double log_sum(float hi, float lo, const LogTable &t) {
    const uint32_t b = bits_of<uint32_t>(hi);
    const int e = static_cast<int>(b >> 23 & 255) - 127, i = b >> 18 & 31;
    const float m = bits_of<float>((b & 0x7fffffu) | 0x3f800000u), r = t.r[i];
    const float u = fmaf(lo / hi, m * r, fmaf(m, r, -1.f));  // m r (1 + lo / hi) - 1
    const float p = u * fmaf(u, fmaf(u, fmaf(u, fmaf(u, 0.2f, -0.25f), 1.f / 3.f), -0.5f), 1.f);
    return static_cast<double>(e) * 0.693147180559945309 + (t.minus_log[i] + static_cast<double>(p));
}

// log n of n >= 1, off by less than 1e-12: n = 2^e m with m between sqrt(1/2) and sqrt(2), and log m = 2 atanh t =
// 2 (t + t^3 / 3 + ... + t^13 / 13), t = (m - 1) / (m + 1), |t| <= 0.172, the series in pairs (Estrin).
__host__ __device__ __forceinline__ double log_of(double x) {
    const int64_t u = bits_of<int64_t>(x);
    const int64_t half = 0x3fe6a09e667f3bcdll;  // sqrt(1/2)
    const int e = static_cast<int>((u - half) >> 52);
    const double m = bits_of<double>(u - (static_cast<int64_t>(e) << 52));
    const double d = m + 1.0;
    const double r0 = static_cast<double>(1.f / static_cast<float>(d));
    const double r = r0 * fma(-d, r0, 2.0);  // one step of Newton: 2^-23 squared
    const double t = (m - 1.0) * r, w = t * t, w2 = w * w;
    const double a = fma(w, 1.0 / 3.0, 1.0), b = fma(w, 1.0 / 7.0, 1.0 / 5.0), c = fma(w, 1.0 / 11.0, 1.0 / 9.0);
    const double p = fma(w2, fma(w2, fma(w2, 1.0 / 13.0, c), b), a);
    return fma(static_cast<double>(e), 0.693147180559945309, 2.0 * t * p);
}

// exp x for |x| <= 400, off by less than 1e-13 of itself: x = k log 2 + r, |r| <= 0.347, and the series of exp r to
// r^13, in pairs.
__host__ __device__ __forceinline__ double exp_of(double x) {
    const double k = rint(x * 1.4426950408889634);
    const double r = fma(-k, 2.3190468138462996e-17, fma(-k, 0.6931471805599453, x));  // log 2 as a sum of two
    const double r2 = r * r, r4 = r2 * r2, r8 = r4 * r4;
    const double p01 = 1.0 + r, p23 = fma(r, 1.0 / 6.0, 0.5), p45 = fma(r, 1.0 / 120.0, 1.0 / 24.0);
    const double p67 = fma(r, 1.0 / 5040.0, 1.0 / 720.0), p89 = fma(r, 1.0 / 362880.0, 1.0 / 40320.0);
    const double pab = fma(r, 1.0 / 39916800.0, 1.0 / 3628800.0), pcd = fma(r, 1.0 / 6227020800.0, 1.0 / 479001600.0);
    const double p03 = fma(r2, p23, p01), p47 = fma(r2, p67, p45), p8b = fma(r2, pab, p89);
    const double p = fma(r8, fma(r4, pcd, p8b), fma(r4, p47, p03));
    return p * bits_of<double>((static_cast<int64_t>(k) + 1023) << 52);
}

}  // namespace
}  // namespace lla
