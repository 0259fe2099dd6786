"""The logarithm and the power of the beam selection (`csrc/lla_beam_math.cuh`), compiled for the host, against libm in
64 and 80 bits over their ranges, at the bounds that their comments state."""
import os
import shutil
import subprocess
import tempfile

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_15456_gb300", "csrc")

CHECK = r"""
#include <cfloat>
#include <cmath>
#include <cstdio>

#include "lla_beam_math.cuh"

typedef long double ld;  // 64 bits or more, whose own error is far below the bounds

static int fails = 0;
static void check(const char *what, double x, double y, ld got, ld want, ld bound, ld *worst) {
    const ld off = fabsl(got - want);
    if (off > *worst) *worst = off;
    if (!(off < bound) && fails++ < 10) std::printf("%s at %.17g %.17g: %.17Lg, not %.17Lg\n", what, x, y, got, want);
}

static uint64_t state = 88172645463325252ull;
static double uniform() {  // Marsaglia's xorshift
    state ^= state << 13; state ^= state >> 7; state ^= state << 17;
    return static_cast<double>(state >> 11) / 9007199254740992.0;
}

int main() {
    using namespace lla;
    ld w_sum = 0, w_log = 0, w_exp = 0, w_pow = 0;
    // log (hi + lo): every table entry's ends and inside, exponents over the normal range, lo on both sides
    for (int e = -126; e <= 127; e += (e > -10 && e < 40 ? 1 : 9))
        for (int k = 0; k < 4096; ++k) {
            const uint32_t frac = k < 2048 ? (k >> 6 << 18) + (k % 64 < 32 ? k % 64 : 0x40000 - 64 + k % 64) : static_cast<uint32_t>(uniform() * 8388608);
            const float hi = bits_of<float>((static_cast<uint32_t>(e + 127) << 23) | (frac & 0x7fffff));
            for (float part : {0.f, 1.f, -1.f, 0.37f, 0x1p-9f}) {
                const float lo = hi * part * 0x1p-11f;
                if (fabsf(lo) < FLT_MIN && lo != 0) continue;
                check("log_sum", hi, lo, log_sum(hi, lo, log_table()), logl(static_cast<ld>(hi) + lo), 4e-9L, &w_sum);
            }
        }
    // log n of whole numbers, and around the switch of the exponent
    for (int64_t n = 1; n < (1 << 16); ++n) check("log_of", n, 0, log_of(static_cast<double>(n)), logl(static_cast<ld>(n)), 1e-12L, &w_log);
    for (int i = 0; i < 2000000; ++i) {
        const double n = floor(exp(uniform() * 21.5)) ;
        if (n >= 1 && n <= 2147483648.0) check("log_of", n, 0, log_of(n), logl(static_cast<ld>(n)), 1e-12L, &w_log);
    }
    for (int b = 1; b <= 31; ++b)
        for (double c : {1.0, 1.4142135623730951, 0.7071067811865476})
            for (int d = -2; d <= 2; ++d) {
                const double n = floor(ldexp(c, b)) + d;
                if (n >= 1) check("log_of", n, 0, log_of(n), logl(static_cast<ld>(n)), 1e-12L, &w_log);
            }
    // exp x, and n^-alpha
    for (int i = 0; i < 4000000; ++i) {
        const double x = i < 2000 ? (i - 1000) * 0.4 : (uniform() * 2 - 1) * (i % 2 ? 400 : 1);
        check("exp_of", x, 0, exp_of(x) / expl(x), 1, 1e-13L, &w_exp);
    }
    for (int k = -577; k <= 577; ++k)  // the ends of the reduction
        for (int d = -3; d <= 3; ++d) {
            const double x = (k + 0.5) * 0.69314718055994531 * (1 + d * 1e-16);
            if (fabs(x) <= 400) check("exp_of", x, 0, exp_of(x) / expl(x), 1, 1e-13L, &w_exp);
        }
    for (int i = 0; i < 2000000; ++i) {  // of itself: 16 times the logarithm's bound, and the exponential's
        const double n = floor(exp(uniform() * 21.48)), alpha = (uniform() * 2 - 1) * 16;
        if (n >= 1) check("power", n, alpha, exp_of(-alpha * log_of(n)) / powl(n, -static_cast<ld>(alpha)), 1, 1.7e-11L, &w_pow);
    }
    std::printf("worst: log_sum %.2Lg, log_of %.2Lg, exp_of %.2Lg, power %.2Lg\n%s\n", w_sum, w_log, w_exp, w_pow, fails ? "FAILED" : "ok");
    return fails ? 1 : 0;
}
"""


@pytest.mark.parametrize("contract", ["off", "fast"])
def test_bounds(contract):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("nvcc not available")
    with tempfile.TemporaryDirectory() as tmp:
        src, exe = os.path.join(tmp, "beam_math.cu"), os.path.join(tmp, "beam_math")
        with open(src, "w") as f:
            f.write(CHECK)
        r = subprocess.run([nvcc, "-gencode", "arch=compute_103a,code=sm_103a", "-O2", "-std=c++17", "-Xcompiler", f"-ffp-contract={contract}",
                            "-I", CSRC, "-I", os.path.join(ROOT, "include"), src, "-o", exe], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
        print(r.stdout)
        assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stdout[-2000:]
