"""The exponentials that pdb_verify decides on (exp_two and FastTerm in verify.cu), taken from the source and compiled for the host, against the C library's
in extended precision: a rounding here and there decides whether a token is the right one, so their error bounds are the kernel's."""
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1508_00703_gb300", "csrc")

SHIM = r"""
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <random>
struct float2 { float x, y; };
#define __device__
#define __forceinline__ inline
static float __fsub_rn(float a, float b) { return a - b; }
static float __fadd_rn(float a, float b) { return a + b; }
static float __fmul_rn(float a, float b) { return a * b; }
static float __fdiv_rn(float a, float b) { return a / b; }
static float __fmaf_rn(float a, float b, float c) { return fmaf(a, b, c); }
static float __ll2float_rn(int64_t x) { return (float)x; }
static int64_t __float2ll_rn(float x) { return llrintf(x); }
static int __float2int_rn(float x) { return (int)lrintf(x); }
static int __float_as_int(float f) { int i; memcpy(&i, &f, 4); return i; }
static uint32_t __float_as_uint(float f) { uint32_t i; memcpy(&i, &f, 4); return i; }
static float __int_as_float(int i) { float f; memcpy(&f, &i, 4); return f; }
static float __uint_as_float(uint32_t i) { float f; memcpy(&f, &i, 4); return f; }
static uint64_t pair(float a, float b) { return (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a); }
static void unpair(uint64_t p, float &a, float &b) { a = __uint_as_float((uint32_t)p), b = __uint_as_float((uint32_t)(p >> 32)); }
template <typename F> static uint64_t each(uint64_t a, uint64_t b, F f)
{
    float x[2], y[2];
    unpair(a, x[0], x[1]), unpair(b, y[0], y[1]);
    return pair(f(x[0], y[0]), f(x[1], y[1]));
}
static uint64_t add2(uint64_t a, uint64_t b) { return each(a, b, [](float x, float y) { return x + y; }); }
static uint64_t mul2(uint64_t a, uint64_t b) { return each(a, b, [](float x, float y) { return x * y; }); }
static uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    float x[2], y[2], z[2];
    unpair(a, x[0], x[1]), unpair(b, y[0], y[1]), unpair(c, z[0], z[1]);
    return pair(fmaf(x[0], y[0], z[0]), fmaf(x[1], y[1], z[1]));
}
constexpr float LOG2E = 1.44269504088896340736f;
"""

MAIN = r"""
int main()
{
    static float2 table[256], fast[STEPS];
    for (int i = 0; i < 256; ++i) table[i] = {EXP2_TABLE.hi[i], EXP2_TABLE.lo[i]};
    for (int i = 0; i < STEPS; ++i) fast[i] = {FAST_TABLE.hi[i], FAST_TABLE.lo[i]};
    std::mt19937_64 g(1);
    std::uniform_real_distribution<double> U(0, 1);
    double rel = 0, absolute = 0, fast_rel = 0, units_off = 0, whole_off = 0;
    for (int k = 0; k < 400000; ++k) {
        const float m = (float)((U(g) - 0.5) * (k % 3 ? 40 : 400)), scale = k % 2 ? 1.0f : (float)(0.05 + U(g) * (k % 3 ? 3 : 1));
        float z = m - (float)(U(g) * (k % 7 ? 30 : 1e-3) / scale);
        if (k % 11 == 0) z *= 1e-3f;
        if (!(z <= m)) z = m;
        const long double x = ((long double)z - (long double)m) * (long double)scale, e = expl(x);
        if (x > -40) {
            const Two t = exp_two(z, m, scale, table);
            const double off = (double)fabsl((long double)t.hi + (long double)t.lo - e);
            if (x > -12) rel = fmax(rel, off / (double)e);
            Units one;
            one.add(t);
            whole_off = fmax(whole_off, (double)fabsl(ldexpl((long double)one.whole(), -46) - (long double)t.hi - (long double)t.lo));
            if (fabsf(t.lo) > t.hi * 0x1p-24f) units_off = 4;
            absolute = fmax(absolute, off);
        }
        if (fabsf(m * scale * LOG2E) >= REACH || x < -40) continue;
        // what all tokens of a row share falls out: against the term at m itself
        const int down = k % 5;
        const FastTerm term(m, scale, down, m, scale, 0);
        float value[2], one[2];
        int high[2], low[2], h1[2], l1[2];
        term(z, z, fast, value, high, low);
        term(m, m, fast, one, h1, l1);
        for (int i = 0; i < 2; ++i) {
            const long double w = (long double)units(high[i] - HIGH0, low[i] - LOW0), w1 = (long double)units(h1[i] - HIGH0, l1[i] - LOW0);
            const long double size = ldexpl(1.0L, 44 - (i ? 0 : down));
            // a unit for the roundings of the two, and what is relative
            const double off = (double)fabsl(w / w1 - e);
            if (off * (double)size > 1.5) fast_rel = fmax(fast_rel, (off - 1.5 / (double)size) / (double)e);
            if ((double)fabsl((long double)value[i] * ldexpl(1.0L, 22) - w) > (double)w * 0x1p-23 + 1) units_off = 1;
        }
    }
    for (float masked : {-INFINITY, -3e38f, -1000.0f}) {
        const FastTerm term(3.0f, 1.0f, 0, 3.0f, 1.0f, 2);
        float value[2];
        int high[2], low[2];
        term(masked, masked, fast, value, high, low);
        if (units(high[0] - HIGH0, low[0] - LOW0) || units(high[1] - HIGH0, low[1] - LOW0)) units_off = 2;
        if (exp_two(masked, 3.0f, 1.0f, table).hi != 0.0f) units_off = 3;
    }
    const Two inv = inverse_of({3.0f, 1e-9f}), sum = two_of(((int64_t)5 << 23) + 7, -3);
    const double inv_off = fabs(((double)inv.hi + (double)inv.lo) * (3.0 + (double)1e-9f) - 1.0);
    const double sum_off = fabs((double)sum.hi + (double)sum.lo - (5.0 + 7 * 0x1p-23 - 3 * 0x1p-46));
    // a row's sum as the kernel forms it
    double row_off = 0;
    for (int row = 0; row < 20; ++row) {
        int64_t high = 0, low = 0;
        long double all = 1;
        Units one;
        one.add(exp_two(3.0f, 3.0f, 1.0f, table));
        high += one.high, low += one.low;
        for (int k = 0; k < 30000; ++k) {
            const float z = (float)(3.0 - U(g) * (row + 1));
            Units more;
            more.add(exp_two(z, 3.0f, 1.0f, table));
            high += more.high, low += more.low, all += expl((long double)z - 3);
        }
        const Two of_row = two_of(high, low);
        row_off = fmax(row_off, fabs((double)(((long double)of_row.hi + (long double)of_row.lo) / all - 1)));
    }
    printf("%.17g %.17g %.17g %.17g %.17g %.17g %.17g %.17g\n", rel, absolute, fast_rel, units_off, inv_off, sum_off, whole_off, row_off);
}
"""


@pytest.fixture(scope="module")
def measured(tmp_path_factory):
    text = open(os.path.join(CSRC, "verify.cu")).read()
    code = text[text.index("constexpr double LN2_D"):text.index("// How far from its token's borders")]
    code = re.sub(r"__device__ const", "static const", code)
    d = tmp_path_factory.mktemp("terms")
    (d / "terms.cpp").write_text(SHIM + code + MAIN)
    subprocess.run(["g++", "-std=c++17", "-O2", "-ffp-contract=off", "-w", str(d / "terms.cpp"), "-o", str(d / "terms")], check=True)
    out = subprocess.run([str(d / "terms")], check=True, capture_output=True, text=True).stdout
    return [float(x) for x in out.split()]


def test_exp_two(measured):
    rel, absolute = measured[:2]
    assert rel <= 2.0 ** -40.5                       # where a row's mass can lie
    assert absolute <= 2.0 ** -42                    # of the largest term, anywhere


def test_fast_term(measured):
    fast_rel, units_off = measured[2:4]
    assert fast_rel <= 2.0 ** -31.5
    assert units_off == 0                            # value and whole numbers agree; masked tokens weigh nothing


def test_sums_and_reciprocals(measured):
    assert measured[4] <= 2.0 ** -45 and measured[5] <= 2.0 ** -46


def test_units(measured):
    # a rounding to units, and one of what is left (below 2^-23) as a float; so is a row's sum as good as its terms
    assert measured[6] <= 2.0 ** -47 + 2.0 ** -48
    assert measured[7] <= 2.0 ** -40.5
