"""The whole numbers that pdb_verify's exact draws are summed as (Units, Weight, share_of_total in verify.cu), taken from the source and compiled for the
host: rows whose largest term stands beside a long tail of equal ones, whose roundings all go one way.  A term good to 2^-40 of itself moves
a border of the tail by at most 2^-40 of the tail, 2^-23 of a token for 128,000; numbers nearer to a border than four times that are left out."""
import os
import re
import subprocess

import pytest

from tests.test_verify_terms import CSRC, SHIM

MAIN = r"""
#include <vector>
static float2 table[256];
constexpr int N = 127999;
int main()
{
    for (int i = 0; i < 256; ++i) table[i] = {EXP2_TABLE.hi[i], EXP2_TABLE.lo[i]};
    std::mt19937_64 g(1);
    std::uniform_real_distribution<double> U(0, 1);
    double sum_off = 0, rel = 0, weight_off = 0;
    long wrong = 0, seen = 0;
    for (float gap : {0.0f, 5.0f, 16.0f, 18.0f, 20.0f, 22.0f, 26.0f, 30.0f, 34.0f, 40.0f}) {
        const long double t = expl(-(long double)gap), exact = 1 + N * t;
        // a row's sum as the kernel forms it
        int64_t whole = 0, rest = 0;
        Units one, more;
        one.add(exp_two(3.0f, 3.0f, 1.0f, table));
        more.add(exp_two(3.0f - gap, 3.0f, 1.0f, table));
        whole = one.whole() + N * more.whole(), rest = one.rest() + N * more.rest();
        const Two sum = two_of(wide(whole, rest));
        sum_off = fmax(sum_off, (double)fabsl(((long double)sum.hi + (long double)sum.lo) / exact - 1));
        const Two inv = inverse_of(sum);
        sum_off = fmax(sum_off, (double)fabsl(((long double)inv.hi + (long double)inv.lo) * exact - 1));
        // draws: the head before the tail, and behind it.  The weights' sum is 1 at most (a power of two below the row's sum), so that
        // its product with a number's 24 bits is one of 127
        const Two unit = {(float)exp2(-std::ilogb((double)exact) - 1), 0.0f};
        const Weight h = weight_of(times(exp_two(3.0f, 3.0f, 1.0f, table), unit));
        const Weight w = weight_of(times(exp_two(3.0f - gap, 3.0f, 1.0f, table), unit));
        const Wide head = wide(h.whole, h.rest), tail = wide(w.whole, w.rest), total = head + N * tail;
        for (int first = 0; first < 2; ++first)
            for (int k = 0; k < 4000; ++k) {
                const long double place = U(g) * N * t + (first ? 1 : 0);
                const float v = (float)(place / exact);
                const long double j = ((long double)v * exact - (first ? 1 : 0)) / t;
                if (!(v < 1) || j < 0 || j >= N || fabsl(j - rintl(j)) < ldexpl(N, -38)) continue;
                ++seen;
                const Wide at = share_of_total(v, total) - (first ? head : 0);
                if (at < 0 || at / tail != (Wide)floorl(j)) ++wrong;
            }
    }
    for (int k = 0; k < 400000; ++k) {
        // terms down to 2^-60, the numbers made of them
        const float z = (float)(-41.0 * U(g));
        const Two t = exp_two(z, 0.0f, 1.0f, table), b = exp_two(z - (float)U(g) * 1e-4f, 0.0f, 1.0f, table);
        rel = fmax(rel, (double)fabsl(((long double)t.hi + (long double)t.lo) / expl(z) - 1));
        for (const Two x : {t, less_by(t, b), less_by(b, t), times(t, {0.3f, 1e-9f})}) {
            const Weight w = weight_of(x);
            const long double want = fmaxl((long double)x.hi + (long double)x.lo, 0);
            // (the second float's own bits below 2^-92 at most)
            weight_off = fmax(weight_off, (double)fabsl(ldexpl((long double)w.whole, -46) + ldexpl((long double)w.rest, -92) - want));
            if (w.whole < 0 || w.rest < 0 || w.rest > REST) weight_off = 1;
        }
    }
    printf("%.17g %.17g %.17g %ld %ld\n", sum_off, rel, weight_off, wrong, seen);
}
"""


@pytest.fixture(scope="module")
def measured(tmp_path_factory):
    text = open(os.path.join(CSRC, "verify.cu")).read()
    code = text[text.index("constexpr double LN2_D"):text.index("// How far from its token's borders")]
    code = re.sub(r"__device__ const", "static const", code)
    d = tmp_path_factory.mktemp("sums")
    (d / "sums.cpp").write_text(SHIM + code + MAIN)
    subprocess.run(["g++", "-std=c++17", "-O2", "-ffp-contract=off", "-w", str(d / "sums.cpp"), "-o", str(d / "sums")], check=True)
    out = subprocess.run([str(d / "sums")], check=True, capture_output=True, text=True).stdout
    return [float(x) for x in out.split()]


def test_sums_of_equal_tails(measured):
    assert measured[0] <= 2.0 ** -40


def test_terms_of_any_size(measured):
    # the argument's last digits count with its size: 41 * 2^-48 beside the terms' own
    assert measured[1] <= 2.0 ** -40


def test_weights_are_the_terms(measured):
    # half a unit of 2^-92, as much for the last remainder as a float, and (long double) 2^-64 of a term of 1 at most
    assert measured[2] <= 2.0 ** -64 + 2.0 ** -91


def test_draws_from_equal_tails(measured):
    wrong, seen = measured[3:]
    assert seen >= 30_000 and wrong == 0
