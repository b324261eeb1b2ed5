"""The operators on the paged KV cache without a GPU: refusals and devices, against the stand-in for the HIP runtime (host_runtime/), and
what the kernels make of page ids and lengths that make no sense, in their own functions compiled for the host."""
import os
import subprocess
import sys

import pytest

from tests.host_runtime.cache_scenarios import SCENARIOS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("fake_hip") / "libfake_hip.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", lib, os.path.join(ROOT, "tests", "host_runtime", "fake_hip.cpp")],
                   check=True)
    return lib


@pytest.mark.parametrize("name", SCENARIOS)
def test_host_code(fake, name):
    r = subprocess.run([sys.executable, "-m", "tests.host_runtime.cache_scenarios", name, fake], cwd=ROOT, capture_output=True, text=True,
                       timeout=120)
    assert r.returncode == 0 and r.stdout.endswith("ok\n"), r.stdout + r.stderr


PROGRAM = r"""
#include "cache_args.hpp"
#include <cstdio>
#include <initializer_list>
using namespace ctkvr;
#define WANT(x) do { if (!(x)) { printf("failed: %s\n", #x); return 1; } } while (0)
int main()
{
    const int32_t table[8] = {3, -1, INT32_MIN, INT32_MAX, 4, 5, 0, 2};
    int32_t cu[3] = {0, 5, 9}, cur[2] = {20, 60};
    CacheView v{};
    v.table = table; v.cu = cu; v.cur = cur; v.batch = 2; v.h = 4; v.g = 2; v.lg = 1; v.page_shift = 4; v.max_pages = 4; v.total = 9; v.num_pages = 5;
    // pages 0 .. 4 are there
    WANT(cache_row(v, 0, 1, 7) == ((3 * 2 + 1) << 4) + 7);
    for (int t : {16, 31, 32, 47, 48, 63}) WANT(cache_row(v, 0, 0, t) == -1);
    WANT(cache_row(v, 1, 0, 15) == ((4 * 2) << 4) + 15);
    WANT(cache_row(v, 1, 0, 16) == -1 && cache_row(v, 1, 1, 32) == 16 && cache_row(v, 1, 0, 63) == ((2 * 2) << 4) + 15);
    v.num_pages = 1u << 30;
    int32_t far[1] = {(1 << 30) - 1};
    v.table = far; v.max_pages = 1;
    WANT(cache_row(v, 0, 1, 15) == ((((int64_t)1 << 30) - 1) * 2 + 1) * 16 + 15);
    v.table = table; v.max_pages = 4; v.num_pages = 5;
    // lengths and token ranges: always inside the arrays
    SeqSpan s = seq_span(v, 1);
    WANT(s.c0 == 5 && s.n == 4 && s.len == 60 && s.old == 56);
    const int odd[] = {INT32_MIN, -1, 0, 1, 8, 9, 10, 1 << 30, INT32_MAX};
    for (int a : odd) for (int b : odd) for (int c : odd) {
        cu[0] = a; cu[1] = b; cur[0] = c;
        s = seq_span(v, 0);
        WANT(s.c0 >= 0 && s.n >= 0 && s.c0 + s.n <= v.total && s.len >= 0 && s.len <= 64);
        ScoreOpts o{};
        int32_t first[9];
        for (int f : odd) for (int prefix : {0, 7, 64}) {
            for (int32_t &x : first) x = f;
            o.first = first;
            for (int i = 0; i < s.n; ++i) {
                const RowSight r = row_sight(v, o, s, prefix < s.len ? prefix : s.len, i);
                WANT(r.lo >= 0 && r.hi >= 0 && r.hi <= s.len && (r.pos >= 0 || r.hi == 0));
            }
        }
    }
    printf("ok\n");
}
"""


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
def test_page_ids_and_lengths_that_make_no_sense(tmp_path):
    src, exe = tmp_path / "host.hip", tmp_path / "host"
    src.write_text(PROGRAM)
    subprocess.run([HIPCC, "--offload-arch=gfx950", "--cuda-host-only", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2512_15550_amd", "csrc"),
                    "-o", str(exe), str(src)], check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout + r.stderr


TURNS = r"""
#include "cache_args.hpp"
#include <cstdio>
#include <cstdlib>
#include <cstring>
int main(int n, char **args)
{
    for (int i = 1; i < n; ++i) {   // frequencies, and bases with the pair's number
        const char *pair = strchr(args[i], ':');
        const long double f = pair ? ctkvr::rope_freq(strtod(args[i], nullptr), atoi(pair + 1)) : (long double)strtod(args[i], nullptr);
        printf("%llu\n", (unsigned long long)ctkvr::turn_of(f));
    }
}
"""


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
def test_frequencies_as_fractions_of_a_turn(tmp_path):
    """Against 150 digits: off by one of 2^-64 for a given frequency, 1.25 for one of a base (powl is off by 2^-63 of it at most, a sixth of a turn)."""
    from decimal import Decimal as D, localcontext
    src, exe = tmp_path / "turns.hip", tmp_path / "turns"
    src.write_text(TURNS)
    subprocess.run([HIPCC, "--offload-arch=gfx950", "--cuda-host-only", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2512_15550_amd", "csrc"),
                    "-o", str(exe), str(src)], check=True, capture_output=True)
    given = [0.0, 1.0, -1.0, 0.1, 7.5, -3.7, 6.283185307179586, 3.141592653589793, 1e6 + 0.1, 123456789.123, -987654321.25, 2.0 ** 31 + 0.5, 2.0 ** 32,
             1e-9, 1e-30, 5e-324, -1e-25] + [10000.0 ** (-i / 64) for i in range(64)]
    bases = [(base, i) for base in (10000.0, 500000.0, 1e6, 1.0, 3.5) for i in range(64)]
    r = subprocess.run([str(exe)] + [x.hex() for x in given] + [f"{x.hex()}:{i}" for x, i in bases], capture_output=True, text=True, timeout=60)
    got = [int(x) for x in r.stdout.split()]
    assert r.returncode == 0 and len(got) == len(given) + len(bases)
    with localcontext() as ctx:
        ctx.prec = 150
        a, b, t, p = D(1), 1 / D(2).sqrt(), D(1) / 4, D(1)
        for _ in range(8):                                  # pi by the arithmetic-geometric mean
            mean = (a + b) / 2
            b, t, a, p = (a * b).sqrt(), t - p * (a - mean) ** 2, mean, 2 * p
        two_pi = (a + b) ** 2 / (2 * t)
        want = [(D(f), D(1)) for f in given] + [(D(base) ** (D(-i) / 64), D("1.25")) for base, i in bases]
        for (f, most), u in zip(want, got):
            off = f / two_pi * 2 ** 64 - u
            off -= (off / 2 ** 64).to_integral_value() * 2 ** 64
            assert abs(off) <= most, (f, u, off)
