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
