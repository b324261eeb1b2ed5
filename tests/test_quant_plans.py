"""How attention over 8-bit rows, in windows and of drafts falls into blocks, in the library's own functions compiled for the host: every plan has a kernel, its runs have room in the
workspace that a handle makes for them, and making one goes through few of them."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

SWEEP = r"""
#include "sight_plan.hpp"
#include <cstdio>
#include <new>
namespace ctkvr {
int fail(int code, const char *, ...) { return code; }
bool device_idle() { return true; }
int pool_get(int, size_t, size_t, PoolBlock *) { return 0; }
void pool_put(int, PoolBlock, bool) {}
}
using namespace ctkvr;
#define WANT(x) do { if (!(x)) { printf("failed: %s; batch %d, %d heads on %d, %d pages, dtype %d, max_new %d: total %d, keys %lld, form %d\n", #x, batch, g * G, g, pages, dtype, \
                                        max_new, total, (long long)keys, form); return 1; } } while (0)
int main()
{
    for (int dtype : {CTKVR_F32, CTKVR_BF16}) for (int batch : {1, 2, 3, 8, 16, 65, 1000}) for (int g : {1, 2, 8, 40}) for (int G : {1, 2, 4, 8})
    for (int pages : {1, 40, 255, 256, 1000, 2048, 1 << 16}) for (int max_new : {1, 17, 300, 5000, 40000}) {
        alignas(16) static char mem[sizeof(ctkvr_cache)];   // (never destroyed: it has no memory)
        ctkvr_cache *c = new (mem) ctkvr_cache();
        c->p.batch = batch; c->p.n_kv_heads = g; c->p.n_q_heads = g * G; c->p.page_size = 16; c->p.max_pages = pages; c->p.dtype = dtype; c->p.max_new = max_new;
        c->G = G; c->lg = __builtin_ctz(G);
        const int64_t slots = 16ll * pages;
        const Room room = sight_room(c);
        int total = 0, form = 0;
        int64_t keys = 0;
        WANT(room.rows * 516 <= 72500000 + (size_t)max_new / 16 * g * G);   // (what the header says of a handle's memory; a sixteenth of a token's rows more)
        for (total = 1; total <= max_new; total += total < 400 ? 1 : total / 97)
            for (int64_t span : {slots, slots / 2, (int64_t)5000, (int64_t)4096, (int64_t)4095, (int64_t)700, (int64_t)1})
                for (form = 0; form < 4; ++form) {
                    keys = std::min(span, slots);
                    const bool codes = form & 1, window = form & 2;
                    SightPlan p = sight_plan(c, total, keys, codes, window);
                    if (dtype == CTKVR_BF16) WANT(p.log == 4 || p.log == 5 || p.log == 7 || (p.log == 8 && (codes || !window)));
                    else WANT(p.log == (codes ? 4 : 5) || p.log == 7);
                    WANT(p.nsplit >= 1 && p.nsplit <= kMaxSplit && (int64_t)p.tiles * g * p.nsplit < (1ll << 31));
                    // a tile for every row, however the tokens fall to the sequences
                    const int used = std::min(total, batch);
                    int64_t tiles = 0;
                    for (int b = 0; b < used; ++b) tiles += ((b ? 1ll : total - used + 1) * G + (1 << p.log) - 1) >> p.log;
                    WANT(p.tiles >= tiles);
                    tiles = 0;
                    for (int b = 0; b < used; ++b) tiles += ((int64_t)((total + b) / used) * G + (1 << p.log) - 1) >> p.log;
                    WANT(p.tiles >= tiles);
                    const SightPlan before = p;
                    fit_plan(c, total, room, p);
                    WANT(p.nsplit == before.nsplit && (p.nsplit == 1 || p.join_inside == before.join_inside));
                    // ... and in one that is too small, or none
                    const Room less{(size_t)total * g * G * 3 / 2, 0};
                    for (const Room &r : {less, Room{0, 0}}) {
                        fit_plan(c, total, r, p);
                        WANT(p.nsplit == 1 && !p.join_inside);
                    }
                }
    }
    printf("ok\n");
}
"""


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
def test_plans_have_kernels_and_room(tmp_path):
    src, exe = tmp_path / "host.hip", tmp_path / "host"
    src.write_text(SWEEP)
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", "--cuda-host-only", "-std=c++17", "-O2", "-I", os.path.join(ROOT, "paper_2512_15550_amd", "csrc"),
                        "-o", str(exe), str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout + r.stderr


CREATION = r"""
import sys, time
from tests.host_runtime.cache_scenarios import Host
x = Host(sys.argv[1])
for geometry in (dict(batch=2, n_q_heads=1, n_kv_heads=1, max_pages=2048), dict(batch=1, n_q_heads=32, n_kv_heads=8, max_pages=2048),
                 dict(batch=16, n_q_heads=8, n_kv_heads=1, max_pages=1 << 16)):
    least = 1e9
    for _ in range(10):
        t = time.perf_counter()
        c = x.create(max_new=32768, **geometry)
        least = min(least, time.perf_counter() - t)
        x.lib.ctkvr_cache_free(c)
    print(geometry, f"{least * 1e6:.0f} us")
    assert least < 1.5e-3
print("ok")
"""


def test_a_handle_is_made_in_little_time(tmp_path):
    """On the host, with a runtime whose calls take none: not by going through every number of tokens, which takes up to 8 ms."""
    lib = str(tmp_path / "libfake_hip.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", lib, os.path.join(ROOT, "tests", "host_runtime", "fake_hip.cpp")], check=True)
    r = subprocess.run([sys.executable, "-c", CREATION, lib], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.endswith("ok\n"), r.stdout + r.stderr
